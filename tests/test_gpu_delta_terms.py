"""What bf16 results of the gated delta rule leave out of the fp32 numbers that enter their last products: 2^-16 of each (include/sf_memory.h).

Each result here is one product of such numbers, and another one that takes nearly all of it away again and whose factors are of 8 and 16
significant bits, which two bf16 terms hold: nothing is left out of that one.  What is left is so small that its own rounding does not hide
what was left out of the first product, 2^-16 of each of its factors that is an fp32 number; 2^-20 of both are for roundings in fp32.
"""
import pytest

from tests.test_gpu_delta import call

pytestmark = pytest.mark.gpu

N, DV = 256, 64


def two_terms(torch, x):
    """The nearest number of 16 significant bits."""
    a = x.double()
    unit = torch.exp2(torch.floor(torch.log2(a.abs())) - 15)
    return (a / unit).round() * unit


def check(got, want, first, factors):
    """first: the size of the first product; factors: of them, how many are fp32 numbers."""
    tol = (factors * 2.0 ** -16 + 2.0 ** -19) * first.abs() + 2.0 ** -8 * want.abs()
    part = ((got.double() - want).abs() / tol).max().item()
    assert part <= 1.0, "%.2f of the tolerance" % part


def inputs(torch, T, dk, seed):
    """All zero but the decays, which are one; a generator of numbers between one and two."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: 1.0 + torch.rand(s, generator=g, device="cuda")
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")
    f = torch.float32
    x = dict(q=z(T, N, 1, dk), k=z(T, N, 1, dk), v=z(T, N, 1, DV), log_decay=z(T, N, 1, dtype=f), beta=z(T, N, 1, dtype=f),
             done=z(T, N, dtype=torch.uint8), state0=z(N, 1, dk, DV, dtype=f))
    return x, r, z(T, N, 1, DV), z(N, 1, dk, DV, dtype=f)


@pytest.mark.parametrize("T", [2, 40, 1100])
@pytest.mark.parametrize("dk", [64, 128])
def test_o_of_the_state(torch_cuda, T, dk):
    torch = torch_cuda
    x, r, _, _ = inputs(torch, T, dk, 1)
    x["q"][T - 1, :, 0, 0] = r(N).bfloat16()
    x["q"][T - 1, :, 0, 1] = -1
    s = r(N, DV)
    x["state0"][:, 0, 0] = s
    first = x["q"][T - 1, :, 0, :1].double() * s.double()
    x["state0"][:, 0, 1] = two_terms(torch, first).float()
    got = call(x, scale=1.0)["o"][T - 1, :, 0]
    check(got, first - x["state0"][:, 0, 1].double(), first, 1)


@pytest.mark.parametrize("T", [2, 40, 1100])
@pytest.mark.parametrize("dk", [64, 128])
def test_o_of_the_chunk(torch_cuda, T, dk):
    """Two steps with keys at right angles: the first one's correction and P are fp32 numbers."""
    torch = torch_cuda
    x, r, _, _ = inputs(torch, T, dk, 2)
    a, b = T - 2, T - 1
    x["k"][a, :, 0, 0], x["k"][b, :, 0, 1] = r(N).bfloat16() / 2, 1
    x["q"][b, :, 0, 0], x["q"][b, :, 0, 1] = r(N).bfloat16(), -1
    x["beta"][a, :, 0], x["beta"][b, :, 0] = r(N) / 2, 1
    x["v"][a, :, 0] = r(N, DV).bfloat16()
    p = x["q"][b, :, 0, 0].double() * x["k"][a, :, 0, 0].double()
    u = (x["beta"][a] * x["v"][a, :, 0].float()).double()  # (rounded to fp32, as the definition's first step is in any order: it is one product)
    first = p[:, None] * u
    x["v"][b, :, 0] = first.bfloat16()
    got = call(x, scale=1.0)["o"][b, :, 0]
    check(got, first - x["v"][b, :, 0].double(), first, 2)


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("dk", [64, 128])
def test_dq_of_the_state(torch_cuda, T, dk):
    torch = torch_cuda
    x, r, do, ds = inputs(torch, T, dk, 3)
    do[T - 1, :, 0, 0], do[T - 1, :, 0, 1] = r(N).bfloat16(), -1
    s = r(N, dk)
    x["state0"][:, 0, :, 0] = s
    first = do[T - 1, :, 0, :1].double() * s.double()
    x["state0"][:, 0, :, 1] = two_terms(torch, first).float()
    got = call(x, do, ds, scale=1.0)["dq"][T - 1, :, 0]
    check(got, first - x["state0"][:, 0, :, 1].double(), first, 1)


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("dk", [64, 128])
def test_dk_of_the_state_behind(torch_cuda, T, dk):
    """u is of 16 bits: nothing of it is left out, but the product of what both leave behind their first 8."""
    torch = torch_cuda
    x, r, do, ds = inputs(torch, T, dk, 4)
    beta = r(N).bfloat16() / 2
    x["beta"][T - 1, :, 0] = beta.float()
    x["v"][T - 1, :, 0, 0], x["v"][T - 1, :, 0, 1] = r(N).bfloat16(), -1
    R = r(N, dk)
    ds[:, 0, :, 0] = R
    ds[:, 0, :, 1] = two_terms(torch, R.double() * x["v"][T - 1, :, 0, :1].double()).float()
    first = R.double() * (beta.double() * x["v"][T - 1, :, 0, 0].double())[:, None]
    got = call(x, do, ds, scale=1.0)["dk"][T - 1, :, 0]
    check(got, first - ds[:, 0, :, 1].double() * beta.double()[:, None], first, 2)
