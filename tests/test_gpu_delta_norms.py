"""The gated delta rule (csrc/k_delta.hip, csrc/k_delta_grad.hip) to the precision that include/sf_memory.h states, by the norms of its errors for
each row and head; limits are those of tests/delta_norms.py."""
import pytest

from tests import delta_norms as norms, delta_reference as ref
from tests.test_gpu_delta import call, step

pytestmark = pytest.mark.gpu


def both(x, do, ds, dk, dv, dtype, scale=None, length=17.0):
    T = x["q"].shape[0]
    norms.check(call(x, scale=scale), ref.oracle(x, scale)[0], dk, dv, length, dtype == "bf16", T)
    norms.check(call(x, do, ds, scale=scale), ref.oracle(x, scale, do, ds)[0], dk, dv, length, dtype == "bf16", T)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (8, 8), (40, 72), (72, 40), (127, 65), (64, 128)])
@pytest.mark.parametrize("T", [1, 2, 17, 32, 33, 64, 70, 333])
def test_lengths_and_head_sizes(torch_cuda, T, dk, dv, dtype):
    x, do, ds = ref.make(T, 3, 2, 2, dk, dv, dtype, seed=T + dk, p_done=0.05)
    both(x, do, ds, dk, dv, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (24, 8)])
@pytest.mark.parametrize("T", [30, 200])
def test_shared_heads(torch_cuda, T, H, Hk, dtype):
    x, do, ds = ref.make(T, 3, H, Hk, 48, 32, dtype, seed=H)
    both(x, do, ds, 48, 32, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv,H,Hk,p_done", [(64, 64, 3, 1, 0.0), (128, 128, 2, 1, 0.01), (40, 72, 2, 2, 0.001), (128, 40, 1, 1, 0.0)])
def test_pieces(torch_cuda, dk, dv, H, Hk, p_done, dtype):
    """Few heads and a long axis: T is cut; the last chunk is not whole."""
    x, do, ds = ref.make(1100, 2, H, Hk, dk, dv, dtype, seed=dk, p_done=p_done)
    both(x, do, ds, dk, dv, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_long_memory(torch_cuda, dtype):
    """Of up to 300 steps, across pieces."""
    x, do, ds = ref.make(2000, 1, 2, 1, 64, 64, dtype, seed=9, p_done=0.0, memory=300.0)
    both(x, do, ds, 64, 64, dtype, length=301.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 128), (40, 72)])
def test_many_heads_with_wide_values(torch_cuda, dk, dv, dtype):
    x, do, ds = ref.make(70, 64, 8, 8, dk, dv, dtype, seed=dv)
    both(x, do, ds, dk, dv, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (40, 72), (128, 128)])
def test_steps_on_a_table(torch_cuda, dk, dv, dtype):
    torch = torch_cuda
    x, _, _ = ref.make(40, 5, 2, 2, dk, dv, dtype, seed=dk)
    table = x["state0"].clone()
    got = dict(o=torch.stack([step(x, t, table, None) for t in range(40)]), state=table)
    norms.check(got, ref.oracle(x)[0], dk, dv, 17.0, dtype == "bf16", 40)
