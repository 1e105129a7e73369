"""The gated feed-forward block (csrc/k_ffn.hip) against its definition in 64 bits.

Tolerances.  Each result is a sum; with A the sum of its terms' magnitudes, every element may be off by c A + 2^-8 |y| (bf16)
or c A (fp32).  c: the inner numbers h, dg, du are rounded to bf16 once, 2^-8 of themselves (bf16 only), and come with the
rounding of their own sums, which is bounded by n 2^-24 of the magnitudes in them; those magnitudes are at most a factor
G above the number itself on average, taken as 16 at these sizes (sums of K random terms: sqrt(K) = 55 at most, with
sqrt(K) of the worst case n for random signs).  So c = 2^-8 (bf16) + 2^-24 (D + F + M) in both.  That bound is wide for a
sum of random signs, so a result of 4096 numbers or more is held to more: its error's norm over its norm is the root mean
square of the roundings: bf16 two of 2^-8 / sqrt(3) each, below 2^-8; fp32 2^-24 sqrt(n) for each of the two sums, with a
factor of 2.  (Of a handful of numbers no mean can be taken: one alone may be off by 2^-7.)
"""
import pytest

pytestmark = pytest.mark.gpu


def act(a, name):
    import math
    import torch
    if name == "gelu":
        return a * 0.5 * torch.erfc(-a / math.sqrt(2.0))
    s = 1 / (1 + torch.exp(-a))
    return s if name == "sigmoid" else a * s


def oracle(x, wg, wu, wd, name, dy=None):
    import torch
    leaf = [a.double().requires_grad_() for a in (x, wg, wu, wd)]
    h = act(leaf[0] @ leaf[1].T, name) * (leaf[0] @ leaf[2].T)
    y = h @ leaf[3].T
    hm = h.detach().abs()
    got, size = dict(y=y.detach()), dict(y=hm @ leaf[3].detach().abs().T)
    if dy is not None:
        dy = dy.double()
        with torch.no_grad():
            g = leaf[0] @ leaf[1].T
            u = leaf[0] @ leaf[2].T
            dh = dy @ leaf[3]
        gg = g.clone().requires_grad_()
        slope, = torch.autograd.grad(act(gg, name).sum(), gg)
        dg, du = (dh * u * slope).abs(), (dh * act(g, name)).abs()
        a = [t.detach().abs() for t in leaf]
        for n, t in zip(("dx", "dw_gate", "dw_up", "dw_down"), torch.autograd.grad((y * dy).sum(), leaf)):
            got[n] = t
        size.update(dx=dg @ a[1] + du @ a[2], dw_gate=dg.T @ a[0], dw_up=du.T @ a[0], dw_down=dy.abs().T @ hm)
    return got, size


def make(torch, M, D, F, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    return [r(M, D).to(dt), (r(F, D) / D ** 0.5).to(dt), (r(F, D) / D ** 0.5).to(dt), (r(D, F) / F ** 0.5).to(dt)], r(M, D).to(dt)


def check(got, want, size, dtype, n, root):
    for name, y in want.items():
        x = got[name].double()
        assert x.shape == y.shape, name
        if not y.numel():
            continue
        c = n * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        tol = c * size[name] + (2.0 ** -8 * y.abs() if dtype == "bf16" else 0.0) + 1e-30
        over = ((x - y).abs() / tol).max().item()
        assert over <= 1.0, "%s: %.2f of the tolerance" % (name, over)
        rel = ((x - y).norm() / y.norm()).item()
        assert y.numel() < 4096 or rel <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23 * root), "%s: off by %.3g" % (name, rel)


def both(torch, ws, dy, dtype, name="silu"):
    from paper_2006_11751_amd import memory
    got = dict(memory.gated_ffn(*ws, act=name))
    got.update(memory.gated_ffn_backward(*ws, dy, act=name))
    torch.cuda.synchronize()
    (M, D), F = ws[0].shape, ws[1].shape[0]
    want, size = oracle(*ws, name, dy)
    check(got, want, size, dtype, D + F + M, D ** 0.5 + F ** 0.5 + M ** 0.5)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [1, 2, 13, 16, 17, 33, 63, 64, 65, 100, 129, 300])
def test_rows(torch_cuda, M, dtype):
    ws, dy = make(torch_cuda, M, 128, 320, dtype, seed=M)
    both(torch_cuda, ws, dy, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [5, 70])
@pytest.mark.parametrize("D,F", [(1, 1), (8, 8), (64, 64), (72, 40), (65, 130), (100, 1), (1, 100), (37, 501), (200, 129), (512, 1365)])
def test_widths(torch_cuda, M, D, F, dtype):
    ws, dy = make(torch_cuda, M, D, F, dtype, seed=D + F)
    both(torch_cuda, ws, dy, dtype, "gelu")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,D,F", [(4100, 200, 3000), (4100, 2900, 72), (130, 2000, 2100), (1000, 512, 2048)])
def test_large_tiles(torch_cuda, M, D, F, dtype):
    ws, dy = make(torch_cuda, M, D, F, dtype, seed=1)
    both(torch_cuda, ws, dy, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("M", [9, 150])
def test_activations(torch_cuda, M, name, dtype):
    ws, dy = make(torch_cuda, M, 64, 192, dtype, seed=4)
    both(torch_cuda, ws, dy, dtype, name)


@pytest.mark.parametrize("name", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("M", [9, 150])
def test_far_tails_of_the_activation(torch_cuda, M, name):
    """Gates from -60 to 60: one input column, so that g is the weight itself."""
    torch = torch_cuda
    F = 121
    x = torch.ones(M, 1, device="cuda")
    wg = torch.linspace(-60, 60, F, device="cuda")[:, None].contiguous()
    ws = [x, wg, torch.ones(F, 1, device="cuda"), torch.eye(1, F, device="cuda")]
    from paper_2006_11751_amd import memory
    for i in range(0, F, 10):
        ws[3] = torch.zeros(1, F, device="cuda")
        ws[3][0, i] = 1.0
        y = memory.gated_ffn(*ws, act=name)["y"].double()
        want = act(wg[i].double(), name)
        assert ((y - want).abs() <= 2.0 ** -20 * want.abs() + 1e-37).all(), (i, y[0, 0], want)
        back = memory.gated_ffn_backward(*ws, torch.ones(M, 1, device="cuda"), act=name)
        g = wg.double().requires_grad_()
        slope, = torch.autograd.grad(act(g, name)[i].sum(), g)
        assert torch.isfinite(back["dw_gate"]).all()
        # (a difference of numbers of size |g| at most)
        assert ((back["dw_gate"].double() - M * slope).abs() <= M * 2.0 ** -20 * (slope.abs() + 2.0 ** -3)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [20, 150])
def test_strides_and_alignment(torch_cuda, M, dtype):
    torch = torch_cuda
    ws, dy = make(torch, M, 128, 192, dtype, seed=6)
    a = both(torch, ws, dy, dtype)
    gu = torch.stack([ws[1], ws[2]], 1)  # one array of both projections
    wide = torch.zeros(M, 301, dtype=dy.dtype, device="cuda")
    wide[:, 3:131], wide[:, 140:268] = ws[0], dy
    flat = torch.empty(128 * 192 + 1, dtype=dy.dtype, device="cuda")[1:].view(128, 192)
    b = both(torch, [wide[:, 3:131], gu[:, 0], gu[:, 1], flat.copy_(ws[3])], wide[:, 140:268], dtype)
    for n in a:
        assert n == "workspace" or torch.equal(a[n], b[n]), n
    from paper_2006_11751_amd import memory
    c = memory.gated_ffn(ws[0].unflatten(0, (M // 5, 5)), *ws[1:])["y"]
    assert c.shape == (M // 5, 5, 128) and torch.equal(c.flatten(0, 1), a["y"])


def test_no_rows(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    ws, dy = make(torch, 0, 64, 100, "bf16")
    assert memory.gated_ffn(*ws)["y"].shape == (0, 64)
    out = dict(dw_gate=torch.ones(100, 64, dtype=torch.bfloat16, device="cuda"))
    memory.gated_ffn_backward(*ws, dy, out=out)
    assert not out["dw_gate"].any() and not out["dw_up"].any() and not out["dw_down"].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [20, 200])
def test_a_row_that_is_not_finite_stays_a_row(torch_cuda, M, dtype):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    ws, dy = make(torch, M, 64, 128, dtype, seed=7)
    clean, cback = memory.gated_ffn(*ws)["y"], memory.gated_ffn_backward(*ws, dy)["dx"]
    ws[0][3, 5], ws[0][M - 1, 0], ws[0][7, 1] = float("nan"), float("inf"), float("-inf")
    got, back = memory.gated_ffn(*ws)["y"], memory.gated_ffn_backward(*ws, dy)["dx"]
    keep = [r for r in range(M) if r not in (3, 7, M - 1)]
    assert torch.equal(got[keep], clean[keep]) and torch.equal(back[keep], cback[keep])
    for r in (3, 7, M - 1):
        assert not torch.isfinite(got[r]).any()


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_gradients_against_differences(torch_cuda, which):
    """Central differences of the kernel's own fp32 results, h = 2^-6 along a random direction: h^2 of the third derivative,
    and 2^-23 / h of the size in rounding."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    ws, dy = make(torch, 90, 48, 80, "fp32", seed=9)
    f = lambda z: (memory.gated_ffn(*z)["y"].double() * dy.double()).sum()
    grad = memory.gated_ffn_backward(*ws, dy)[("dx", "dw_gate", "dw_up", "dw_down")[which]].double()
    way = torch.randn(ws[which].shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    way = way / way.norm() * ws[which].norm()
    h = 2.0 ** -6
    at = lambda s: [a + s * way if i == which else a for i, a in enumerate(ws)]
    want = (grad * way.double()).sum()
    assert abs((f(at(h)) - f(at(-h))) / (2 * h) - want) <= 2e-3 * grad.norm() * way.norm() / 8


def test_same_bits_on_another_stream_and_in_a_graph(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    for M in (30, 700):
        ws, dy = make(torch, M, 192, 500, "bf16", seed=2)
        run = lambda a, b: (memory.gated_ffn(*ws, out=a), memory.gated_ffn_backward(*ws, dy, out=b))
        first = [{k: t.clone() for k, t in r.items() if k != "workspace"} for r in run({}, {})]
        same = lambda a, b: all(torch.equal(r[k], f[k]) for r, f in zip((a, b), first) for k in f)
        side, a, b = torch.cuda.Stream(), {}, {}
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(a, b)
        torch.cuda.synchronize()
        assert same(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(a, b)
        for _ in range(3):
            for r in (a, b):
                for t in r.values():
                    t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same(a, b)


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    (x, wg, wu, wd), dy = make(torch, 4, 32, 48, "fp32")
    base = dict(x=x, w_gate=wg, w_up=wu, w_down=wd)
    for bad in (dict(x=x.double()), dict(x=x.cpu()), dict(x=x[:, :16]), dict(w_gate=wg.bfloat16()), dict(w_up=wu[:4]), dict(w_down=wd.T),
                dict(w_down=wg), dict(act="relu"), dict(out=dict(y=x[:2])), dict(w_gate=wg[0])):
        with pytest.raises(ValueError):
            memory.gated_ffn(**dict(base, **bad))
    with pytest.raises(ValueError):
        memory.gated_ffn_backward(dy=dy[:2], **base)
    with pytest.raises(ValueError):
        memory.gated_ffn_backward(dy=dy, out=dict(dw_up=wd), **base)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,D,F", [(500, 130, 1150), (1030, 120, 1000), (700, 100, 2100), (1024, 64, 1024)])
def test_tiles_on_both_sides_of_one_round(torch_cuda, M, D, F, dtype):
    ws, dy = make(torch_cuda, M, D, F, dtype, seed=2)
    both(torch_cuda, ws, dy, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("M,D,F", [(20, 64, 72), (150, 64, 8), (150, 64, 72), (150, 100, 200), (200, 128, 192), (2100, 128, 1288)])
def test_what_lies_between_rows_is_not_read_as_numbers(torch_cuda, M, D, F, name, dtype):
    """Arrays whose rows are farther apart than they are long, NaN and infinities between them: the dense call's bits."""
    torch = torch_cuda
    ws, dy = make(torch, M, D, F, dtype, seed=8)
    dense = both(torch, ws, dy, dtype, name)

    def gaps(a):
        wide = torch.full((a.shape[0], (a.shape[1] + 64) // 64 * 64 + 64), float("nan"), dtype=a.dtype, device="cuda")
        wide[1::2] = float("inf")
        wide[:, :a.shape[1]] = a
        return wide[:, :a.shape[1]]

    for which in ((3,), (0, 1, 2, 3, 4)):  # w_down alone (F a multiple of 8 but not of 64 is read where it is), all of them
        arrays = [gaps(a) if i in which else a for i, a in enumerate(ws + [dy])]
        got = both(torch, arrays[:4], arrays[4], dtype, name)
        for n in dense:
            assert n == "workspace" or torch.equal(got[n], dense[n]), n
