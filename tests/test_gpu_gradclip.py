"""The global norm of a list of gradients and their clipping (csrc/k_gradclip.hip) against sums in 64 bits.

Tolerances.  Squares of fp32 numbers are exact in 64 bits and their sum is off by 2^-53 for each addition on the way, less than
2^-30 altogether here; so the norm is off by its rounding to 32 bits, 2^-24, and little more: 1.01 2^-24.  The factor is rounded once
(2^-24), its product with a gradient once (2^-24), and to bf16 once more (2^-8 of the result).  Results below 2^-126 may be zero.
"""
import pytest

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -126


def reference(grads, max_norm, eps=1e-6):
    import math
    norm = math.sqrt(math.fsum((g.double() ** 2).sum().item() for g in grads))
    return norm, min(1.0, max_norm / (norm + eps))


def check(torch, grads, got, max_norm, norm, eps=1e-6):
    want, by = reference(grads, max_norm, eps)
    assert norm.shape == (1,) and norm.dtype == torch.float32
    assert abs(norm.item() - want) <= 1.01 * 2.0 ** -24 * want + TINY
    for i, (g, c) in enumerate(zip(grads, got)):
        assert c.shape == g.shape and c.dtype == g.dtype
        y = g.double() * by
        tol = (2.01 * 2.0 ** -24 + (2.0 ** -8 * (1 + 2.0 ** -20) if g.dtype == torch.bfloat16 else 0.0)) * y.abs() + TINY
        assert ((c.double() - y).abs() <= tol).all(), i


def make(torch, sizes, kinds="fb", level=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    types = dict(f=torch.float32, b=torch.bfloat16)
    return [(level * torch.randn(s, generator=g, device="cuda")).to(types[kinds[i % len(kinds)]]) for i, s in enumerate(sizes)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e6, float("inf")])
@pytest.mark.parametrize("kinds", ["f", "b", "fb", "bbf"])
@pytest.mark.parametrize("sizes", [[1], [3, 1, 7, 8, 9], [(4, 5, 6), 0, (2, 0), 31], [16383, 16384, 16385], [100003, 5, 70001], [5] * 300, [0, 0]])
def test_lists(torch_cuda, sizes, kinds, max_norm, in_place):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    grads = make(torch, sizes, kinds)
    kept = [g.clone() for g in grads]
    out = memory.clip_gradients(grads, max_norm, in_place=in_place)
    check(torch, kept, grads if in_place else out["grads"], max_norm, out["norm"])
    assert ("grads" in out) != in_place
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(grads, kept))


def test_a_large_list(torch_cuda):
    """Chunks larger than the least one, 420 tensors in four launches, one of them far larger than the others."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    grads = make(torch, [40_000_003] + [1 + 997 * i % 30011 for i in range(419)], "bf", 0.01)
    out = memory.clip_gradients(grads, 1.0, in_place=False)
    check(torch, grads, out["grads"], 1.0, out["norm"])


@pytest.mark.parametrize("off_in,off_out", [(0, 1), (1, 0), (1, 2), (3, 3), (5, 7)])
@pytest.mark.parametrize("kind", ["f", "b"])
def test_any_alignment(torch_cuda, kind, off_in, off_out):
    """Tensors and results anywhere in larger buffers, whose other numbers stay as they are."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    buf, to = make(torch, [50021, 50021], kind, seed=off_in)
    before = to.clone()
    n = 40007
    out = dict(grads=[to[off_out:off_out + n]])
    memory.clip_gradients([buf[off_in:off_in + n]], 2.0, in_place=False, out=out)
    check(torch, [buf[off_in:off_in + n]], out["grads"], 2.0, out["norm"])
    assert torch.equal(to[:off_out], before[:off_out]) and torch.equal(to[off_out + n:], before[off_out + n:])


def test_other_orders_of_axes(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    a, b, c = make(torch, [(40, 70), (6, 5, 4, 3), (9, 8)], "f")
    grads = [a.T, b.contiguous(memory_format=torch.channels_last), c]
    out = memory.clip_gradients(grads, 1.0, in_place=False)
    check(torch, grads, out["grads"], 1.0, out["norm"])
    assert [g.stride() for g in out["grads"]] == [g.stride() for g in grads]
    with pytest.raises(ValueError, match="not dense"):
        memory.clip_gradients([a[:, ::2]], 1.0)
    with pytest.raises(ValueError, match="does not fit"):  # results in another order
        memory.clip_gradients(grads, 1.0, in_place=False, out=dict(grads=[a.T.contiguous(), grads[1], c]))


def test_sizes_that_leave_32_bits_when_squared(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    for level in (1e30, 1e-30):
        grads = make(torch, [1000, 77], "fb", level)
        out = memory.clip_gradients(grads, 2.0 * level, eps=1e-38, in_place=False)
        check(torch, grads, out["grads"], 2.0 * level, out["norm"], 1e-38)


def test_not_finite(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    for bad in (float("inf"), -float("inf"), float("nan")):
        for at in (0, 1):
            grads = make(torch, [100, 33], "fb")
            grads[at][17] = bad
            out = memory.clip_gradients(grads, 1.0, in_place=False)
            if bad != bad:
                assert out["norm"].isnan().all() and all(g.isnan().all() for g in out["grads"])
            else:
                assert torch.isinf(out["norm"]).all() and out["norm"] > 0
                for i, g in enumerate(out["grads"]):
                    g = g.float()
                    assert g.isnan().sum() == (i == at) and (g[~g.isnan()] == 0).all()


def test_clipped_twice_and_not_at_all(torch_cuda):
    """In place; a norm below the largest one leaves every bit."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    grads, out = make(torch, [5000, 301], "fb"), {}
    memory.clip_gradients(grads, 1.0, out=out)
    first = out["norm"].clone()
    kept = [g.clone() for g in grads]
    memory.clip_gradients(grads, 1.5, out=out)
    assert first > 60 and abs(out["norm"].item() - 1.0) < 2.0 ** -8
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))


def test_the_same_bits_each_time_in_a_graph_and_on_a_stream(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    made = make(torch, [70001, 13, 40000] + [50] * 200, "fb")
    grads = [g.clone() for g in made]
    want = memory.clip_gradients(grads, 1.0, in_place=False)
    out, side = {}, torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    memory.clip_gradients(grads, 1.0, in_place=False, out=out, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out["norm"], want["norm"]) and all(torch.equal(a, b) for a, b in zip(out["grads"], want["grads"]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        memory.clip_gradients(grads, 1.0, in_place=False, out=out)
    for i in range(4):
        for g, m in zip(grads, made):
            g.copy_(m * (i + 1))
        want = memory.clip_gradients(grads, 1.0, in_place=False)
        out["norm"].zero_()
        for g in out["grads"]:
            g.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["norm"], want["norm"]) and all(torch.equal(a, b) for a, b in zip(out["grads"], want["grads"]))


def test_tensors_may_be_dropped_right_after_a_call_on_another_stream(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    made = make(torch, [300000, 200001], "fb")
    want = memory.clip_gradients(made, 1.0, in_place=False)
    torch.cuda.synchronize()
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    torch.cuda.empty_cache()
    mine = [g.clone() for g in made]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(10):
            busy @ busy
    out = memory.clip_gradients(mine, 1.0, in_place=False, stream=side)
    del mine
    taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1200000, 400002, 512, 16384) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out["norm"], want["norm"]) and all(torch.equal(a, b) for a, b in zip(out["grads"], want["grads"]))
    del taken


def test_it_runs_on_its_tensors_device(torch_cuda, monkeypatch):
    """With another device current (there is one here: that it is another is pretended until torch is told to change to it)."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    grads = make(torch, [1000, 30], "fb")
    want = memory.clip_gradients(grads, 1.0, in_place=False)
    real, told = torch.cuda.device, []

    class device(real):
        def __init__(self, d):
            told.append(d)
            super().__init__(d)

    other = lambda: 0 if told else 1
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", other)
    monkeypatch.setattr(memory, "_current_device", other, raising=False)
    got = memory.clip_gradients(grads, 1.0, in_place=False)
    monkeypatch.undo()
    assert told == [grads[0].device] and torch.equal(got["norm"], want["norm"])


def test_tensors_of_no_numbers_beside_other_orders_of_axes(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    a, b = make(torch, [(40, 70), 31], "f")
    grads = [a.T, torch.zeros(2, 0, device="cuda"), b, torch.zeros(4, 6, device="cuda")[:, 3:3]]
    out = {}
    for _ in range(2):
        memory.clip_gradients(grads, 1.0, in_place=False, out=out)
        check(torch, grads, out["grads"], 1.0, out["norm"])
    kept = [g.clone() for g in grads]
    norm = memory.clip_gradients(grads, 1.0)["norm"]
    check(torch, kept, grads, 1.0, norm)


def test_results_of_another_shape_are_refused(torch_cuda):
    """Also where they have as many numbers, and are contiguous like the gradients."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    grads = make(torch, [(6, 4), 5], "f")
    for shape in ((4, 6), (24,), (6, 4, 1), (6, 5)):
        with pytest.raises(ValueError, match="does not fit"):
            memory.clip_gradients(grads, 1.0, in_place=False, out=dict(grads=make(torch, [shape, 5], "f")))
    out = dict(grads=make(torch, [(6, 4), 5], "f", seed=1))
    memory.clip_gradients(grads, 1.0, in_place=False, out=out)
    check(torch, grads, out["grads"], 1.0, out["norm"])


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n", [119, 120, 121, 4100, 20000])
def test_thousands_of_tensors(torch_cuda, n, in_place):
    """On both sides of what one launch takes, and so many that the chunks' sums are far more than a workgroup adds up in one round; the same bits
    each time and in a graph."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    sizes = [1 + 37 * i % 53 for i in range(n)]
    whole, = make(torch, [sum(sizes)], "f", seed=n)
    grads = list(whole.split(sizes))
    kept, out = whole.clone(), {}
    memory.clip_gradients(grads, 1.0, in_place=in_place, out=out)
    got = [whole if in_place else torch.cat(out["grads"])]
    check(torch, [kept], got, 1.0, out["norm"])
    first = out["norm"].clone(), got[0].clone()
    whole.copy_(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        memory.clip_gradients(grads, 1.0, in_place=in_place, out=out)
    for _ in range(3):
        whole.copy_(kept)
        out["norm"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["norm"], first[0]) and torch.equal(whole if in_place else torch.cat(out["grads"]), first[1])
