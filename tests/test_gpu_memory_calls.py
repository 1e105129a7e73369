"""What the binding of the memory operators does around a call (paper_2006_11751_amd/memory.py): numbers given as tensors,
the device, the stream, the results and the workspace that a program keeps.  Results are compared bit by bit."""
import pytest

pytestmark = pytest.mark.gpu


def _attention(torch, T=6, N=3, H=2, d=16, dtype=None):
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype or torch.float32)
    return r(T, N, H, d), r(T, N, H, d), r(T, N, H, d), torch.full((H,), -0.1, device="cuda")


def test_a_number_that_changes_in_place_is_read_at_every_call(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    args, b = _attention(torch), torch.randn(4, 32, device="cuda")
    do = torch.randn_like(args[2])
    scale, eps = torch.tensor(0.5), torch.tensor(1e-6)
    calls = (lambda: memory.linear_attention(*args, scale=scale)["o"], lambda: memory.linear_attention_backward(*args, do, scale=scale)["dq"],
             lambda: memory.linear_attention_step(*(a[0] for a in args[:3]), args[3], torch.zeros(3, 2, 16, 16, device="cuda"), scale=scale)["o"])
    before = [c() for c in calls]
    norm = [memory.residual_norm(b, eps=eps)["n"], memory.residual_norm_backward(b, b, b, eps=eps)["db"]]
    scale.fill_(1.0)
    eps.fill_(1.0)
    for c, was in zip(calls, before):
        assert torch.equal(c(), 2 * was)
    assert torch.equal(memory.residual_norm(b, eps=eps)["n"], memory.residual_norm(b, eps=1.0)["n"])
    assert torch.equal(memory.residual_norm_backward(b, b, b, eps=eps)["db"], memory.residual_norm_backward(b, b, b, eps=1.0)["db"])
    assert not torch.equal(memory.residual_norm(b, eps=eps)["n"], norm[0])


def _calls(torch, F=200):
    """Every function: f(tensors, **more) -> dict, and its tensors."""
    from paper_2006_11751_amd import memory
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k, v, ld = _attention(torch, T=700, dtype=torch.bfloat16)  # (cut into pieces: a workspace)
    do, table, b, w = torch.randn_like(v), torch.randn(3, 2, 16, 16, device="cuda"), r(300, 96), [r(300, 64), r(F, 64), r(F, 64), r(64, F)]
    return {
        "linear_attention": (lambda t, **m: memory.linear_attention(*t, **m), [q, k, v, ld]),
        "linear_attention_backward": (lambda t, **m: memory.linear_attention_backward(*t, **m), [q, k, v, ld, do]),
        "linear_attention_step": (lambda t, **m: memory.linear_attention_step(*t, **m), [q[0], k[0], v[0], ld, table]),
        "residual_norm": (lambda t, **m: memory.residual_norm(t[0], pre_w=t[1], **m), [b, b[0].clone()]),
        "residual_norm_backward": (lambda t, **m: memory.residual_norm_backward(*t[:3], pre_w=t[3], **m), [b, b, b, b[0].clone()]),
        "gated_ffn": (lambda t, **m: memory.gated_ffn(*t, **m), w),
        "gated_ffn_backward": (lambda t, **m: memory.gated_ffn_backward(*t, **m), w + [r(300, 64)]),
    }


NAMES = ("linear_attention", "linear_attention_backward", "linear_attention_step", "residual_norm", "residual_norm_backward", "gated_ffn",
         "gated_ffn_backward")


@pytest.mark.parametrize("name", NAMES)
def test_tensors_may_be_dropped_right_after_a_call_on_another_stream(torch_cuda, name):
    """The call waits behind other work of its stream, while the stream that is current takes all memory that has been let go
    of and writes to it."""
    torch = torch_cuda
    call, tensors = _calls(torch)[name]
    copy = lambda: [t.clone() for t in tensors]
    want = {n: t.clone() for n, t in call(copy()).items() if n != "workspace"}
    torch.cuda.synchronize()
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for kept in (False, True):
        torch.cuda.empty_cache()
        mine, out = copy(), {}
        if kept:  # buffers of the stream that is current
            call(copy(), out=out)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(10):
                busy @ busy
        got = call(mine, out=out, stream=side)
        assert got is out
        sizes = [t.numel() * t.element_size() for t in mine + list(got.values())]
        got = {n: got[n] for n in want}
        del mine, out
        taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
        torch.cuda.current_stream().wait_stream(side)
        for n, t in want.items():
            assert torch.equal(got[n], t), (n, kept)
        del taken


def test_a_stream_argument_gives_the_same_bits_in_a_graph(torch_cuda):
    torch = torch_cuda
    side = torch.cuda.Stream()
    for name, (call, tensors) in _calls(torch).items():
        if name == "linear_attention_step":  # (its table changes)
            continue
        want = {n: t.clone() for n, t in call(tensors).items() if n != "workspace"}
        out = {}
        side.wait_stream(torch.cuda.current_stream())
        call(tensors, out=out, stream=side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            side.wait_stream(torch.cuda.current_stream())
            call(tensors, out=out, stream=side)
            torch.cuda.current_stream().wait_stream(side)
        for _ in range(3):
            for t in out.values():
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for n, t in want.items():
                assert torch.equal(out[n], t), (name, n)


@pytest.mark.parametrize("name", NAMES)
def test_a_call_runs_on_its_tensors_device(torch_cuda, name, monkeypatch):
    """With another device current (there is one here: that it is another is pretended until torch is told to change to it)."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    call, tensors = _calls(torch)[name]
    copy = lambda: [t.clone() for t in tensors]
    want = {n: t.clone() for n, t in call(copy()).items() if n != "workspace"}
    real, told = torch.cuda.device, []

    class device(real):
        def __init__(self, d):
            told.append(d)
            super().__init__(d)

    other = lambda: 0 if told else 1
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", other)
    monkeypatch.setattr(memory, "_current_device", other, raising=False)
    got = call(copy())
    monkeypatch.undo()
    assert told == [tensors[0].device]
    for n, t in want.items():
        assert torch.equal(got[n], t), n


def test_a_stream_of_another_device_is_refused(torch_cuda):
    from paper_2006_11751_amd import memory

    class Other:
        device, cuda_stream = torch_cuda.device("cuda", 1), 0

    with pytest.raises(ValueError, match="cuda:1"):
        memory.residual_norm(torch_cuda.zeros(2, 8, device="cuda"), stream=Other())
