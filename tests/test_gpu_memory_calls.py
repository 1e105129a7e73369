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
