"""examples/memory_block.py with the gated delta rule and clipped gradients: it runs, its gradients are those of its definition, and it steps
as it unrolls."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("memory_block", os.path.join(ROOT, "examples", "memory_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_trains_with_clipped_gradients(torch_cuda, monkeypatch):
    torch = torch_cuda
    m = _example()
    real, norms = m.memory.clip_gradients, []

    def clip(grads, max_norm, **kw):
        out = real(grads, max_norm, **kw)
        after = math.sqrt(sum((g.double() ** 2).sum().item() for g in grads))
        norms.append((out["norm"].item(), after))
        return out

    monkeypatch.setattr(m.memory, "clip_gradients", clip)
    losses, block = m.train(4, T=40, N=8, report=None, mixer="delta", max_norm=0.05)
    assert all(math.isfinite(v) for v in losses) and len(norms) == 4
    for before, after in norms:
        # (bf16 gradients are rounded again, each by 2^-8 at most)
        assert abs(after - min(before, 0.05)) <= (2.0 ** -8 + 1e-4) * 0.05
    assert all(torch.isfinite(p).all() for p in block.p.values())


def test_it_steps_as_it_unrolls(torch_cuda):
    m = _example()
    y, state = m.compare_steps(m.MemoryBlock(mixer="delta"))
    # bf16 between the operators: a rounding (2^-8) that falls the other way is passed on by the following ones
    assert y < 2.0 ** -5 and state < 2.0 ** -5, (y, state)


def test_its_gradients_against_autograd(torch_cuda):
    """The whole block in 64 bits by autograd of its definition; bf16 roundings of some twelve operators in a row leave less
    than twelve times 2^-8 of each gradient's norm."""
    torch = torch_cuda
    m = _example()
    H, d = 2, 32
    block = m.MemoryBlock(D=64, H=H, d=d, F=96, seed=3, mixer="delta")
    g = torch.Generator(device="cuda").manual_seed(4)
    x, done, _ = m.trajectories(20, 6, 64, 0.1, g)
    w = block.weights()
    y, _, kept = block.unroll(w, x, done, None)
    dy = torch.randn(y.shape, generator=g, device="cuda").bfloat16()
    grads = block.backward(w, kept, dy)
    leaf = {k: v.double().requires_grad_() for k, v in w.items()}
    rms = lambda a: a / (a.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    silu = lambda a: a * torch.sigmoid(a)
    xd = x.double()
    n = rms(xd) * leaf["norm_in"]
    q, k, v, gate = (n @ leaf["w_in"].T).split(H * d, -1)
    q, k, v = (a.unflatten(-1, (H, d)) for a in (q, k, v))
    q, k = rms(q) * d ** -0.5, rms(k) * d ** -0.5
    a, b = (n @ leaf["w_step"].T).split(H, -1)
    log_decay, beta = 2.0 * block.log_decay.double() * torch.sigmoid(a), torch.sigmoid(b)
    s, o = torch.zeros(6, H, d, d, dtype=torch.float64, device="cuda"), []
    for t in range(20):
        s = log_decay[t].exp()[..., None, None] * (done[t] == 0).double()[:, None, None, None] * s
        s = s + k[t][..., None] * (beta[t][..., None] * (v[t] - (s * k[t][..., None]).sum(-2)))[..., None, :]
        o.append(d ** -0.5 * (q[t][..., None] * s).sum(-2))
    c = rms(torch.stack(o)).flatten(-2) * leaf["norm_o"] * silu(gate)
    y1 = xd + leaf["scale_b"] * rms(c @ leaf["w_out"].T) * leaf["norm_b"]
    n1 = rms(y1) * leaf["norm_f_in"]
    f = (silu(n1 @ leaf["w_gate"].T) * (n1 @ leaf["w_up"].T)) @ leaf["w_down"].T
    yd = y1 + leaf["scale_f"] * rms(f) * leaf["norm_f"]
    assert (y.double() - yd).norm() <= 12 * 2.0 ** -8 * yd.norm()
    names = [name for name in leaf if name != "head"]
    for name, want in zip(names, torch.autograd.grad((yd * dy.double()).sum(), [leaf[name] for name in names])):
        off = ((grads[name].double() - want).norm() / want.norm()).item()
        assert off <= 12 * 2.0 ** -8, (name, off)
