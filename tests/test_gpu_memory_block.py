"""examples/memory_block.py: the operators together, trained, and stepped as they were unrolled."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("memory_block", os.path.join(ROOT, "examples", "memory_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_block_learns_and_steps_as_it_unrolls(torch_cuda):
    m = _example()
    losses, block = m.train(140, report=None)
    # chance is log 8 = 2.08; with a memory the cue is known at every step
    assert losses[0] > 1.5 and sum(losses[-5:]) / 5 < 0.5 * losses[0], losses[::10]
    # bf16 between the operators: a rounding (2^-8) that falls the other way is passed on by the following ones
    y, state = m.compare_steps(block)
    assert y < 2.0 ** -5 and state < 2.0 ** -5, (y, state)


def test_the_blocks_gradients_against_autograd(torch_cuda):
    """The whole block in 64 bits by autograd of its definition; bf16 roundings of some ten operators in a row leave less
    than ten times 2^-8 of each gradient's norm."""
    torch = torch_cuda
    m = _example()
    block = m.MemoryBlock(D=64, H=2, d=32, F=96, seed=3)
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
    q, k, v, gate = ((rms(xd) * leaf["norm_in"]) @ leaf["w_in"].T).split(64, -1)
    q, k, v = (a.unflatten(-1, (2, 32)) for a in (q, k, v))
    s, o = 0.0, []
    for t in range(20):
        keep = block.log_decay.double().exp()[None, :, None, None] * (done[t] == 0).double()[:, None, None, None]
        s = keep * s + k[t][..., None] * v[t][..., None, :]
        o.append(32 ** -0.5 * (q[t][..., None] * s).sum(-2))
    a = rms(torch.stack(o)).flatten(-2) * leaf["norm_o"] * silu(gate)
    y1 = xd + leaf["scale_b"] * rms(a @ leaf["w_out"].T) * leaf["norm_b"]
    n1 = rms(y1) * leaf["norm_f_in"]
    f = (silu(n1 @ leaf["w_gate"].T) * (n1 @ leaf["w_up"].T)) @ leaf["w_down"].T
    yd = y1 + leaf["scale_f"] * rms(f) * leaf["norm_f"]
    assert (y.double() - yd).norm() <= 10 * 2.0 ** -8 * yd.norm()
    names = [n for n in leaf if n != "head"]
    for n, want in zip(names, torch.autograd.grad((yd * dy.double()).sum(), [leaf[n] for n in names])):
        off = ((grads[n].double() - want).norm() / want.norm()).item()
        assert off <= 10 * 2.0 ** -8, (n, off)
