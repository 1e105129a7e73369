"""Linear attention with a decay for each head (csrc/k_linattn.hip) against its definition, step by step in 64 bits.

Tolerances.  With A = the same recurrence on absolute values (an upper bound of the sum of the terms' magnitudes), an
fp32 result is a sum of at most dk + 64 products and T / 32 running states, each rounded to 2^-24: n 2^-24 A with
n = dk + 160 + T / 16.  bf16 arrays: what enters a product from fp32 is two bf16 numbers, which leave 2^-16 of it
out at most (half a unit in the last of 8 bits is 2^-8 of a power of two, and that twice), and the result is rounded to 8
bits: (2^-16 + n 2^-24) A (1 + 2^-8) + 2^-8 |y|.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def oracle(q, k, v, ld, done, s0, scale, do=None, ds=None):
    """Everything in 64 bits, token by token; q [T,N,H,dk], k, v with shared heads.  With do: the gradients."""
    import torch
    T, N, H, dk = q.shape
    Hk, dv = v.shape[2:]
    rep = lambda a: a.double().repeat_interleave(H // Hk, 2)
    q, k, v = q.double(), rep(k), rep(v)
    g = torch.exp(ld.double())[None, :, None, None]
    start = lambda t: (done[t] != 0)[:, None, None, None] if done is not None else torch.zeros(N, 1, 1, 1, dtype=torch.bool, device=q.device)
    s = torch.zeros(N, H, dk, dv, dtype=torch.float64, device=q.device) if s0 is None else s0.double()
    o = torch.zeros(T, N, H, dv, dtype=torch.float64, device=q.device)
    dq = torch.zeros(T, N, H, dk, dtype=torch.float64, device=q.device)
    for t in range(T):
        s = torch.where(start(t), 0.0, g * s) + k[t][..., :, None] * v[t][..., None, :]
        o[t] = scale * (q[t][..., :, None] * s).sum(-2)
        if do is not None:
            dq[t] = scale * (s * do[t].double()[..., None, :]).sum(-1)
    if do is None:
        return dict(o=o, state=s)
    r = torch.zeros_like(s) if ds is None else ds.double()
    gk, gv = torch.zeros_like(q), torch.zeros_like(o)
    for t in reversed(range(T)):
        r = r + scale * q[t][..., :, None] * do[t].double()[..., None, :]
        gk[t], gv[t] = (r * v[t][..., None, :]).sum(-1), (r * k[t][..., :, None]).sum(-2)
        r = torch.where(start(t), 0.0, g * r)
    share = lambda a: a.unflatten(2, (Hk, H // Hk)).sum(3)
    return dict(dq=dq, dk=share(gk), dv=share(gv), dstate0=r)


def check(got, want, size, n, dtype):
    import torch
    for name, y in want.items():
        x = got[name].double()
        assert x.shape == y.shape, name
        bad = torch.isfinite(y) != torch.isfinite(x)
        assert not bad.any(), "%s: %d of other finiteness" % (name, bad.sum())
        A = size[name]
        tol = ((2.0 ** -16 + n * 2.0 ** -24) * (1 + 2.0 ** -8) * A + 2.0 ** -8 * y.abs() if dtype == "bf16" and "state" not in name else n * 2.0 ** -24 * A) + 1e-37
        fine = torch.isfinite(y)
        over = ((x - y).abs()[fine] / tol[fine]).max().item() if fine.any() else 0.0
        assert over <= 1.0, "%s: %.2f of the tolerance" % (name, over)


def make(torch, T, N, H, Hk, dk, dv, dtype, p_done=0.1, seed=0, tau=20.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = dict(q=r(T, N, H, dk).to(dt), k=r(T, N, Hk, dk).to(dt), v=r(T, N, Hk, dv).to(dt),
             log_decay=-(2.0 ** -torch.arange(H, device="cuda").float()) * 4.0 / tau, done=(torch.rand(T, N, generator=g, device="cuda") < p_done).byte(),
             state0=0.3 * r(N, H, dk, dv))
    return x, r(T, N, H, dv).to(dt), 0.3 * r(N, H, dk, dv)


def both(torch, x, do, ds, dtype, scale=None):
    from paper_2006_11751_amd import memory
    T, N, H, dk = x["q"].shape
    sc = dk ** -0.5 if scale is None else scale
    n = dk + 160 + T / 16
    ab = lambda a: None if a is None else a.abs()
    y = {a: x[a] for a in ("done", "state0")}
    args = (x["q"], x["k"], x["v"], x["log_decay"])
    absargs = (ab(x["q"]), ab(x["k"]), ab(x["v"]), x["log_decay"])
    got = memory.linear_attention(*args, scale=scale, **y)
    back = memory.linear_attention_backward(*args, do, dstate=ds, scale=scale, **y)
    torch.cuda.synchronize()
    check(got, oracle(*args, y["done"], y["state0"], sc), oracle(*absargs, y["done"], ab(y["state0"]), abs(sc)), n, dtype)
    check(back, oracle(*args, y["done"], y["state0"], sc, do, ds),
          oracle(*absargs, y["done"], ab(y["state0"]), abs(sc), ab(do), ab(ds)), n * (x["q"].shape[2] // x["k"].shape[2]), dtype)
    return got, back


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 129, 255, 257, 600])
def test_lengths(torch_cuda, T, dtype):
    x, do, ds = make(torch_cuda, T, 3, 2, 2, 64, 64, dtype, seed=T)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv", [(1, 1), (8, 16), (13, 7), (40, 72), (64, 128), (128, 64), (128, 128), (127, 65), (100, 24)])
def test_head_sizes(torch_cuda, dk, dv, dtype):
    x, do, ds = make(torch_cuda, 70, 2, 3, 3, dk, dv, dtype, seed=dk + dv)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (3, 3), (1, 1)])
def test_shared_heads(torch_cuda, H, Hk, dtype):
    x, do, ds = make(torch_cuda, 90, 3, H, Hk, 48, 32, dtype, seed=H)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("marks", ["none", "null", "first", "all", "last", "edges"])
def test_episode_ends(torch_cuda, marks, dtype):
    torch = torch_cuda
    T = 700  # several pieces
    x, do, ds = make(torch, T, 2, 2, 2, 32, 64, dtype, seed=5, tau=300.0)
    d = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    if marks == "first":
        d[0] = 1
    elif marks == "all":
        d[:] = 255
    elif marks == "last":
        d[T - 1, 1] = 1
    elif marks == "edges":
        for t in (32, 63, 64, 255, 256, 512):
            d[t, 0] = 1
        d[320, 1] = 1
    x["done"] = None if marks == "null" else d
    both(torch, x, do, ds, dtype)


@pytest.mark.parametrize("T", [40, 1500])
def test_decays_of_zero_and_one_and_no_state(torch_cuda, T):
    torch = torch_cuda
    x, do, _ = make(torch, T, 2, 3, 3, 64, 64, "fp32", p_done=0.01, seed=9)
    x["log_decay"] = torch.tensor([0.0, float("-inf"), -1e-3], device="cuda")
    x["state0"] = None
    both(torch, x, do, None, "fp32", scale=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strided_and_unaligned_arrays(torch_cuda, dtype):
    torch = torch_cuda
    T, N, H, dk, dv = 75, 3, 4, 64, 64
    x, do, ds = make(torch, T, N, H, H, dk, dv, dtype, seed=3)
    packed = torch.cat([x["q"].flatten(2), x["k"].flatten(2), x["v"].flatten(2)], -1)
    x["q"], x["k"], x["v"] = (a.unflatten(-1, (H, 64)) for a in packed.split(H * 64, -1))
    a, _ = both(torch, x, do, ds, dtype)
    # rows first, heads first in memory; one element off a 16-byte boundary
    y = dict(x, q=x["q"].transpose(0, 1).contiguous().transpose(0, 1), k=x["k"].permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3))
    odd = torch.empty(T * N * H * dv + 1, dtype=do.dtype, device="cuda")[1:].view(T, N, H, dv)
    y["v"] = odd.copy_(x["v"])
    b, _ = both(torch, y, do.transpose(0, 2).contiguous().transpose(0, 2), ds, dtype)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [64, 700])
def test_not_finite_values_stay_where_they_are(torch_cuda, T, dtype):
    """An episode with NaN and infinities in it: the ones before and behind it are as if it were not there, and so are
    its own steps before the first of them (backwards: those behind)."""
    torch = torch_cuda
    x, do, ds = make(torch, T, 2, 2, 2, 64, 64, dtype, seed=11, p_done=0.0)
    d = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    d[20], d[45] = 1, 1
    x["done"] = d
    x["state0"][0, 0, 3, 5] = float("inf")
    x["k"][30, 0, 0, 7], x["v"][33, 0, 1, 2], x["q"][31, 1] = float("nan"), float("inf"), float("nan")
    do[34, 0, 1, 4] = float("-inf")
    from paper_2006_11751_amd import memory
    args = (x["q"], x["k"], x["v"], x["log_decay"])
    got = memory.linear_attention(*args, done=d, state0=x["state0"])
    back = memory.linear_attention_backward(*args, do, done=d, state0=x["state0"], dstate=ds)
    clean = lambda a: torch.nan_to_num(a, nan=0.0, posinf=0.0, neginf=0.0)
    cargs = tuple(clean(a) for a in args[:3]) + (x["log_decay"],)
    sc = 64 ** -0.5
    want = oracle(*cargs, d, clean(x["state0"]), sc)
    wback = oracle(*cargs, d, clean(x["state0"]), sc, clean(do), ds)
    size = oracle(*(a.abs() for a in cargs[:3]), x["log_decay"], d, clean(x["state0"]).abs(), sc)
    sback = oracle(*(a.abs() for a in cargs[:3]), x["log_decay"], d, clean(x["state0"]).abs(), sc, clean(do).abs(), ds.abs())
    n = 64 + 160 + T / 16
    part = lambda r, names, sl: {a: r[a][sl] for a in names}
    for sl in (slice(45, T), slice(20, 30)):
        check(part(got, ["o"], sl), part(want, ["o"], sl), part(size, ["o"], sl), n, dtype)
        check(part(back, ["dq"], sl), part(wback, ["dq"], sl), part(sback, ["dq"], sl), n, dtype)
    check({"state": got["state"]}, {"state": want["state"]}, size, n, dtype)
    for sl in (slice(45, T), slice(35, 45), slice(0, 20)):
        check(part(back, ["dk", "dv"], sl), part(wback, ["dk", "dv"], sl), part(sback, ["dk", "dv"], sl), n, dtype)
    check({"dstate0": back["dstate0"]}, {"dstate0": wback["dstate0"]}, sback, n, dtype)
    assert not torch.isfinite(got["o"][30:45, 0, 0].float()).all(-1).any()  # and there they are
    assert torch.isfinite(got["o"][0:20, 0, 0].float()).sum() < 20 * 64


def test_no_steps_and_no_rows(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = make(torch, 0, 2, 2, 2, 64, 64, "bf16")
    args = (x["q"], x["k"], x["v"], x["log_decay"])
    assert torch.equal(memory.linear_attention(*args, done=x["done"], state0=x["state0"])["state"], x["state0"])
    assert torch.equal(memory.linear_attention_backward(*args, do, done=x["done"], dstate=ds)["dstate0"], ds)
    x, do, ds = make(torch, 5, 0, 2, 2, 64, 64, "bf16")
    assert memory.linear_attention(x["q"], x["k"], x["v"], x["log_decay"])["o"].shape == (5, 0, 2, 64)
    memory.linear_attention_backward(x["q"], x["k"], x["v"], x["log_decay"], do)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", ["q", "k", "v", "state0"])
def test_gradients_against_differences(torch_cuda, name):
    """o and the state are linear in each of the arrays: a difference over a whole unit is the derivative, up to rounding
    (2^-24 of sums of T N H dv numbers of size ~ 10, each with its own sign)."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = make(torch, 150, 2, 4, 2, 32, 48, "fp32", seed=21)
    args = lambda y: (y["q"], y["k"], y["v"], y["log_decay"])
    kw = lambda y: dict(done=y["done"], state0=y["state0"])
    loss = lambda y: sum((a.double() * b.double()).sum() for a, b in zip(
        (memory.linear_attention(*args(y), **kw(y))[n] for n in ("o", "state")), (do, ds)))
    grad = memory.linear_attention_backward(*args(x), do, dstate=ds, **kw(x))["dstate0" if name == "state0" else "d" + name]
    way = torch.randn(x[name].shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    up, down = (loss(dict(x, **{name: x[name] + s * way})) for s in (0.5, -0.5))
    want = (grad.double() * way.double()).sum()
    scale = (grad.double() * way.double()).square().sum().sqrt()
    assert abs(up - down - want) <= 1e-4 * scale, (up - down, want, scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,H,Hk,dk,dv", [(1, 1, 1, 64, 64), (5, 4, 2, 128, 128), (33, 3, 3, 13, 7), (3, 2, 2, 40, 72), (7, 8, 1, 128, 6), (2, 1, 1, 1, 128)])
def test_step(torch_cuda, B, H, Hk, dk, dv, dtype):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    n_env = 2 * B + 3
    x, _, _ = make(torch, 1, B, H, Hk, dk, dv, dtype, p_done=0.3, seed=B)
    table = torch.randn(n_env, H, dk, dv, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    ids = torch.randperm(n_env, device="cuda")[:B].int()
    q, k, v = (x[n][0] for n in "qkv")
    for ids_ in (ids, None):
        t = table.clone()
        rows = torch.arange(B, device="cuda") if ids_ is None else ids.long()
        got = memory.linear_attention_step(q, k, v, x["log_decay"], t, env_ids=ids_, done=x["done"][0])
        torch.cuda.synchronize()
        args = (x["k"], x["v"], x["log_decay"], x["done"])
        want = oracle(x["q"], *args, table[rows], dk ** -0.5)
        size = oracle(x["q"].abs(), x["k"].abs(), x["v"].abs(), *args[2:], table[rows].abs(), dk ** -0.5)
        check(dict(o=got["o"][None], state=t[rows]), want, size, dk + 160, dtype)
        rest = torch.ones(n_env, dtype=torch.bool, device="cuda")
        rest[rows] = False
        assert torch.equal(t[rest], table[rest])


def test_step_with_ids_outside_the_table_and_states_that_are_not_finite(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, _, _ = make(torch, 1, 4, 2, 2, 64, 64, "fp32", p_done=0.0)
    table = torch.randn(3, 2, 64, 64, device="cuda")
    table[2] = float("nan")
    t = table.clone()
    ids = torch.tensor([-1, 3, 1, 2], dtype=torch.int32, device="cuda")
    done = torch.tensor([0, 0, 0, 1], dtype=torch.uint8, device="cuda")
    q, k, v = (x[n][0] for n in "qkv")
    o = memory.linear_attention_step(q, k, v, x["log_decay"], t, env_ids=ids, done=done)["o"]
    torch.cuda.synchronize()
    s0 = torch.zeros(4, 2, 64, 64, device="cuda")
    s0[2] = table[1]
    want = oracle(x["q"], x["k"], x["v"], x["log_decay"], None, s0, 0.125)
    size = oracle(x["q"].abs(), x["k"].abs(), x["v"].abs(), x["log_decay"], None, s0.abs(), 0.125)
    check(dict(o=o[None]), {"o": want["o"]}, size, 64 + 160, "fp32")
    assert torch.equal(t[0], table[0])
    check(dict(state=t[1:]), {"state": want["state"][2:]}, {"state": size["state"][2:]}, 64 + 160, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steps_follow_the_pass_over_a_trajectory(torch_cuda, dtype):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, _, _ = make(torch, 50, 4, 2, 2, 64, 64, dtype, seed=8)
    whole = memory.linear_attention(x["q"], x["k"], x["v"], x["log_decay"], done=x["done"], state0=x["state0"])
    table = x["state0"].clone()
    o = torch.stack([memory.linear_attention_step(x["q"][t], x["k"][t], x["v"][t], x["log_decay"], table, done=x["done"][t])["o"]
                     for t in range(50)])
    torch.cuda.synchronize()
    size = oracle(x["q"].abs(), x["k"].abs(), x["v"].abs(), x["log_decay"], x["done"], x["state0"].abs(), 0.125)
    tol = 2 * ((2.0 ** -16 + 230 * 2.0 ** -24) * 1.01 * size["o"] + 2.0 ** -8 * 1.01 * whole["o"].double().abs()) if dtype == "bf16" else 2 * 230 * 2.0 ** -24 * size["o"]
    assert ((o.double() - whole["o"].double()).abs() <= tol).all()
    assert ((table.double() - whole["state"].double()).abs() <= 2 * 230 * 2.0 ** -24 * size["state"]).all()


def test_a_state_beyond_32_bit_offsets(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    n_env, H = 20000, 8  # 20000 x 8 x 128 x 128 floats: 10.5 GB
    table = torch.zeros(n_env, H, 128, 128, device="cuda")
    x, _, _ = make(torch, 1, 2, H, H, 128, 128, "bf16", p_done=0.0, seed=4)
    ids = torch.tensor([n_env - 1, 17000], dtype=torch.int32, device="cuda")
    table[ids.long()] = x["state0"]
    q, k, v = (x[n][0] for n in "qkv")
    memory.linear_attention_step(q, k, v, x["log_decay"], table, env_ids=ids)
    want = oracle(x["q"], x["k"], x["v"], x["log_decay"], None, x["state0"], 1.0)["state"]
    assert torch.allclose(table[ids.long()].double(), want, rtol=1e-5, atol=1e-6)
    assert table[:17000].abs().max() == 0


def test_same_bits_on_another_stream_and_in_a_graph(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = make(torch, 600, 2, 2, 1, 64, 64, "bf16", seed=2)
    args, kw = (x["q"], x["k"], x["v"], x["log_decay"]), dict(done=x["done"], state0=x["state0"])
    run = lambda a, b: (memory.linear_attention(*args, out=a, **kw), memory.linear_attention_backward(*args, do, dstate=ds, out=b, **kw))
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
            for k, t in r.items():
                t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(a, b)


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import SfError, memory
    x, do, ds = make(torch, 4, 2, 4, 2, 16, 16, "fp32")
    q, k, v, ld = x["q"], x["k"], x["v"], x["log_decay"]
    for bad in (dict(q=q.double()), dict(q=q.cpu()), dict(k=k[:3]), dict(v=v.bfloat16()), dict(log_decay=ld[:3]), dict(log_decay=ld.double()),
                dict(done=x["done"].int()), dict(done=x["done"].T), dict(state0=x["state0"][:1]), dict(k=k[..., :8]),
                dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), dict(out=dict(o=q.clone()[:2]))):
        with pytest.raises(ValueError):
            memory.linear_attention(**dict(dict(q=q, k=k, v=v, log_decay=ld), **bad))
    with pytest.raises(SfError) as e:
        memory.linear_attention(q[:, :, :3], k, v, ld[:3])
    assert e.value.code == -2 and "Hk = 2" in str(e.value)
    with pytest.raises(SfError):
        memory.linear_attention(q, k, v, ld, scale=float("nan"))
    wide = torch.zeros(1, 1, 1, 129, device="cuda")
    with pytest.raises(SfError):
        memory.linear_attention(wide, wide, wide, ld[:1].contiguous())
    with pytest.raises(SfError):
        memory.linear_attention_step(q[0], k[0], v[0], ld, torch.zeros(1, 4, 16, 16, device="cuda"))
    with pytest.raises(SfError) as e:
        memory.linear_attention_backward(q, k, v, ld, do, dstate=ds, out=dict(dstate0=ds))
    assert e.value.code == -4


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N,H,Hk,dk,dv", [(1, 1, 1, 1, 8, 8), (7, 5, 4, 1, 24, 64), (16, 50, 6, 2, 64, 40), (17, 3, 4, 2, 48, 32),
                                            (31, 130, 2, 2, 56, 8), (32, 7, 3, 3, 64, 64), (32, 2, 8, 4, 16, 64)])
def test_short_trajectories(torch_cuda, T, N, H, Hk, dk, dv, dtype):
    """At most 32 steps: the backward pass has a kernel of its own for them."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = make(torch, T, N, H, Hk, dk, dv, dtype, seed=T + dk)
    _, a = both(torch, x, do, ds, dtype, scale=-0.7)
    # the same bits in another order in memory
    y = [x[n].transpose(0, 1).contiguous().transpose(0, 1) for n in "qkv"]
    b = memory.linear_attention_backward(*y, x["log_decay"], do.transpose(0, 2).contiguous().transpose(0, 2), dstate=ds, done=x["done"],
                                         state0=x["state0"], scale=-0.7)
    for n in ("dq", "dk", "dv", "dstate0"):
        assert torch.equal(a[n], b[n]), n
    # no states, no episode ends
    args = (x["q"], x["k"], x["v"], x["log_decay"])
    c = memory.linear_attention_backward(*args, do)
    absargs = tuple(t.abs() for t in args[:3]) + (x["log_decay"],)
    check(c, oracle(*args, None, None, dk ** -0.5, do), oracle(*absargs, None, None, dk ** -0.5, do.abs()), (dk + 160 + T / 16) * (H // Hk), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_short_trajectories_with_values_that_are_not_finite(torch_cuda, dtype):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    T, inf, nan = 24, float("inf"), float("nan")
    x, do, ds = make(torch, T, 2, 2, 2, 64, 64, dtype, seed=5, p_done=0.0)
    x["done"][8], x["done"][17] = 1, 1
    x["k"][11, 0, 0, 7], x["v"][12, 0, 1, 2], x["q"][11, 1], do[12, 0, 1, 4] = nan, inf, nan, -inf
    x["state0"][0, 0, 3, 5], ds[1, 0, 2, 2] = inf, -inf
    args = (x["q"], x["k"], x["v"], x["log_decay"])
    back = memory.linear_attention_backward(*args, do, dstate=ds, done=x["done"], state0=x["state0"])
    clean = lambda a: torch.nan_to_num(a, nan=0.0, posinf=0.0, neginf=0.0)
    cargs = tuple(clean(a) for a in args[:3]) + (x["log_decay"],)
    want = oracle(*cargs, x["done"], clean(x["state0"]), 0.125, clean(do), clean(ds))
    size = oracle(*(a.abs() for a in cargs[:3]), x["log_decay"], x["done"], clean(x["state0"]).abs(), 0.125, clean(do).abs(), clean(ds).abs())
    within = torch.arange(T, device="cuda")[:, None, None]
    row, head = torch.arange(2, device="cuda")[:, None], torch.arange(2, device="cuda")
    first = (within < 8) & ~((row == 0) & (head == 0))           # state0 is not finite there
    last = (within >= 17) & ~((row == 1) & (head == 0))          # dstate is not finite there
    inside = (within >= 8) & (within < 17)
    for n, fine in (("dq", first | (inside & (within < 11)) | (within >= 17)), ("dk", (within < 8) | (inside & (within > 12)) | last),
                    ("dv", (within < 8) | (inside & (within > 12)) | last)):
        pick = lambda a: {n: torch.where(fine[..., None], a[n], torch.zeros((), dtype=a[n].dtype, device="cuda"))}
        check(pick(back), pick(want), pick(size), 64 + 160 + T / 16, dtype)
    check(back, {"dstate0": want["dstate0"]}, size, 64 + 160 + T / 16, dtype)
    assert not torch.isfinite(back["dq"][3, 0, 0]).all() and not torch.isfinite(back["dk"][20, 1, 0]).all()
    assert not torch.isfinite(back["dq"][14, 0]).all() and not torch.isfinite(back["dk"][9, 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N,H,dk,dv", [(700, 2, 2, 128, 128), (1300, 5, 4, 64, 64), (1027, 3, 5, 24, 100), (513, 1, 1, 8, 8)])
def test_long_trajectories_of_few_rows(torch_cuda, T, N, H, dk, dv, dtype):
    """Lengths that are cut into pieces, whose states are made first."""
    x, do, ds = make(torch_cuda, T, N, H, H, dk, dv, dtype, seed=T, p_done=0.003)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N", [(1500, 1), (40, 3), (24, 3)])
def test_a_state_that_is_not_finite_stays_so_however_long_the_trajectory(torch_cuda, T, N, dtype):
    """g^T is zero in 32 bits, NaN and infinity times it are not; in pieces of T (1500 steps of few rows) as without."""
    torch = torch_cuda
    x, do, ds = make(torch, T, N, 2, 2, 64, 64, dtype, p_done=0.0, seed=12)
    x["log_decay"] = torch.tensor([-1.0, -0.01], device="cuda")
    x["state0"][0, 0, 3, 5], x["state0"][N - 1, 1, 7, 2] = float("nan"), float("-inf")
    ds[0, 0, 9, 11], ds[N - 1, 1, 1, 4] = float("inf"), float("nan")
    both(torch, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [24, 70, 1500])
def test_a_decay_that_is_nan_is_in_its_heads_results(torch_cuda, T, dtype):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = make(torch, T, 2, 3, 3, 64, 64, dtype, p_done=0.0, seed=13)
    bad = x["log_decay"].clone()
    bad[1] = float("nan")
    pairs = []
    for ld in (x["log_decay"], bad):
        args, kw = (x["q"], x["k"], x["v"], ld), dict(done=x["done"], state0=x["state0"])
        r = dict(memory.linear_attention(*args, **kw), **{"back_" + n: t for n, t in memory.linear_attention_backward(*args, do, dstate=ds, **kw).items()})
        table = x["state0"].clone()
        r["step"] = memory.linear_attention_step(x["q"][0], x["k"][0], x["v"][0], ld, table)["o"][None]
        r["table"] = table
        pairs.append(r)
    for n in ("o", "state", "back_dq", "back_dk", "back_dv", "back_dstate0", "step", "table"):
        at = 2 if pairs[0][n].dim() == 4 and "state" not in n and n != "table" else 1  # the head's axis
        head = lambda a, h: a.select(at, h)
        for h in (0, 2):
            assert torch.equal(head(pairs[0][n], h), head(pairs[1][n], h)), n
        got = head(pairs[1][n], 1)
        if n in ("back_dk", "back_dv"):
            got = got[:-1]  # (no decay enters the last step's)
        assert torch.isnan(got).all(), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [24, 40])
@pytest.mark.parametrize("stride", [1 << 23, (1 << 23) + 8])
def test_steps_far_apart(torch_cuda, T, stride, dtype):
    """Steps up to 2^23 elements apart are read through 32-bit offsets from the chunk, others through 64-bit addresses."""
    torch = torch_cuda
    x, do, ds = make(torch, T, 2, 2, 2, 64, 64, dtype, seed=14)
    a, b = both(torch, x, do, ds, dtype)
    wide = torch.full((T, stride), float("nan"), dtype=do.dtype, device="cuda")
    parts = wide[:, :4 * 256].unflatten(1, (4, 2, 2, 64)).unbind(1)
    for n, part, t in zip(("q", "k", "v", "do"), parts, (x["q"], x["k"], x["v"], do)):
        part.copy_(t)
    c, d = both(torch, dict(x, q=parts[0], k=parts[1], v=parts[2]), parts[3], ds, dtype)
    for n in ("o", "state"):
        assert torch.equal(a[n], c[n]), n
