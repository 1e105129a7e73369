"""The gated delta rule (csrc/k_delta.hip) against its definition, step by step in 64 bits; sizes and tolerances are those of
tests/delta_reference.py."""
import pytest

from tests import delta_reference as ref

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "log_decay", "beta")


def call(x, do=None, dstate=None, **kw):
    from paper_2006_11751_amd import memory
    args, more = [x[n] for n in NAMES], dict(done=x["done"], state0=x["state0"], **kw)
    return memory.delta_rule(*args, **more) if do is None else memory.delta_rule_backward(*args, do, dstate=dstate, **more)


def both(torch, x, do, ds, dtype, scale=None, length=17.0):
    """length: steps that the memory is long (at most T)."""
    got, back = call(x, scale=scale), call(x, do, ds, scale=scale)
    torch.cuda.synchronize()
    sizes = x["q"].shape[3], x["v"].shape[3], length, dtype == "bf16", x["q"].shape[0]
    ref.check(got, *ref.oracle(x, scale), *sizes)
    ref.check(back, *ref.oracle(x, scale, do, ds), *sizes)
    return got, back


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129, 257, 600])
def test_lengths(torch_cuda, T, dtype):
    x, do, ds = ref.make(T, 3, 2, 2, 64, 64, dtype, seed=T)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [20, 70])
@pytest.mark.parametrize("dk,dv", [(1, 1), (8, 16), (13, 7), (40, 72), (64, 128), (128, 64), (128, 128), (127, 65), (100, 24), (16, 33)])
def test_head_sizes(torch_cuda, dk, dv, T, dtype):
    x, do, ds = ref.make(T, 2, 3, 3, dk, dv, dtype, seed=dk + dv)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (40, 72), (100, 24), (13, 7), (127, 65), (72, 128), (16, 96)])
def test_pieces(torch_cuda, dk, dv, dtype):
    """Few heads and a long axis: T is cut; the last chunk is not whole."""
    x, do, ds = ref.make(1100, 2, 3, 1, dk, dv, dtype, seed=dk, p_done=0.01)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 128), (40, 72), (16, 96), (100, 120)])
def test_many_heads_with_wide_values(torch_cuda, dk, dv, dtype):
    """(128 columns of v for each workgroup.)"""
    x, do, ds = ref.make(70, 64, 8, 8, dk, dv, dtype, seed=dv)
    both(torch_cuda, x, do, ds, dtype)


def test_many_pieces_with_wide_values(torch_cuda):
    torch = torch_cuda
    x, _, _ = ref.make(16390, 1, 8, 4, 24, 72, "bf16", seed=7, p_done=0.0005, memory=300.0)
    got = call(x)
    want, size = ref.oracle(x)
    ref.check(got, want, size, 24, 72, 301.0, True, 16390)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [30, 90])
@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (3, 3), (1, 1), (24, 8)])
def test_shared_heads(torch_cuda, H, Hk, T, dtype):
    x, do, ds = ref.make(T, 3, H, Hk, 48, 32, dtype, seed=H)
    both(torch_cuda, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("marks", ["none", "null", "first", "all", "last", "edges"])
@pytest.mark.parametrize("T", [32, 333, 900])
def test_episode_ends(torch_cuda, T, marks, dtype):
    torch = torch_cuda
    x, do, ds = ref.make(T, 2, 2, 2, 32, 64, dtype, seed=5, memory=100.0)
    d = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    if marks == "first":
        d[0] = 1
    elif marks == "all":
        d[:] = 255
    elif marks == "last":
        d[T - 1, 1] = 1
    elif marks == "edges":
        for t in (16, 31, 32, 63, 64, 255, 256, 332):
            if t < T:
                d[t, 0] = 1
        d[T // 2, 1] = 1
    x["done"] = None if marks == "null" else d
    both(torch, x, do, ds, dtype, length=101.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("behind", [0, 30, 62])
@pytest.mark.parametrize("T", [1, 2, 3, 5])
def test_every_order_of_episode_begins(torch_cuda, T, behind, dtype):
    """A row for each; few steps and columns, so that the tolerance is near the roundings.  With `behind` steps before them the T steps cross
    the border of a chunk: the steps before are of another episode, and nothing of them is looked at."""
    torch = torch_cuda
    N = 2 ** T
    x, do, ds = ref.make(T, N, 2, 2, 8, 8, dtype, seed=40 + T)
    x["done"] = (torch.arange(N, device="cuda")[None] >> torch.arange(T, device="cuda")[:, None] & 1).byte()
    if not behind:
        _, back = both(torch, x, do, ds, dtype)
    else:
        y, ydo, _ = ref.make(behind, N, 2, 2, 8, 8, dtype, seed=50)
        x["done"][0], x["state0"] = 1, None
        want, wback = ref.oracle(x), ref.oracle(x, None, do, ds)
        z = {n: torch.cat([y[n], x[n]]) for n in x if n != "state0"}
        z["state0"] = y["state0"]
        got, back = call(z), call(z, torch.cat([ydo, do]), ds)
        sizes = 8, 8, 17.0, dtype == "bf16", T
        ref.check(dict(o=got["o"][behind:], state=got["state"]), *want, *sizes)
        back = {n: a[behind:] for n, a in back.items() if n not in ("dstate0", "workspace")}
        ref.check(back, {n: a for n, a in wback[0].items() if n != "dstate0"}, wback[1], *sizes)
    # a decay that was made with has a gradient, another one none
    if T > 1 or not behind:
        assert torch.equal(back["dlog_decay"] == 0, (x["done"] != 0)[..., None].expand(T, N, 2))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [30, 300, 900])
def test_decays_of_zero_and_one_and_no_state(torch_cuda, T, dtype):
    torch = torch_cuda
    x, do, _ = ref.make(T, 2, 4, 2, 64, 64, dtype, p_done=0.01, seed=9)
    x["log_decay"][..., 0] = 0.0
    x["log_decay"][..., 1] = float("-inf")
    x["log_decay"][::3, :, 2] = -200.0
    x["log_decay"][1::5, :, 3] = -80.0  # (steps behind it do not lose their own small decays to it)
    x["state0"] = None
    both(torch, x, do, None, dtype, scale=0.5, length=float(T))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("strength", [0.0, 1.0, 1.9])
@pytest.mark.parametrize("T", [32, 200])
def test_the_same_key_again_and_again(torch_cuda, T, strength, dtype):
    """All entries of the chunk's system are then as large as they can be (with a strength of 1.9 corrections overshoot)."""
    torch = torch_cuda
    x, do, ds = ref.make(T, 2, 2, 2, 64, 32, "fp32", seed=13, p_done=0.0)
    x["k"][:] = x["k"][:1]
    x["k"][1::7] *= -1.0
    x["beta"][:] = strength
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x["q"], x["v"], do = x["q"].to(dt), x["v"].to(dt), do.to(dt)
    # (of a length at most one after rounding to 8 bits)
    x["k"] = (x["k"] * (1.0 - 2.0 ** -7)).to(dt)
    both(torch, x, do, ds, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [32, 75])
def test_strided_and_unaligned_arrays(torch_cuda, T, dtype):
    torch = torch_cuda
    N, H, dk, dv = 3, 4, 64, 64
    x, do, ds = ref.make(T, N, H, H, dk, dv, dtype, seed=3)
    packed = torch.cat([x["q"].flatten(2), x["k"].flatten(2), x["v"].flatten(2)], -1)
    x["q"], x["k"], x["v"] = (a.unflatten(-1, (H, 64)) for a in packed.split(H * 64, -1))
    a = both(torch, x, do, ds, dtype)
    # rows first, heads first in memory; one element off a 16-byte boundary
    y = dict(x, q=x["q"].transpose(0, 1).contiguous().transpose(0, 1), k=x["k"].permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3))
    odd = torch.empty(T * N * H * dv + 1, dtype=do.dtype, device="cuda")[1:].view(T, N, H, dv)
    y["v"] = odd.copy_(x["v"])
    b = both(torch, y, do.transpose(0, 2).contiguous().transpose(0, 2), ds, dtype)
    for one, other in zip(a, b):
        for n in one:
            assert n == "workspace" or torch.equal(one[n], other[n]), n


def test_results_at_odd_addresses_and_nothing_behind_them(torch_cuda):
    torch = torch_cuda
    for dtype, dk, dv, T in (("bf16", 36, 20, 41), ("fp32", 64, 64, 32), ("bf16", 64, 64, 32), ("bf16", 128, 128, 33)):
        x, do, ds = ref.make(T, 2, 2, 1, dk, dv, dtype, seed=3)
        for extra in ((), (do, ds)):
            want = call(x, *extra)
            out, guard = {}, []
            for n, t in want.items():
                if n == "workspace":
                    continue
                whole = torch.full((t.numel() + 33,), 7.0, dtype=t.dtype, device="cuda")
                out[n] = whole[1:1 + t.numel()].view(t.shape)
                guard.append(whole)
            call(x, *extra, out=out)
            for n, t in want.items():
                assert n == "workspace" or torch.equal(out[n], t), n
            for g in guard:
                assert g[0] == 7.0 and (g[-32:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,dk,dv", [(32, 64, 64), (32, 128, 128), (32, 40, 72), (100, 64, 64), (100, 40, 128), (700, 64, 64), (700, 128, 72)])
def test_not_finite_values_stay_where_they_are(torch_cuda, T, dk, dv, dtype):
    """An episode with NaN and infinities in it: the ones before and behind it are as if it were not there, and so are the
    results and query gradients of its own steps before the first of them."""
    torch = torch_cuda
    x, do, ds = ref.make(T, 2, 2, 2, dk, dv, dtype, seed=11, p_done=0.0)
    d = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    first, at, behind = (8, 14, 22) if T == 32 else (20, 30, 45)
    d[first], d[behind] = 1, 1
    x["done"] = d
    clean, cdo = dict(x), do
    bad = {n: (a.clone() if a is not None else None) for n, a in x.items()}
    bad["state0"][0, 0, 3, 5] = float("inf")
    bad["k"][at, 0, 0, 7], bad["v"][at + 3, 0, 1, 2], bad["q"][at + 1, 1] = float("nan"), float("inf"), float("nan")
    bad["beta"][at + 2, 0, 0], bad["log_decay"][at + 4, 0, 0] = float("nan"), float("nan")
    bdo = do.clone()
    bdo[at + 4, 0, 1, 4] = float("-inf")
    got, back = call(bad), call(bad, bdo, ds)
    want, size = ref.oracle(clean)
    wback, sback = ref.oracle(clean, None, cdo, ds)
    sizes = dk, dv, 17.0, dtype == "bf16", T
    for part in (slice(behind, T), slice(first, at)):
        ref.check({"o": got["o"]}, {"o": want["o"]}, size, *sizes, part=part)
        ref.check({"dq": back["dq"]}, {"dq": wback["dq"]}, sback, *sizes, part=part)
    ref.check({"state": got["state"]}, {"state": want["state"]}, size, *sizes)
    for n in ("dk", "dv", "dlog_decay", "dbeta"):
        ref.check({n: back[n]}, {n: wback[n]}, sback, *sizes, part=slice(behind, T))
    # the first episode's gradients do not see the infinity of state0 where they do not read it
    ref.check({"dv": back["dv"]}, {"dv": wback["dv"]}, sback, *sizes, part=slice(0, first))
    ref.check({"dstate0": back["dstate0"]}, {"dstate0": wback["dstate0"]}, sback, *sizes)
    assert not torch.isfinite(got["o"][at:behind, 0, 0].float()).all(-1).any()  # and there they are
    assert not torch.isfinite(back["dk"][at:at + 3, 0, 0].float()).all()
    assert torch.isfinite(got["o"][:first, 1].float()).all() and torch.isfinite(back["dk"][:first, 1].float()).all()


def test_no_steps_and_no_rows(torch_cuda):
    torch = torch_cuda
    x, do, ds = ref.make(0, 2, 2, 2, 64, 64, "bf16")
    assert torch.equal(call(x)["state"], x["state0"])
    assert torch.equal(call(x, do, ds)["dstate0"], ds)
    assert not call(dict(x, state0=None))["state"].any() and not call(dict(x, state0=None), do)["dstate0"].any()
    x, do, ds = ref.make(5, 0, 2, 2, 64, 64, "bf16")
    assert call(x)["o"].shape == (5, 0, 2, 64) and call(x, do, ds)["dlog_decay"].shape == (5, 0, 2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_state_in_place_and_pieces_of_a_trajectory(torch_cuda, dtype):
    """The state of one call is the next one's; 70 steps in pieces are the same function."""
    torch = torch_cuda
    x, _, _ = ref.make(70, 3, 4, 2, 64, 40, dtype, seed=21)
    want, size = ref.oracle(x)
    out, o = dict(state=x["state0"].clone()), []
    for t0, t1 in ((0, 1), (1, 33), (33, 66), (66, 70)):
        part = {n: (a[t0:t1] if n != "state0" else out["state"]) for n, a in x.items()}
        out.pop("o", None)
        call(part, out=out)
        o.append(out["o"])
    ref.check(dict(o=torch.cat(o), state=out["state"]), want, size, 64, 40, 17.0, dtype == "bf16", 70)


# ---- single steps ---------------------------------------------------------------------------


def step(x, t, table, ids, **kw):
    from paper_2006_11751_amd import memory
    return memory.delta_rule_step(*(x[n][t] for n in NAMES), table, env_ids=ids, done=None if x["done"] is None else x["done"][t], **kw)["o"]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hk,dk,dv", [(2, 2, 64, 64), (6, 2, 40, 72), (1, 1, 1, 1), (3, 1, 128, 128), (2, 1, 13, 7), (4, 4, 127, 65)])
def test_steps_on_a_table(torch_cuda, H, Hk, dk, dv, dtype):
    torch = torch_cuda
    T, N, n_env = 40, 5, 12
    x, _, _ = ref.make(T, N, H, Hk, dk, dv, dtype, seed=dk)
    x["log_decay"][3::11] = float("-inf")
    want, size = ref.oracle(x)
    ids = torch.randperm(n_env, device="cuda")[:N].int()
    table = torch.randn(n_env, H, dk, dv, device="cuda")
    table[ids.long()] = x["state0"]
    before = table.clone()
    got = dict(o=torch.stack([step(x, t, table, ids) for t in range(T)]), state=table[ids.long()])
    ref.check(got, want, size, dk, dv, 17.0, dtype == "bf16", T)
    others = torch.ones(n_env, dtype=torch.bool, device="cuda")
    others[ids.long()] = False
    assert torch.equal(table[others], before[others])


def test_steps_without_ids_and_with_unknown_ones(torch_cuda):
    torch = torch_cuda
    x, _, _ = ref.make(1, 4, 2, 2, 32, 32, "fp32", seed=2, p_done=0.0)
    table = x["state0"].clone()
    o = step(x, 0, table, None)
    want, size = ref.oracle(x)
    ref.check(dict(o=o[None], state=table), want, size, 32, 32, 17.0, False, 1)
    ids = torch.tensor([2, -1, 4, 0], dtype=torch.int32, device="cuda")  # two are not in the table: from a zero state, dropped
    table = x["state0"].clone()
    before = table.clone()
    o = step(x, 0, table, ids)
    y = dict(x, state0=torch.stack([before[2], 0 * before[0], 0 * before[0], before[0]]))
    want, size = ref.oracle(y)
    ref.check(dict(o=o[None]), dict(o=want["o"]), size, 32, 32, 17.0, False, 1)
    assert torch.equal(table[1], before[1]) and torch.equal(table[3], before[3])
    ref.check(dict(state=table[[2, 0]]), dict(state=want["state"][[0, 3]]), dict(state=size["state"][[0, 3]]), 32, 32, 17.0, False, 1)


def test_a_step_does_not_read_the_state_of_an_episode_that_ended(torch_cuda):
    torch = torch_cuda
    x, _, _ = ref.make(1, 3, 2, 2, 32, 32, "bf16", seed=4, p_done=0.0)
    x["done"][0, 0] = 1
    x["log_decay"][0, 1] = float("-inf")
    table = torch.full((3, 2, 32, 32), float("nan"), device="cuda")
    o = step(x, 0, table, None)
    assert torch.isfinite(o[:2].float()).all() and torch.isfinite(table[:2]).all() and o[2].isnan().all() and table[2].isnan().all()


def test_states_behind_32_bits_of_offset(torch_cuda):
    """A table of 5 GB (1.25 2^30 numbers): rows at its end."""
    torch = torch_cuda
    n_env = (5 << 28) // (8 * 128 * 128)
    x, _, _ = ref.make(1, 2, 8, 8, 128, 128, "bf16", seed=6, p_done=0.0)
    table = torch.zeros(n_env, 8, 128, 128, device="cuda")
    ids = torch.tensor([n_env - 1, n_env - 2], dtype=torch.int32, device="cuda")
    table[ids.long()] = x["state0"]
    o = step(x, 0, table, ids)
    want, size = ref.oracle(x)
    ref.check(dict(o=o[None], state=table[ids.long()]), want, size, 128, 128, 17.0, True, 1)
    assert not table[:n_env - 2].any()


# ---- the binding ----------------------------------------------------------------------------


@pytest.mark.parametrize("T,d,dtype", [(100, 64, "bf16"), (20, 128, "bf16"), (40, 128, "fp32"), (700, 128, "bf16")])
def test_the_same_bits_each_time_in_a_graph_and_on_a_stream(torch_cuda, T, d, dtype):
    torch = torch_cuda
    x, do, ds = ref.make(T, 3, 4, 2, d, d, dtype, seed=1)
    side = torch.cuda.Stream()
    for extra in ((), (do, ds)):
        want = {n: t.clone() for n, t in call(x, *extra).items() if n != "workspace"}
        out, graph = {}, torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        call(x, *extra, out=out, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], t) for n, t in want.items())
        with torch.cuda.graph(graph):
            call(x, *extra, out=out)
        for i in range(4):
            for t in out.values():
                t.zero_()
            call(x, *extra)  # (eager work of the program between replays)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for n, t in want.items():
                assert torch.equal(out[n], t), (n, i)


def test_inputs_that_change_under_a_graph(torch_cuda):
    torch = torch_cuda
    x, do, ds = ref.make(64, 2, 2, 1, 32, 48, "bf16", seed=1)
    out, graph = {}, torch.cuda.CUDAGraph()
    call(x, do, ds, out=out)
    with torch.cuda.graph(graph):
        call(x, do, ds, out=out)
    for seed in (2, 3, 4):
        y, ydo, yds = ref.make(64, 2, 2, 1, 32, 48, "bf16", seed=seed)
        for n in x:
            x[n].copy_(y[n])
        do.copy_(ydo)
        ds.copy_(yds)
        graph.replay()
        want = call(y, ydo, yds)
        torch.cuda.synchronize()
        for n, t in want.items():
            assert n == "workspace" or torch.equal(out[n], t), n


def test_tensors_may_be_dropped_right_after_a_call_on_another_stream(torch_cuda):
    torch = torch_cuda
    x, do, ds = ref.make(100, 3, 4, 2, 64, 64, "bf16", seed=1)
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for extra in ((), (do, ds)):
        want = {n: t.clone() for n, t in call(x, *extra).items() if n != "workspace"}
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        mine, more = {n: t.clone() for n, t in x.items()}, [t.clone() for t in extra]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(10):
                busy @ busy
        got = call(mine, *more, stream=side)
        sizes = [t.numel() * t.element_size() for t in (*mine.values(), *more, *got.values())]
        got = {n: got[n] for n in want}
        del mine, more
        taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
        torch.cuda.current_stream().wait_stream(side)
        for n, t in want.items():
            assert torch.equal(got[n], t), n
        del taken


def test_many_rows_of_shared_heads(torch_cuda):
    """Sums of shared heads' gradients over more rows than the workgroups of a launch have at a time: those of heads of their own, added."""
    torch = torch_cuda
    x, do, ds = ref.make(1100, 130, 2, 1, 128, 16, "fp32", seed=1)
    own = dict(x, q=x["q"].expand(-1, -1, 2, -1).contiguous(), k=x["k"].expand(-1, -1, 2, -1).contiguous())
    got, want = call(x, do, ds), call(own, do, ds)
    assert all(torch.equal(got[n], want[n][:, :, :1] + want[n][:, :, 1:]) for n in ("dq", "dk"))
    assert all(torch.equal(got[n], want[n]) for n in ("dv", "dlog_decay", "dbeta", "dstate0"))


def test_calls_at_the_same_time_on_two_streams(torch_cuda):
    """Each with results and a workspace of its own."""
    torch = torch_cuda
    made = [ref.make(700, 2, 4, 2, 64, 128, "bf16", seed=s) for s in (1, 2)]
    want = [(call(*m), call(m[0])) for m in made]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in made], [({}, {}) for _ in made]
    for _ in range(3):
        for m, st, (back, forth) in zip(made, streams, outs):
            call(*m, out=back, stream=st)
            call(m[0], out=forth, stream=st)
    torch.cuda.synchronize()
    for pair, got in zip(want, outs):
        for w, g in zip(pair, got):
            assert all(torch.equal(w[n], g[n]) for n in w if n != "workspace")


def test_a_call_runs_on_its_tensors_device(torch_cuda, monkeypatch):
    """With another device current (there is one here: that it is another is pretended until torch is told to change to it)."""
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = ref.make(40, 3, 4, 2, 32, 32, "bf16", seed=1)
    calls = (lambda: call(x)["state"], lambda: call(x, do, ds)["dk"], lambda: step(x, 0, x["state0"].clone(), None))
    want = [c() for c in calls]
    real, told = torch.cuda.device, []

    class device(real):
        def __init__(self, d):
            told.append(d)
            super().__init__(d)

    other = lambda: 0 if told else 1
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", other)
    monkeypatch.setattr(memory, "_current_device", other, raising=False)
    got = []
    for c in calls:
        del told[:]
        got.append(c())
        assert told == [do.device]
    monkeypatch.undo()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_number_that_changes_in_place_is_read_at_every_call(torch_cuda):
    torch = torch_cuda
    x, do, ds = ref.make(40, 2, 2, 2, 16, 16, "fp32", seed=1)
    scale = torch.tensor(0.5)
    calls = (lambda: call(x, scale=scale)["o"], lambda: call(x, do, scale=scale)["dq"], lambda: step(x, 0, x["state0"].clone(), None, scale=scale))
    before = [c() for c in calls]
    scale.fill_(1.0)
    assert all(torch.equal(c(), 2 * was) for c, was in zip(calls, before))


def test_what_the_binding_refuses(torch_cuda):
    torch = torch_cuda
    from paper_2006_11751_amd import memory
    x, do, ds = ref.make(3, 2, 4, 2, 8, 8, "fp32")
    good = [x[n] for n in NAMES]
    for i, t, text in ((1, x["k"][:2], "k: "), (1, x["k"].bfloat16(), "k: "), (2, x["v"][:, :1], "v: "), (3, x["log_decay"][..., :2], "log_decay: "),
                       (3, x["log_decay"].double(), "log_decay: "), (4, x["beta"].transpose(0, 1), "beta: "), (4, x["beta"].cpu(), "beta: "),
                       (0, x["q"].half(), "k: "), (2, x["v"][..., ::2], "v: ")):
        args = list(good)
        args[i] = t
        with pytest.raises(ValueError, match=text):
            memory.delta_rule(*args)
    for kw, text in ((dict(done=x["done"].bool()), "done"), (dict(state0=x["state0"].bfloat16()), "state0"), (dict(state0=x["state0"][..., :4]), "state0"),
                     (dict(out=dict(o=torch.zeros(1, device="cuda"))), "out\\['o'\\]")):
        with pytest.raises(ValueError, match=text):
            memory.delta_rule(*good, **kw)
    with pytest.raises(ValueError, match="do"):
        memory.delta_rule_backward(*good, do[:, :, :1])
    with pytest.raises(ValueError, match="dstate"):
        memory.delta_rule_backward(*good, do, dstate=ds[:1])
    with pytest.raises(ValueError, match="env_ids"):
        memory.delta_rule_step(*(a[0] for a in good), x["state0"], env_ids=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(memory.SfError, match="H = 4"):
        memory.delta_rule(*(torch.zeros(3, 2, 3, 8, device="cuda") for _ in range(2)), x["v"], x["log_decay"], x["beta"])


@pytest.mark.parametrize("T", [2, 34])
def test_many_rows_of_one_head(torch_cuda, T):
    """Steps of the decays 8 MB apart, near the most rows of a call; the first and last rows."""
    torch = torch_cuda
    N, rows = (1 << 21) - 1, [0, 1, (1 << 20) + 3, (1 << 21) - 2]
    x, do, ds = ref.make(T, len(rows), 1, 1, 1, 2, "bf16", seed=T)
    y = {n: torch.zeros((a.shape[0], N) + a.shape[2:] if n != "state0" else (N,) + a.shape[1:], dtype=a.dtype, device="cuda") for n, a in x.items()}
    ydo, yds = torch.zeros(T, N, 1, 2, dtype=do.dtype, device="cuda"), torch.zeros(N, 1, 1, 2, device="cuda")
    for n, a in x.items():
        if n == "state0":
            y[n][rows] = a
        else:
            y[n][:, rows] = a
    ydo[:, rows], yds[rows] = do, ds
    pick = lambda r: {n: a[rows] if "state" in n else a[:, rows] for n, a in r.items() if n != "workspace"}
    sizes = 1, 2, 17.0, True, T
    ref.check(pick(call(y)), *ref.oracle(x), *sizes)
    ref.check(pick(call(y, ydo, yds)), *ref.oracle(x, None, do, ds), *sizes)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("which", ["q", "k", "v", "do", "all"])
@pytest.mark.parametrize("T", [3, 35])
def test_steps_far_apart(torch_cuda, T, which, dtype):
    """More than 2^23 elements from step to step, as a packed projection of many rows has them: in 35 steps 640 MB (fp32 1.3 GB) and more."""
    torch = torch_cuda
    apart = (1 << 23) + (1 << 20) + 8
    x, do, ds = ref.make(T, 3, 2, 2, 64, 72, dtype, seed=T)
    want, back = call(x), call(x, do, ds)
    arrays = dict(q=x["q"], k=x["k"], v=x["v"], do=do)
    for n in arrays if which == "all" else (which,):
        a = arrays[n]
        whole = torch.full((T * apart,), float("nan"), dtype=a.dtype, device="cuda")
        far = whole.as_strided(a.shape, (apart,) + a.stride()[1:])
        far.copy_(a)
        arrays[n] = far
    y = dict(x, **{n: a for n, a in arrays.items() if n != "do"})
    sizes = 64, 72, 17.0, dtype == "bf16", T
    got, gback = call(y), call(y, arrays["do"], ds)
    ref.check(got, *ref.oracle(x), *sizes)
    ref.check(gback, *ref.oracle(x, None, do, ds), *sizes)
    assert all(torch.equal(a, got[n]) for n, a in want.items() if n != "workspace")
    assert all(torch.equal(a, gback[n]) for n, a in back.items() if n != "workspace")


@pytest.mark.parametrize("dtype,N", [("bf16", 1 << 14), ("fp32", 1 << 14), ("bf16", 1 << 15)])
@pytest.mark.parametrize("T", [2, 34])
def test_results_whose_steps_are_far_apart(torch_cuda, T, N, dtype):
    """2^24 or 2^25 numbers of o in a step: a chunk of results is 2^31 bytes, or in bf16 half of that; some rows, the first and last ones among them."""
    torch = torch_cuda
    rows = [0, 1, N // 2 + 5, N - 1]
    x, do, ds = ref.make(T, N, 8, 8, 8, 128, dtype, seed=T)
    pick = lambda r: {n: a[rows] if "state" in n else a[:, rows] for n, a in r.items() if n != "workspace"}
    few, sizes = pick(x), (8, 128, 17.0, dtype == "bf16", T)
    ref.check(pick(call(x)), *ref.oracle(few), *sizes)
    ref.check(pick(call(x, do, ds)), *ref.oracle(few, None, do[:, rows], ds[rows]), *sizes)
