"""The reference of the gated delta rule (tests/delta_reference.py) against differences and autograd, and what the binding and
the library refuse, on the CPU."""
import ctypes as C
import os

import pytest
import torch

from tests import delta_reference as ref


def test_its_gradients_against_differences():
    x, do, ds = ref.make(9, 2, 4, 2, 3, 5, torch.float64, p_done=0.2, seed=1, device="cpu")
    x = {n: (a if n == "done" else a.double()) for n, a in x.items()}
    x["done"][4, 0] = 1
    x["log_decay"][6, 1, 2] = -1000.0  # (begins the memory anew)
    do, ds = do.double(), ds.double()
    value = lambda y: sum((ref.oracle(y, scale=0.7)[0][n] * g).sum() for n, g in (("o", do), ("state", ds)))
    got, _ = ref.oracle(x, 0.7, do, ds)
    g = torch.Generator().manual_seed(2)
    for name in ("q", "k", "v", "log_decay", "beta", "state0"):
        for _ in range(3):
            way = torch.randn(x[name].shape, generator=g, dtype=torch.float64)
            h = 1e-5
            slope = (value(dict(x, **{name: x[name] + h * way})) - value(dict(x, **{name: x[name] - h * way}))) / (2 * h)
            want = (got["d" + name] * way).sum()
            assert abs(slope - want) <= 1e-7 * (got["d" + name].abs() * way.abs()).sum(), name  # (h^2, and 2^-53 / h)


def test_its_gradients_against_autograd():
    x, do, ds = ref.make(40, 2, 3, 1, 8, 4, torch.float64, seed=3, device="cpu")
    leaf = {n: (a if n == "done" else a.double().requires_grad_()) for n, a in x.items()}
    k, q = (leaf[n].repeat_interleave(3, 2) for n in "kq")
    s, out = leaf["state0"], 0.0
    for t in range(40):
        s = (leaf["log_decay"][t].exp() * (x["done"][t] == 0)[:, None])[..., None, None] * s
        s = s + k[t][..., None] * (leaf["beta"][t][..., None] * (leaf["v"][t] - (s * k[t][..., None]).sum(-2)))[..., None, :]
        out = out + (8 ** -0.5 * (s * q[t][..., None]).sum(-2) * do[t].double()).sum()
    names = [n for n in leaf if n != "done"]
    want = torch.autograd.grad(out + (s * ds.double()).sum(), [leaf[n] for n in names])
    got, _ = ref.oracle(x, None, do, ds)
    for n, w in zip(names, want):
        # (where done is set the decay's gradient is 0 in both)
        assert (got["d" + n] - w).abs().max() <= 1e-12 * w.abs().max(), n


# ---- refusals -------------------------------------------------------------------------------


def _memory():
    from paper_2006_11751_amd import binding, memory
    if not os.path.exists(binding.library_path()):
        binding.build_library()
    return memory


GOOD = dict(dtype=0, T=8, N=2, H=4, Hk=2, dk=16, dv=16, scale=0.25)


def _config(memory, **kw):
    S = memory.SfDeltaruleConfig
    return C.byref(S(**dict(dict(struct_size=C.sizeof(S)), **dict(GOOD, **kw))))


@pytest.mark.parametrize("kw,code,text", [
    (dict(struct_size=4), -1, "struct_size"), (dict(dtype=2), -1, "dtype"), (dict(Hk=3), -2, "Hk = 3"), (dict(H=0), -2, "H = 0"), (dict(T=-1), -2, "T = -1"),
    (dict(N=-1), -2, "N = -1"), (dict(dk=129), -2, "dk = 129"), (dict(dk=0), -2, "dk = 0"), (dict(dv=0), -2, "dv = 0"), (dict(dv=129), -2, "dv = 129"),
    (dict(scale=float("inf")), -2, "scale"), (dict(scale=float("nan")), -2, "scale"), (dict(T=1 << 20, N=1 << 20), -2, "2^31"),
    (dict(T=1 << 15, N=1 << 15, H=128), -2, "2^21"), (dict(T=1 << 17, N=1 << 14, H=128), -2, "2^31"), ({}, -1, "q is null")])
def test_bad_configurations(kw, code, text):
    memory = _memory()
    lib = memory.load_library()
    err = lambda: lib.sf_last_error().decode()
    assert lib.sf_deltarule(_config(memory, **kw), *[None] * 11) == code and text in err(), err()
    assert lib.sf_deltarule_backward(_config(memory, **kw), *[None] * 17) == code and text in err(), err()
    if "T" not in kw:
        assert lib.sf_deltarule_step(_config(memory, T=1, **kw), *[None] * 6, 9, *[None] * 4) == code and text in err(), err()
    assert kw == {} or lib.sf_deltarule_workspace_bytes(_config(memory, **kw), 1) == -1
    assert lib.sf_deltarule(None, *[None] * 11) == -1


def test_the_most_chunks_of_a_call():
    """What a launch can count: 2^26 chunks of 32 steps forwards, 2^23 for gradients, less 128."""
    memory = _memory()
    lib = memory.load_library()
    size = lambda backward, **kw: lib.sf_deltarule_workspace_bytes(_config(memory, Hk=1, dk=1, dv=1, **kw), backward)
    for backward, T in ((0, 1 << 13), (1, 1 << 10)):
        assert size(backward, T=32 * T - 32, N=1 << 11, H=4) > 0
        assert size(backward, T=32 * T, N=1 << 11, H=4) == -1 and "2^2%d" % (3 if backward else 6) in lib.sf_last_error().decode()
    kw = dict(T=1 << 15, N=1 << 11, H=4, Hk=1, dk=1, dv=1)
    assert lib.sf_deltarule_backward(_config(memory, **kw), *[None] * 17) == -2 and "2^23" in lib.sf_last_error().decode()
    assert lib.sf_deltarule(_config(memory, **kw), *[None] * 11) == -1 and "q is null" in lib.sf_last_error().decode()
    assert lib.sf_deltarule(_config(memory, **dict(kw, T=1 << 18)), *[None] * 11) == -2 and "2^26" in lib.sf_last_error().decode()


def test_bad_pointers_and_tables():
    """(Addresses that are never read: the calls come back before they launch anything.)"""
    memory = _memory()
    lib = memory.load_library()
    err = lambda: lib.sf_last_error().decode()
    a = 1 << 20
    names = ("q", "k", "v", "log_decay", "beta", None, "state0", "o", "state")
    for i, name in enumerate(names):
        if name is None:
            continue
        args = [a, a, a, a, a, None, None, a, None]
        args[i] = a + 2
        assert lib.sf_deltarule(_config(memory), *args, None, None) == -1 and name + " is null or not 4-byte" in err(), (name, err())
    names = ("q", "k", "v", "log_decay", "beta", "do", None, "state0", "dstate", "dq", "dk", "dv", "dlog_decay", "dbeta", "dstate0")
    for i, name in enumerate(names):
        if name is None:
            continue
        args = [a] * 6 + [None] * 3 + [a] * 5 + [None]
        args[i] = a + 2
        assert lib.sf_deltarule_backward(_config(memory), *args, a, None) == -1 and name + " is null or not 4-byte" in err(), (name, err())
    assert lib.sf_deltarule_backward(_config(memory), *[a] * 6, *[None] * 3, *[a] * 5, None, None, None) == -1 and "workspace" in err()
    step = lambda n_env, table=a, ids=None, T=1: lib.sf_deltarule_step(_config(memory, T=T), a, a, a, a, a, table, n_env, ids, None, a, None)
    assert step(2, T=8) == -2 and "T = 8" in err()
    assert step(0) == -2 and "n_env = 0" in err()
    assert step(1) == -2 and "no ids" in err()
    assert step(2, table=a + 4) == -1 and "state_table" in err()
    assert step(2, ids=a + 1) == -1 and "env_ids" in err()


def test_states_that_overlap():
    memory = _memory()
    lib = memory.load_library()
    cfg = _config(memory, Hk=4)
    size = 2 * 4 * 16 * 16 * 4
    a, states = 1 << 20, 1 << 24
    for off in (4 - size, -size // 2, 4, size - 4):
        assert lib.sf_deltarule(cfg, a, a, a, a, a, None, states, a, states + off, None, None) == -4, off
        assert "state overlaps state0" in lib.sf_last_error().decode()
    for off in (4 - size, -size // 2, 0, 4, size - 4):
        for where in ((states, states + (1 << 20)), (states + (1 << 20), states)):  # state0, dstate
            assert lib.sf_deltarule_backward(cfg, *[a] * 6, None, *where, *[a] * 5, states + off, a, None) == -4, off
            assert "dstate0 overlaps" in lib.sf_last_error().decode()


def test_workspace_bytes():
    memory = _memory()
    lib = memory.load_library()
    size = lambda back, **kw: lib.sf_deltarule_workspace_bytes(_config(memory, **kw), back)
    assert size(0) == 0 and size(0, T=32) == 0 and size(1, Hk=4, T=32) == 0
    assert size(0, T=33) >= 2 * 2 * 4 * 2 * 32 * 32 * 4             # two matrices for each chunk
    assert size(1) >= 2 * 8 * 2 * 4 * 16 * 4                        # the shared heads' partial sums
    assert size(1, Hk=4, T=33) >= 2 * 2 * 2 * 4 * 16 * 16 * 4  # two states for each chunk


def test_the_binding_refuses_what_is_not_on_the_gpu():
    memory = _memory()
    x, do, ds = ref.make(3, 2, 2, 2, 8, 8, "fp32", device="cpu")
    args = [x[n] for n in ("q", "k", "v", "log_decay", "beta")]
    with pytest.raises(ValueError, match="not on the GPU"):
        memory.delta_rule(*args)
    with pytest.raises(ValueError, match="not on the GPU"):
        memory.delta_rule_backward(*args, do)
    with pytest.raises(ValueError, match="not on the GPU"):
        memory.delta_rule_step(*(a[0] for a in args), ds)
