"""include/sf_memory.h: every function it declares is exported and bound, the ctypes mirrors of its structs have the
sizes and offsets that the C compiler gives them, and bad arguments come back as errors without a GPU."""
import ctypes
import os
import re
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _memory():
    from paper_2006_11751_amd import binding, memory
    if not os.path.exists(binding.library_path()):
        binding.build_library()
    return memory


def test_every_declared_symbol_is_exported_and_bound():
    memory = _memory()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sf_memory.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(sf_[a-z0-9_]+)\s*\(", text))
    assert set(memory.EXPORTS) == names
    lib = memory.load_library()
    for n in names:
        assert getattr(lib, n).argtypes, n


def test_struct_layouts_match_the_header():
    memory = _memory()
    structs = {v: k for k, v in memory.STRUCTS.items()}
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "sf_memory.h"\nint main(void){\n'
    for s, name in structs.items():
        src += 'printf("%%zu\\n", sizeof(%s));\n' % name
        src += "".join('printf("%%zu\\n", offsetof(%s, %s));\n' % (name, f[0]) for f in s._fields_)
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "s.c"), os.path.join(d, "s")
        open(c, "w").write(src + "return 0;}\n")
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), c, "-o", exe], check=True)
        got = [int(v) for v in subprocess.run([exe], capture_output=True, check=True).stdout.split()]
    want = []
    for s in structs:
        want += [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


def test_linattn_refuses_without_a_gpu():
    memory = _memory()
    lib, C = memory.load_library(), memory.SfLinattnConfig
    err = lambda: lib.sf_last_error().decode()
    good = dict(struct_size=ctypes.sizeof(C), dtype=0, T=8, N=2, H=4, Hk=2, dk=16, dv=16, scale=0.25)
    make = lambda **kw: ctypes.byref(C(**dict(good, **kw)))
    none = [None] * 10
    assert lib.sf_linattn(None, *none) == -1
    for kw, code, text in ((dict(struct_size=4), -1, "struct_size"), (dict(dtype=2), -1, "dtype"), (dict(Hk=3), -2, "Hk = 3"),
                           (dict(H=0), -2, "H = 0"), (dict(T=-1), -2, "T = -1"), (dict(dk=129), -2, "dk = 129"), (dict(dv=0), -2, "dv = 0"),
                           (dict(scale=float("inf")), -2, "scale"), (dict(T=1 << 20, N=1 << 20), -2, "2^31"), ({}, -1, "q is null")):
        assert lib.sf_linattn(make(**kw), *none) == code and text in err(), (kw, err())
    assert lib.sf_linattn(make(), 2, 4, 4, 4, None, None, 4, None, None, None) == -1 and "q is null or not 4-byte" in err()
    assert lib.sf_linattn_backward(make(), *[None] * 14) == -1
    assert lib.sf_linattn_step(make(), *[None] * 5, 1, *[None] * 4) == -2 and "T = 8" in err()
    assert lib.sf_linattn_step(make(T=1), *[None] * 5, 1, *[None] * 4) == -2 and "no ids" in err()
    assert lib.sf_linattn_workspace_bytes(make(), 0) == 0
    assert lib.sf_linattn_workspace_bytes(make(Hk=3), 0) == -1
    assert lib.sf_linattn_workspace_bytes(make(), 1) >= 8 * 2 * 4 * 32 * 4  # the shared heads' partial sums


def test_resnorm_refuses_without_a_gpu():
    memory = _memory()
    lib, C = memory.load_library(), memory.SfResnormConfig
    err = lambda: lib.sf_last_error().decode()
    good = dict(struct_size=ctypes.sizeof(C), dtype=0, M=8, D=64, groups=1, post=1, pre=1, gate_act=0, eps=1e-6, b_stride=64)
    make = lambda **kw: ctypes.byref(C(**dict(good, **kw)))
    for kw, code, text in ((dict(struct_size=4), -1, "struct_size"), (dict(dtype=2), -1, "dtype"), (dict(post=3), -1, "post = 3"),
                           (dict(pre=-1), -1, "pre = -1"), (dict(gate_act=3), -1, "gate_act"), (dict(M=-1), -2, "M = -1"), (dict(D=0), -2, "D = 0"),
                           (dict(D=8193), -2, "8193"), (dict(groups=5), -2, "groups = 5"), (dict(groups=2), -2, "groups = 2"),
                           (dict(eps=-1.0), -2, "eps"), (dict(eps=float("nan")), -2, "eps"), ({}, -1, "b is null")):
        assert lib.sf_resnorm(make(**kw), *[None] * 9) == code and text in err(), (kw, err())
    assert lib.sf_resnorm(make(gate_act=1), 16, None, None, None, None, None, 16, 16, None) == -1 and "gate" in err()
    assert lib.sf_resnorm(make(), 16, None, None, None, None, None, 16, None, None) == -1 and "n is null" in err()
    assert lib.sf_resnorm_backward(make(), 16, *[None] * 15) == -1 and "dn" in err()
    assert lib.sf_resnorm_workspace_bytes(make(groups=5)) == -1
    assert lib.sf_resnorm_workspace_bytes(make()) > 0


def test_ffn_refuses_without_a_gpu():
    memory = _memory()
    lib, C = memory.load_library(), memory.SfFfnConfig
    err = lambda: lib.sf_last_error().decode()
    good = dict(struct_size=ctypes.sizeof(C), dtype=1, M=8, D=64, F=128, act=0, x_stride=64, w_gate_stride=64, w_up_stride=64,
                w_down_stride=128, dy_stride=64)
    make = lambda **kw: ctypes.byref(C(**dict(good, **kw)))
    for kw, code, text in ((dict(struct_size=4), -1, "struct_size"), (dict(dtype=2), -1, "dtype"), (dict(act=3), -1, "act = 3"),
                           (dict(M=-1), -2, "M = -1"), (dict(D=0), -2, "D = 0"), (dict(F=1 << 21), -2, "F = "), ({}, -1, "x is null")):
        assert lib.sf_ffn(make(**kw), *[None] * 7) == code and text in err(), (kw, err())
        assert lib.sf_ffn_backward(make(**kw), *[None] * 11) == code and text in err(), (kw, err())
    assert lib.sf_ffn(make(), 16, 16, 16, 16, 8, 256, None) == -1 and "y is" in err()
    assert lib.sf_ffn(make(), 16, 16, 16, 16, 16, 128, None) == -1 and "workspace" in err()
    assert lib.sf_ffn(make(), 16, 16, 17, 16, 16, 256, None) == -1 and "w_up" in err()
    assert lib.sf_ffn_workspace_bytes(make(act=-1), 0) == -1
    assert lib.sf_ffn_workspace_bytes(make(), 0) >= 8 * 128 * 2
    assert lib.sf_ffn_workspace_bytes(make(M=100), 1) > lib.sf_ffn_workspace_bytes(make(M=100), 0) > 0


def test_linattn_refuses_states_that_overlap():
    """(Addresses that are never read: the calls come back before they launch anything.)"""
    memory = _memory()
    lib, C = memory.load_library(), memory.SfLinattnConfig
    cfg = ctypes.byref(C(struct_size=ctypes.sizeof(C), dtype=0, T=8, N=2, H=4, Hk=4, dk=16, dv=16, scale=0.25))
    size = 2 * 4 * 16 * 16 * 4
    a, states = 1 << 20, 1 << 24
    for off in (4 - size, -size // 2, 4, size - 4):
        assert lib.sf_linattn(cfg, a, a, a, a, None, states, a, states + off, None, None) == -4, off
        assert "state overlaps state0" in lib.sf_last_error().decode()
    for off in (4 - size, -size // 2, 0, 4, size - 4):
        for where in ((states, states + (1 << 20)), (states + (1 << 20), states)):  # state0, dstate
            assert lib.sf_linattn_backward(cfg, a, a, a, a, a, None, *where, a, a, a, states + off, None, None) == -4, off
            assert "dstate0 overlaps" in lib.sf_last_error().decode()


def test_resnorm_refuses_the_gradient_of_a_gate_that_is_not_there():
    """(Nothing would be written to it.)"""
    memory = _memory()
    lib, C = memory.load_library(), memory.SfResnormConfig
    cfg = ctypes.byref(C(struct_size=ctypes.sizeof(C), dtype=0, M=8, D=64, groups=1, post=1, pre=0, gate_act=0, eps=1e-6, b_stride=64, dy_stride=64))
    a = 1 << 20
    assert lib.sf_resnorm_backward(cfg, a, None, a, None, None, None, a, None, None, a, a, None, None, None, None, None) == -1
    assert "dgate" in lib.sf_last_error().decode()


def test_linattn_is_cut_into_pieces_only_where_workgroups_are_few():
    """What pieces need is in the workspace; a head of more than 64 columns has two workgroups."""
    memory = _memory()
    lib, C = memory.load_library(), memory.SfLinattnConfig
    size = lambda T, N, d, back: lib.sf_linattn_workspace_bytes(ctypes.byref(C(
        struct_size=ctypes.sizeof(C), dtype=1, T=T, N=N, H=8, Hk=8, dk=d, dv=d, scale=1.0)), back)
    for T, N, d, back, cut in ((4096, 1, 64, 0, 1), (512, 1, 64, 0, 0), (4096, 30, 64, 0, 1), (4096, 60, 64, 0, 0), (4096, 12, 64, 1, 1),
                               (4096, 4, 128, 0, 1), (4096, 12, 128, 0, 1), (4096, 30, 128, 0, 0), (4096, 6, 128, 1, 1), (4096, 12, 128, 1, 0)):
        assert (size(T, N, d, back) > 0) == bool(cut), (T, N, d, back)
