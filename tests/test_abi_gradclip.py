"""sf_gradclip (include/sf_memory.h): bad arguments come back as errors without a GPU (addresses that are never read: the
calls come back before they launch anything), and what the binding refuses."""
import ctypes as C
import os

import pytest


def _memory():
    from paper_2006_11751_amd import binding, memory
    if not os.path.exists(binding.library_path()):
        binding.build_library()
    return memory


A = 1 << 20  # an address


def _call(memory, sizes=(8, 8), dtypes=(0, 0), grads=(A, A + 4096), out=(A, A + 4096), norm=A + 65536, workspace=A + 131072, max_norm=1.0,
          eps=1e-6, size=None, n=None, null=()):
    lib, k = memory.load_library(), len(sizes)
    cfg = memory.SfGradclipConfig(C.sizeof(memory.SfGradclipConfig) if size is None else size, k if n is None else n, max_norm, eps)
    arrays = dict(grads=(C.c_void_p * k)(*grads), sizes=(C.c_int64 * k)(*sizes), dtypes=(C.c_int32 * k)(*dtypes), out=(C.c_void_p * k)(*out))
    arrays.update({a: None for a in null})
    rc = lib.sf_gradclip(C.addressof(cfg), arrays["grads"], arrays["sizes"], arrays["dtypes"], arrays["out"], norm, workspace, None)
    return rc, lib.sf_last_error().decode()


@pytest.mark.parametrize("kw,code,text", [
    (dict(size=4), -1, "struct_size"), (dict(n=-1), -2, "-1 tensors"), (dict(n=(1 << 20) + 1), -2, "tensors"), (dict(null=("sizes",)), -1, "sizes is null"),
    (dict(sizes=(8, -1)), -2, "tensor 1 of -1"), (dict(sizes=((1 << 40) + 1, 8)), -2, "tensor 0"), (dict(max_norm=-1.0), -2, "max_norm"),
    (dict(max_norm=float("nan")), -2, "max_norm"), (dict(eps=0.0), -2, "eps"), (dict(eps=float("inf")), -2, "eps"), (dict(eps=float("nan")), -2, "eps"),
    (dict(null=("grads",)), -1, "null"), (dict(null=("dtypes",)), -1, "null"), (dict(null=("out",)), -1, "null"), (dict(norm=None), -1, "norm"),
    (dict(norm=A + 65538), -1, "norm"), (dict(workspace=None), -1, "workspace"), (dict(workspace=A + 131072 + 16), -1, "workspace"),
    (dict(dtypes=(0, 2)), -1, "dtype of tensor 1"), (dict(grads=(A, None)), -1, "tensor 1"), (dict(out=(None, A)), -1, "tensor 0"),
    (dict(grads=(A + 2, A + 4096)), -1, "tensor 0"), (dict(grads=(A, A + 4097), dtypes=(0, 1)), -1, "tensor 1")])
def test_bad_arguments(kw, code, text):
    rc, err = _call(_memory(), **kw)
    assert rc == code and text in err, (rc, err)


@pytest.mark.parametrize("kw", [
    dict(grads=(A, A), out=(A, A)),                               # the same tensor twice
    dict(grads=(A, A + 28), out=(A, A + 28)),                     # one that begins in another
    dict(out=(A, A)),                                             # two results at one place, one of them a gradient
    dict(out=(A + 4096, A)),                                      # results at each other's gradient
    dict(out=(A + 4, A + 4096)),                                  # a result that overlaps its own gradient in part
    dict(out=(A + 8192, A + 8192 + 31)) | dict(dtypes=(1, 1), out=(A + 8192, A + 8192 + 14)),
    dict(norm=A + 28), dict(norm=A + 131072), dict(workspace=A + 4096), dict(sizes=(1 << 16, 8), grads=(A - 4096, A + (1 << 21)), out=(A - 4096, A + (1 << 21)))])
def test_overlaps_are_refused(kw):
    rc, err = _call(_memory(), **kw)
    assert rc == -4 and "overlaps" in err, (rc, err)


def test_workspace_bytes():
    lib = _memory().load_library()
    size = lambda *s: lib.sf_gradclip_workspace_bytes(len(s), (C.c_int64 * len(s))(*s))
    assert size() == 0 and size(0, 0) == 0 and size(1) == 256 and size(*[1] * 40) == 512
    assert size(-1) == -1 and lib.sf_gradclip_workspace_bytes(1, None) == -1
    # a number for each chunk, at most 2048 and one more for each tensor's rest
    assert size(1 << 40) <= 8 * 2049 + 256 and size(1 << 30, 1, 1 << 31) <= 8 * 2051 + 256


def test_the_binding_refuses():
    import torch
    memory = _memory()
    for grads, text in (([], "an empty list"), ([torch.zeros(3)], "CPU"), ([None], "a list of tensors"), ([torch.zeros(2), 3.0], "a list of tensors")):
        with pytest.raises(ValueError, match=text):
            memory.clip_gradients(grads, 1.0)


def test_what_is_dense():
    import torch
    memory = _memory()
    t = torch.zeros(4, 6, 5)
    for a, dense in ((t, True), (t.transpose(0, 2), True), (t.permute(1, 0, 2), True), (t[:, :3], False), (t[:1], True), (t[:, ::2], False), (t[0, 0, 0], True),
                     (t[:, :1, :1], False), (torch.zeros(3).expand(4, 3), False), (torch.zeros(2, 3, 4, 5).contiguous(memory_format=torch.channels_last), True),
                     (torch.zeros(3, 1).expand(3, 2), False)):
        assert memory._dense(a) == dense, (a.shape, a.stride())
