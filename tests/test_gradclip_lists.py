"""Lists of gradients that the binding of sf_gradclip has to take or refuse by what their tensors are (CPU)."""
import torch

from paper_2006_11751_amd import memory


def test_a_tensor_of_no_numbers_is_dense():
    """However its axes lie: it has no memory to fill."""
    for shape in ((0,), (0, 5), (5, 0), (2, 0), (3, 0, 4), (0, 0)):
        t = torch.zeros(shape)
        assert memory._dense(t), shape
        assert memory._dense(t.T if t.dim() == 2 else t), shape
    assert memory._dense(torch.zeros(4, 6)[:, :0]) and memory._dense(torch.zeros(4, 6)[:, 3:3].T)


def key(monkeypatch, *tensors):
    monkeypatch.setattr(memory, "_tensor_facts", None)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    return memory._list_key("grads", list(tensors))


def test_lists_that_are_the_same_and_that_are_not(monkeypatch):
    """By shapes, types and, of tensors that are not contiguous, strides."""
    z = torch.zeros
    base = key(monkeypatch, z(6, 4), z(5))
    assert base == key(monkeypatch, z(6, 4), z(5))
    for other in ((z(4, 6), z(5)), (z(24), z(5)), (z(6, 4), z(5, 1)), (z(6, 4), z(6)), (z(6, 4, dtype=torch.bfloat16), z(5)), (z(4, 6).T, z(5)), (z(6, 4),),
                  (z(6, 4), z(5), z(0))):
        assert base != key(monkeypatch, *other), [t.shape for t in other]
    assert key(monkeypatch, z(4, 6).T, z(5)) == key(monkeypatch, z(4, 6).T, z(5))
    # strides of an axis of one element, in a tensor that is contiguous: any
    one = z(7, 4)[::2][:1]
    assert one.stride() == (8, 1) and key(monkeypatch, one, z(4, 6).T) == key(monkeypatch, z(1, 4), z(4, 6).T)


def test_the_workspace_of_lists_that_take_several_launches():
    """A number for each chunk, and from 121 tensors that have numbers on one more for their sum."""
    import ctypes as C
    lib = memory.load_library()
    size = lambda *s: lib.sf_gradclip_workspace_bytes(len(s), (C.c_int64 * len(s))(*s))
    up = lambda n: (8 * n + 255) // 256 * 256
    for n in (1, 32, 33, 96, 120):
        assert size(*[5] * n) == up(n) and size(*[5] * n, *[0] * 200) == up(n)
    for n in (127, 128, 4095, 4096, 100000):
        assert size(*[5] * n) == up(n + 1)
