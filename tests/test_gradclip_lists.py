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
