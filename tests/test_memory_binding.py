"""The buffers that a program of the memory operators keeps (paper_2006_11751_amd/memory.py), on the CPU."""
import types

import pytest


def _plan(n_bytes):
    import torch
    return types.SimpleNamespace(n_bytes=n_bytes, device=torch.device("cpu"))


def test_a_workspace_that_is_outgrown_stays_in_the_dict():
    """A graph that was recorded with it goes on writing to it."""
    from paper_2006_11751_amd import memory
    out, used = {}, []
    for n in (100, 5000, 5000, 64, 90000, 5000):
        used.append(memory._workspace(out, _plan(n)))
        assert out["workspace"].numel() >= n and out["workspace"].data_ptr() == used[-1]
    assert used[1] == used[2] == used[3] and used[4] == used[5]
    assert set(used) == {t.data_ptr() for t in out.values()} and len(out) == 3
    assert memory._workspace({}, _plan(0)) is None


def test_a_workspace_with_gaps_is_refused():
    """Its number of elements says nothing of the bytes from its first one on."""
    import torch
    from paper_2006_11751_amd import memory
    for w in (torch.empty(1, dtype=torch.uint8).expand(4096), torch.empty(8192, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            memory._workspace(dict(workspace=w), _plan(2048))
