"""A workspace on another device than the tensors is refused by the binding, as every other tensor there is.  CPU only: nothing is launched."""
import pytest
import torch

import paper_2505_18663_amd as dvdq


class OnDevice(torch.Tensor):
    """A CPU tensor that says it is on a GPU."""
    is_cuda = True
    index = 0

    @property
    def device(self):
        return torch.device("cuda", self.index)


def on(index, *shape, dtype=torch.bfloat16):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)
    t.index = index
    return t


def test_workspace_of_another_device():
    here, there = (on(i, 1 << 16, dtype=torch.uint8) for i in (0, 1))
    assert dvdq._workspace(here, 100, torch.device("cuda", 0), None)[1] == 1 << 16
    x, w, y = on(0, 40, 64), on(0, 24, 64), on(0, 40, 24)
    with pytest.raises(ValueError, match="workspace"):
        dvdq.linear(x, w, y=y, workspace=there)
    with pytest.raises(ValueError, match="workspace"):
        dvdq.group_norm(on(0, 2, 10, 8), 2, y=on(0, 2, 10, 8), workspace=there)
    with pytest.raises(TypeError):
        dvdq.linear(x, w, y=y, workspace=torch.zeros((1 << 16,), dtype=torch.uint8))
