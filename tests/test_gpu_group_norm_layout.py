"""A new output of group_norm lies in memory as x does, whichever way the call takes."""
import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu


def tensors():
    r = lambda *s: torch.randn(s, device="cuda").bfloat16()   # noqa: E731
    yield r(3, 40, 48)
    yield r(40, 3, 48).transpose(0, 1)                              # batches inside of rows
    yield r(3, 40, 50)[:, :, 1:49]                                  # not dense
    yield r(40, 6, 48).transpose(0, 1)[::2]
    yield r(1, 40, 48).expand(3, -1, -1)
    yield r(3, 40, 1)
    yield r(3, 1, 40).transpose(1, 2)
    yield r(3, 48)
    yield r(2, 48, 5, 8).contiguous(memory_format=torch.channels_last).movedim(1, -1)



def test_layout(monkeypatch):
    dvdq.lib()
    native = dvdq._marshal
    assert native.__file__ == dvdq._MARSHAL_PATH
    for x in tensors():
        groups = 6 if x.shape[-1] % 6 == 0 else 1
        out = []
        for path in (native, dvdq._Handback):
            monkeypatch.setattr(dvdq, "_marshal", path)
            out.append(dvdq.group_norm(x, groups, act=dvdq.ACT_SILU))
        a, b = out
        want = torch.empty_like(x).stride()
        assert a.shape == x.shape and a.stride() == b.stride() == want, (x.shape, x.stride(), a.stride(), b.stride())
        assert torch.equal(a, b) and torch.equal(a, dvdq.group_norm(x.contiguous(), groups, act=dvdq.ACT_SILU))
