"""Outputs of linear over a gate with a row per token, in the same places: every element is read where it is written, and nowhere else."""
import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(1, 300, 64), (7, 300, 64), (300, 264, 136), (129, 257, 1157), (512, 640, 4096), (3000, 520, 264)])
def test_output_over_the_gate(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, gate = (torch.randn(s, generator=g, device="cuda").to(torch.float16) for s in ((M, K), (N, K), (M, N)))
    want = dvdq.linear(x, w, gate=gate)
    y = gate.clone()
    assert dvdq.linear(x, w, gate=y, y=y) is y and torch.equal(y, want)


def test_refusals():
    x = torch.randn((64, 64), device="cuda").bfloat16()
    w = torch.randn((64, 64), device="cuda").bfloat16()
    y = torch.empty_like(x)
    for kw in (dict(y=x), dict(y=w), dict(bias=y[0], y=y), dict(gate=y[0], y=y), dict(gate=y[:2], y=y)):
        with pytest.raises(dvdq.DvdqError) as e:
            dvdq.linear(x, w, **kw)
        assert e.value.status == 3
