"""More rows than one launch takes: 2^21 workgroups, of 32 rows where they are short, and a loop over rows where they are long."""
import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu
DEV = "cuda"


def windows(g, rows, C, dtype=torch.bfloat16):
    """[rows, C] whose rows begin an element apart: all of them different, in little memory"""
    return torch.randn((rows + C,), generator=g, device=DEV).to(dtype).as_strided((rows, C), (1, 1))


def test_short_rows():
    rows, C = (1 << 26) + 33, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    x = windows(g, rows, C)
    codes, scale, sums = dvdq.quant8(x, want_rowsum=True)
    for first in range(0, rows, 1 << 24):
        a, b, c = dvdq.quant8(x[first:first + (1 << 24)], want_rowsum=True)
        part = slice(first, first + len(b))
        assert torch.equal(codes[part], a) and torch.equal(scale[part], b) and torch.equal(sums[part], c), first
    assert len(b) == 33 and bool(b.all())


@pytest.mark.parametrize("B,S", [(3, 22369633), (22369633, 3), (67, 1001627)])
def test_short_rows_of_batches(B, S):
    """Rows found by a division, at numbers up to 2^26."""
    C = 8
    assert B * S > 1 << 26
    g = torch.Generator(device=DEV).manual_seed(2)
    flat = windows(g, B * (S + 5), C)
    x = flat.as_strided((B, S, C), (S + 5, 1, 1))                             # (batches lie apart)
    w = torch.randn((C,), generator=g, device=DEV).bfloat16()
    y = dvdq.rms_norm(x, w)
    codes, scale = dvdq.rms_norm_quant(x, w)
    want = dvdq.rms_norm(flat[:1 << 24], w)
    # some whole batches, and rows on both sides of the launches' border
    at = (1 << 26) // S
    for b in {0, 1, B // 2, at - 1, at, min(at + 1, B - 1), B - 1}:
        for s0 in {0, max((1 << 26) % S - 40, 0), max(S - 70, 0)}:
            part = flat[b * (S + 5) + s0:b * (S + 5) + min(s0 + 70, S)]
            n = len(part)
            assert torch.equal(y[b, s0:s0 + n], dvdq.rms_norm(part, w)), (b, s0)
            c, t = dvdq.rms_norm_quant(part, w)
            assert torch.equal(codes[b, s0:s0 + n], c) and torch.equal(scale[b, s0:s0 + n], t), (b, s0)
    n = min(S, 1 << 24)
    assert torch.equal(y[0, :n], want[:n])


@pytest.mark.parametrize("rows,C", [((1 << 21) + 5, 2056), ((1 << 20) + 3, 32776)])
def test_longer_rows(rows, C):
    g = torch.Generator(device=DEV).manual_seed(3)
    x = windows(g, rows, C)
    codes, scale = dvdq.quant8(x)
    for first in (0, 1000, rows // 2, rows - 40):
        a, b = dvdq.quant8(x[first:first + 40])
        assert torch.equal(codes[first:first + 40], a) and torch.equal(scale[first:first + 40], b), first
