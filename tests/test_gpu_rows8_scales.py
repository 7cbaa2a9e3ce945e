"""Scales of rows to 8 bits are max|z| / 127 rounded once."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import F32, act64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("C", [7, 700, 6000, 40001])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_one_rounding(C, dtype):
    g = torch.Generator(device=DEV).manual_seed(C)
    rows = 4000 if C < 100 else 100
    x, up = ((torch.randn((rows, C), generator=g, device=DEV) * torch.exp(torch.randn((rows, 1), generator=g, device=DEV))).to(dtype) for _ in range(2))
    for act in (dvdq.ACT_NONE, dvdq.ACT_SILU):
        for second in (None, up):
            _, scale = dvdq.quant8(x, up=second, act=act)
            z = act64(x.cpu().double(), act)
            if second is not None:
                z = z * second.cpu().double()
            want = z.abs().amax(-1) / 127
            # half a unit of fp32, 2^-24 of the value, and what 64 bits lose in z, its maximum's quotient and the activation (a few 2^-52)
            assert ((scale.cpu().double() - want).abs() <= (F32 + 2.0 ** -48) * want).all(), (act, second is not None)
