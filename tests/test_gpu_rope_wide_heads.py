"""Heads as wide as they may be, of which a part is turned: every element of a new output is written."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import F32, assert_close, rope64

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D", [1021, 1022, 1023, 1024])
def test_part_of_a_wide_head(D, interleaved, dtype):
    g = torch.Generator().manual_seed(D)
    q, k = (torch.randn((2, 3, h, D), generator=g).to(DTYPES[dtype]).cuda() for h in (9, 2))
    pos = torch.randint(0, 40, (2, 3), generator=g, dtype=torch.int32).cuda()
    for R in (2, 4, 6, 510, 514, 1016, 1018, 1020, D // 2 * 2):
        table = dvdq.rope_table(40, dvdq.rope_frequencies(R)[0])
        out = [torch.full_like(t, float("nan")) for t in (q, k)]
        dvdq.rope(q, k, table, pos, None, interleaved, q_out=out[0], k_out=out[1])
        for name, x, y in zip("qk", (q, k), out):
            ref, mag = rope64(x, table, pos[..., None], (R,), interleaved)
            assert_close(y, ref, 3 * F32 * mag, f"{name}, {R} of {D}")
            assert torch.equal(y[..., R:], x[..., R:])
        dvdq.rope(q, None, table, pos, None, interleaved, q_out=out[0].copy_(q))       # in place
        dvdq.rope(out[0], None, table, pos, None, interleaved, q_out=out[0])
        twice = dvdq.rope(dvdq.rope(q, None, table, pos, None, interleaved), None, table, pos, None, interleaved)
        assert torch.equal(out[0], twice)
