"""Group norm of groups with one value that is nothing like the others, wherever it stands: the statistics are as good as without it."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import assert_close, group_norm64

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# groups that fit a workgroup's registers, in pieces of 16 bytes down to one element, then ones that do not
@pytest.mark.parametrize("shape", [(1, 1024, 16, 1), (2, 300, 64, 4), (1, 700, 48, 4), (1, 900, 20, 2), (1, 500, 30, 2), (1, 3, 8, 1),
                                   (1, 40000, 16, 1), (1, 9000, 30, 2), (2, 20000, 64, 4)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_one_large_value(shape, dtype):
    B, S, C, groups = shape
    g = torch.Generator().manual_seed(3)
    x = torch.randn((B, S, C), generator=g).to(DTYPES[dtype]).cuda()
    for value in (100.0, -3e4) + ((1e6,) if dtype != "fp16" else ()):
        for s, c in ((0, 0), (0, C // groups - 1), (1, 0), (S // 2, C // groups // 2), (S - 1, C // groups - 1)):
            t = x.clone()
            t[:, s, c] = value                        # in the first group; the others have none
            for act in (0, 1):
                ref, slack = group_norm64(t, groups, act=act)
                assert_close(dvdq.group_norm(t, groups, act=act), ref, slack, f"{value} at {s}, {c}, act {act}")
