"""Group norm of values whose squares are beyond fp32: a constant group has no deviations, however large the constant."""
import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu


# C / groups: whole pieces of 16 bytes, and not; S: in one launch; in slabs, the last of them with fewer rows than a workgroup takes at once
@pytest.mark.parametrize("C,groups", [(48, 6), (30, 3), (48, 16), (7, 1)])
@pytest.mark.parametrize("S", [3, 2000, 40970])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [1e20, -3e38])
def test_large_constant_groups(value, dtype, S, C, groups):
    x = torch.full((2, S, C), value, dtype=dtype, device="cuda")
    w = torch.full((C,), 2.0, dtype=dtype, device="cuda")
    b = torch.arange(C, dtype=dtype, device="cuda")
    assert torch.equal(dvdq.group_norm(x, groups, w, b), b.expand(2, S, C))
