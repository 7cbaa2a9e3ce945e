"""quant8 behind an activation whose value is too small for fp32 and whose second factor is large: the product counts all the same."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import act64
from plain8 import check_codes

pytestmark = pytest.mark.gpu
DEV = "cuda"
# where each activation falls through 2^-118, the last that fp32 arithmetic is good for
DEEP = {dvdq.ACT_SILU: (-100.0, -76.0), dvdq.ACT_GELU_TANH: (-11.0, -9.2), dvdq.ACT_GELU: (-15.0, -12.0)}


def test_one_value_deep_in_the_tail_is_the_largest():
    x = torch.tensor([[-90.0, -88.0, 1.0, 2.0, -3.0], [-88.0, 1.0, 0.5, 0.0, 1.0]], device=DEV)
    up = torch.tensor([[1e30, 1e29, 1e-9, -1e-9, 1e-9], [1e38, 1.0, 1.0, 1.0, -1.0]], device=DEV)
    z = act64(x.double().cpu(), dvdq.ACT_SILU) * up.double().cpu()
    codes, scale, sums = dvdq.quant8(x, up=up, act=dvdq.ACT_SILU, want_rowsum=True)
    assert int(codes[0, 0]) == -127 and int(codes[1, 0]) == -127
    check_codes(codes, scale, z, 1.0, 0.0, "largest", loose=True, rowsum=sums)


@pytest.mark.parametrize("act", DEEP)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [5, 30, 250, 520, 1533, 5120, 9001, 13824, 16384, 33000, 40001])
def test_rows_that_mix_tails_with_large_factors(C, dtype, act):
    """Rows of ordinary values with a few, or all, of their elements deep in the tail, of all sizes beside the others."""
    g = torch.Generator(device=DEV).manual_seed(C + act)
    uniform = lambda lo, hi, *s: lo + (hi - lo) * torch.rand(s, generator=g, device=DEV)   # noqa: E731
    rows = 24 if C < 9000 else 8
    x = 2 * torch.randn((rows, C), generator=g, device=DEV)
    up = torch.randn((rows, C), generator=g, device=DEV) * 10.0 ** uniform(-14, 4, rows, 1)
    some = torch.rand((rows, C), generator=g, device=DEV) < 3.0 / C
    some[0], some[1, C - 1], some[2, 0] = True, True, True
    sign = torch.randint(0, 2, (rows, C), generator=g, device=DEV) * 2.0 - 1
    x = torch.where(some, uniform(*DEEP[act], rows, C), x).to(dtype)
    up = torch.where(some, sign * 10.0 ** uniform(20, 38, rows, C), up).to(dtype)
    z = act64(x.cpu().double(), act) * up.cpu().double()
    codes, scale, sums = dvdq.quant8(x, up=up, act=act, want_rowsum=True)
    check_codes(codes, scale, z, 1.0, 0.0, f"{C} {dtype} act {act}", loose=True, rowsum=sums)
