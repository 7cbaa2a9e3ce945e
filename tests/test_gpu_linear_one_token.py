"""Products of one token whose operands are rows of larger tensors: one row has no pitch, so the strides of its first dimension may be anything."""
import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu
DEV = "cuda"
# a long clip's last token x[:, -1], 2^29 bytes, more than 2^32 bytes for every row, and what no tensor has
PITCHES = [32760 * 5120, 118800 * 5120, 1 << 28, 1 << 31, 1 << 40]
# (N, K, whether rows are whole pieces): as tiles in parts of K, of whole channels and not; through registers; copied first; few tokens
SIZES = [(320, 4104, True), (333, 4104, True), (5120, 5120, True), (333, 4104, False), (65, 4099, False), (5000, 4099, False), (333, 512, True)]


def lay(t, pitch):
    """t [1, n] where it is, its first dimension's stride something else"""
    return t.as_strided((1, t.size(1)), (pitch, 1))


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_any_pitch(size, dtype):
    N, K, whole = size
    if K > 4096:
        assert dvdq.bench_linear_choice(1, N, K, not whole) != -1
    g = torch.Generator(device=DEV).manual_seed(N + K)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)   # noqa: E731
    x, w, bias, gate, residual = r(1, K + 1)[:, 1 - whole:K + 1 - whole], r(N, K), r(N), r(1, N), r(1, N)
    want = dvdq.linear(x, w, bias, dvdq.ACT_SILU, gate, residual)
    for pitch in PITCHES:
        y = torch.zeros((1, N), dtype=dtype, device=DEV)
        got = dvdq.linear(lay(x, pitch), w, bias, dvdq.ACT_SILU, lay(gate, pitch), lay(residual, pitch), y=lay(y, pitch))
        assert torch.equal(got, want) and torch.equal(y, want), pitch
        y = residual.clone()
        dvdq.linear(x, w, bias, dvdq.ACT_SILU, gate, lay(y, pitch), y=lay(y, pitch))
        assert torch.equal(y, want), f"in place, {pitch}"


@pytest.mark.parametrize("size", [(333, 4104), (70, 513)])
def test_any_pitch_of_8_bit_rows(size):
    N, K = size
    g = torch.Generator(device=DEV).manual_seed(N)
    i = lambda *s: torch.randint(-127, 128, s, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)   # noqa: E731
    x, w, xs, ws = i(1, K), i(N, K), torch.rand((1,), generator=g, device=DEV), torch.rand((N,), generator=g, device=DEV)
    residual = torch.randn((1, N), generator=g, device=DEV)
    want = dvdq.linear8(x, xs, w, ws, residual=residual, dtype=torch.float32)
    for pitch in PITCHES:
        y = torch.zeros((1, N), device=DEV)
        dvdq.linear8(lay(x, pitch), xs, w, ws, residual=lay(residual, pitch), y=lay(y, pitch))
        assert torch.equal(y, want), pitch


def test_the_last_token_of_a_clip():
    """The residual as a model has it, not laid by hand: the address 4 GiB below it belongs to nobody."""
    hidden = torch.empty((1, 32760, 5120), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    hidden[:, -1] = torch.randn((1, 5120), generator=g, device=DEV).bfloat16()
    x, w = (torch.randn(s, generator=g, device=DEV).bfloat16() for s in ((1, 5120), (5120, 5120)))
    last = hidden[:, -1]
    assert last.stride(0) == 32760 * 5120
    assert torch.equal(dvdq.linear(x, w, residual=last), dvdq.linear(x, w, residual=last.clone()))


@pytest.mark.parametrize("M,K", [(1, 4104), (40, 264), (300, 260), (200, 4099)])
def test_one_channel_of_any_pitch(M, K):
    """The same of weights that are one row."""
    g = torch.Generator(device=DEV).manual_seed(M)
    x, w = (torch.randn((n, K), generator=g, device=DEV).bfloat16() for n in (M, 1))
    want = dvdq.linear(x, w)
    for pitch in PITCHES:
        assert torch.equal(dvdq.linear(x, lay(w, pitch)), want), pitch
