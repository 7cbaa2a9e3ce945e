"""Rows of every length that are no whole 16-byte pieces: what lies beside a row does not enter, and tiles end with tokens, channels or both."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import assert_close, linear64
from plain8 import linear8_64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_length_of_16_bit_rows(dtype):
    g = torch.Generator(device=DEV).manual_seed(1)
    M, N = 40, 72
    nan = float("nan")
    for K in (*range(1, 140), 191, 193, 255, 257, 1027):
        xb, wb = (torch.full((n + 2, K + 5), nan, dtype=dtype, device=DEV) for n in (M, N))
        x, w = xb[1:M + 1, 1:K + 1], wb[1:N + 1, 3:K + 3]
        x.copy_(torch.randn((M, K), generator=g, device=DEV))
        w.copy_(torch.randn((N, K), generator=g, device=DEV) * K ** -0.5)
        assert_close(dvdq.linear(x, w), *linear64(x, w, device=DEV), f"K = {K}")


def test_every_length_of_8_bit_rows():
    g = torch.Generator(device=DEV).manual_seed(2)
    M, N = 40, 72
    xs, ws = torch.rand((M,), generator=g, device=DEV) / 50, torch.rand((N,), generator=g, device=DEV) / 50
    for K in (*range(1, 300), 511, 513, 1025):
        xb, wb = (torch.full((n + 2, K + 5), 127, dtype=torch.int8, device=DEV) for n in (M, N))
        x, w = xb[1:M + 1, 1:K + 1], wb[1:N + 1, 3:K + 3]
        x.random_(-127, 128, generator=g)
        w.random_(-127, 128, generator=g)
        assert_close(dvdq.linear8(x, xs, w, ws, dtype=torch.float32), *linear8_64(x, xs, w, ws, device=DEV), f"K = {K}")


@pytest.mark.parametrize("M", [40, 64, 128, 129, 256, 300])
def test_ends_of_tiles(M):
    """Tokens and channels that end inside tiles, each with the other whole and not; nothing beside the output is written."""
    g = torch.Generator(device=DEV).manual_seed(M)
    dtype = torch.bfloat16
    for N in (8, 64, 72, 128, 136, 200, 201, 256, 260):
        for K in (131, 136):
            r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)   # noqa: E731
            x, w, bias, gate, residual = r(M, K + 1)[:, 1:], r(N, K), r(N), r(M, N), r(M, N)
            out = torch.full((M + 2, N + 16), 7.0, dtype=dtype, device=DEV)
            y = out[1:M + 1, 8:N + 8]
            dvdq.linear(x, w, bias, dvdq.ACT_GELU, gate, residual, y=y)
            assert_close(y, *linear64(x, w, bias, dvdq.ACT_GELU, gate, residual, device=DEV), f"{M} x {N} x {K}")
            y.fill_(7.0)
            assert bool((out == 7.0).all()), f"{M} x {N} x {K}: wrote beside the output"
