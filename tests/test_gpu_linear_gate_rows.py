"""Gates whose rows belong to few tokens, or to one, against the formula in 64 bits: tokens of a tile then have rows of their own."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import assert_close, linear64
from plain8 import linear8_64
from test_gpu_linear import WAYS as WAYS16
from test_gpu_linear8 import WAYS as WAYS8, operands

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gates(M):
    """Rows of the gate: one a token, and the divisors of M next to these (rows end anywhere inside a wave's 16 to 128 tokens)."""
    divisors = [d for d in range(2, M) if M % d == 0]
    return {M, *(min(divisors, key=lambda d: abs(M / d - tokens)) for tokens in (3, 17, 100) if divisors)}


def tensor(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


@pytest.mark.parametrize("way", WAYS16)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_way(way, dtype):
    M, N, K = way[:3]
    g = torch.Generator(device=DEV).manual_seed(M)
    x, w, bias, res = tensor(g, M, K, dtype=dtype), tensor(g, N, K, dtype=dtype, scale=K ** -0.5), tensor(g, N, dtype=dtype), tensor(g, M, N, dtype=dtype)
    for i, G in enumerate(sorted(gates(M))):
        gate = tensor(g, G, N, dtype=dtype)
        residual = res if i % 2 else None
        got = dvdq.linear(x, w, bias, i % 4, gate, residual)
        assert_close(got, *linear64(x, w, bias, i % 4, gate, residual, device=DEV), f"{way} {G} rows")
    # a row a token (the last): with a residual, over it, and over the gate
    want = dvdq.linear(x, w, bias, 1, gate, res)
    assert_close(want, *linear64(x, w, bias, 1, gate, res, device=DEV), f"{way} residual")
    for over in (res, gate):
        y = over.clone()
        dvdq.linear(x, w, bias, 1, y if over is gate else gate, y if over is res else res, y=y)
        assert torch.equal(y, want), f"{way} in place"


@pytest.mark.parametrize("way", WAYS8)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_every_way_of_8_bit_products(way, dtype):
    M, N, K = WAYS8[way]
    g = torch.Generator(device=DEV).manual_seed(M)
    args = operands(g, M, N, K)
    res = tensor(g, M, N, dtype=dtype)
    for i, G in enumerate(sorted(gates(M))):
        gate = tensor(g, G, N, dtype=dtype)
        residual = None if i % 2 else res
        got = dvdq.linear8(*args, act=i % 4, gate=gate, residual=residual, dtype=dtype)
        assert_close(got, *linear8_64(*args, act=i % 4, gate=gate, residual=residual, device=DEV), f"{way} {G} rows")
    want = dvdq.linear8(*args, gate=gate, residual=res, dtype=dtype)
    for over in (res, gate):
        y = over.clone()
        dvdq.linear8(*args, gate=y if over is gate else gate, residual=y if over is res else res, y=y)
        assert torch.equal(y, want), f"{way} in place"


def test_gates_inside_larger_tensors():
    """Rows of the gate of any pitch at any address; what lies beside them is NaN."""
    g = torch.Generator(device=DEV).manual_seed(5)
    M, N, K = 600, 328, 256
    x, w = tensor(g, M, K, dtype=torch.bfloat16), tensor(g, N, K, dtype=torch.bfloat16, scale=K ** -0.5)
    for G in (600, 200, 40, 8):
        around = torch.full((G + 2, N + 13), float("nan"), dtype=torch.bfloat16, device=DEV)
        for offset in (0, 3, 8):
            gate = around[1:G + 1, offset:offset + N]
            gate.copy_(tensor(g, G, N, dtype=torch.bfloat16))
            got = dvdq.linear(x, w, gate=gate)
            assert_close(got, *linear64(x, w, gate=gate.clone(), device=DEV), f"{G} rows, offset {offset}")
            gate.fill_(float("nan"))
