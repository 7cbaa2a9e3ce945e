"""The activations of a product's epilogue over their whole range, the tails included, against their formulas in 64 bits.

A product with a single nonzero term is exact in fp32, so the bound is that of the activation alone: one rounding to the type, and
  (4 |t| + 16) 2^-24 of the result, where the result falls like e^-|t|: the few roundings of t on its way into the exponential count |t|
  times each, the operations behind it (exponential or erfc, sum, reciprocal, product) with a few units
  2^-118 beside it: results that small may come out as zero (the reciprocal's argument has passed 2^126)
"""
import math

import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import F32, act64, assert_close

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def values(dtype):
    z = torch.cat([torch.linspace(-14.0, 14.0, 5000), torch.linspace(-100.0, 100.0, 1500), torch.logspace(-6, 0, 300), -torch.logspace(-6, 0, 300)])
    return z.to(dtype).unique()


# tokens and terms: straight from the weights, through registers, copied rows, tiles, tiles with K in parts
@pytest.mark.parametrize("M,K", [(3, 1), (40, 1), (700, 3), (300, 64), (20, 4096)])
@pytest.mark.parametrize("act", [1, 2, 3])
@pytest.mark.parametrize("dtype", DTYPES)
def test_activation(dtype, act, M, K):
    dt = DTYPES[dtype]
    z = values(dt)
    w = torch.zeros((z.numel(), K), dtype=dt)
    w[:, K // 2] = z
    x = torch.ones((M, K), dtype=dt)
    got = dvdq.linear(x.cuda(), w.cuda(), act=act)
    z = z.double()
    ref = act64(z, act)
    t = {1: z.abs(), 2: 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3).abs(), 3: z * z}[act]
    t = torch.where(z < 0, t, torch.zeros_like(t))                 # (above zero the result does not fall)
    slack = (4 * t + 16) * F32 * ref.abs() + 2.0 ** -118
    assert_close(got, ref.expand(M, -1), slack.expand(M, -1), f"act {act}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", [1, 2, 3])
def test_limits(dtype, act):
    """Towards infinity the activations are the identity; what follows from NaN is NaN."""
    w = torch.tensor([[float("inf")], [float("nan")], [0.0], [-0.0], [6e4]], dtype=DTYPES[dtype], device="cuda")
    y = dvdq.linear(torch.ones((2, 1), dtype=w.dtype, device="cuda"), w, act=act)
    assert bool((y[:, 0] == float("inf")).all()) and bool(y[:, 1].isnan().all()) and not bool(y[:, 2:4].any())
    assert torch.equal(y[:, 4], w[4].expand(2))
