"""Plain 64-bit forms of the operators around the quantized layer, on the CPU, and the bounds their outputs are judged by.

A result may differ from the 64-bit value by the one rounding to its type plus what fp32 arithmetic may lose on the way:
  rounding       u |ref|, u = 2^-8 (bf16: 8 bits of significand), 2^-11 (fp16: 11; 2^-25 absolute below its normal range), 2^-24 (fp32), with 2 % to spare
  products       2^-24 per operation on the magnitudes that go in
  long sums      4 sqrt(K) 2^-24 sum |terms| (rounding errors of a sum of K terms add up like a random walk; four standard deviations)
  activations    2^-19 of the result and of its argument's share of it (exp2, rcp and erf are good to a few units of 2^-24)
"""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
F32 = 2.0 ** -24


def assert_close(got, ref, slack, what):
    """|got - ref| <= one rounding + slack, elementwise; NaN where, and only where, the reference is NaN."""
    u, tiny = UNIT[got.dtype], TINY[got.dtype]
    got, ref = got.detach().to(ref.device).double(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    nan = ref.isnan()
    assert torch.equal(got.isnan(), nan), f"{what}: NaN in other places"
    inf = ref.isinf()
    assert torch.equal(got[inf & ~nan], ref[inf & ~nan]), f"{what}: infinities differ"
    ok = ~(nan | inf)
    slack = slack if isinstance(slack, torch.Tensor) else torch.full_like(ref, slack)
    over = ((got - ref).abs() - (1.02 * u * ref.abs() + tiny + slack))[ok]
    if over.numel():
        assert over.max() <= 0, f"{what}: {int((over > 0).sum())} of {over.numel()} off, worst by {float(over.max()):.3g}"


def act64(z, act):
    if act == 1:
        return z / (1 + torch.exp(-z))
    if act == 2:
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == 3:
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    return z


def rope64(x, table, positions, sections, interleaved, inverse=False):
    """x [B, T, H, D]; positions [B, T, axes].  Returns (reference, sum of magnitudes that went into it)."""
    x, table = x.cpu().double(), table.cpu().double()
    positions = positions.cpu().long()
    half = table.shape[1]
    axis = torch.cat([torch.full((r // 2,), a) for a, r in enumerate(sections)])
    p = positions[..., axis]                                     # [B, T, half]
    j = torch.arange(half).expand_as(p)
    cs = table[p.clamp(0, table.shape[0] - 1), j]
    cs = torch.where((p >= table.shape[0])[..., None], torch.full_like(cs, float("nan")), cs)[:, :, None]
    c, s = cs[..., 0], cs[..., 1] * (-1 if inverse else 1)
    ia = torch.arange(half) * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else half)
    a, b = x[..., ia], x[..., ib]
    keep = (p < 0)[:, :, None]
    out, mag = x.clone(), torch.zeros_like(x)
    out[..., ia] = torch.where(keep, a, a * c - b * s)
    out[..., ib] = torch.where(keep, b, a * s + b * c)
    mag[..., ia] = torch.where(keep, torch.zeros_like(a), (a * c).abs() + (b * s).abs())
    mag[..., ib] = torch.where(keep, torch.zeros_like(a), (a * s).abs() + (b * c).abs())
    return out, mag.nan_to_num(0.0, 0.0, 0.0)


def linear64(x, w, bias=None, act=0, gate=None, residual=None, device="cpu"):
    """Returns (reference, slack)."""
    f = lambda t: None if t is None else t.to(device).double()   # noqa: E731
    x, w, bias, gate, residual = map(f, (x, w, bias, gate, residual))
    M, K = x.shape
    z, mag = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, mag = z + bias, mag + bias.abs()
    err = (4 * math.sqrt(K) + 2) * F32 * mag
    y = act64(z, act)
    if act:
        err = 1.2 * err + 2.0 ** -19 * (y.abs() + z.abs())       # (the slope of each of the activations is at most 1.13)
    if gate is not None:
        g = gate.reshape(-1, gate.shape[-1]).repeat_interleave(M // (gate.numel() // gate.shape[-1]), 0)
        y, err = y * g, err * g.abs() + 2 * F32 * (y * g).abs()
    if residual is not None:
        y = y + residual
        err = err + 2 * F32 * (y.abs() + residual.abs())
    return y, err


def group_norm64(x, groups, weight=None, bias=None, eps=1e-5, act=0):
    """x [B, S, C].  Returns (reference, slack)."""
    f = lambda t: None if t is None else t.cpu().double()   # noqa: E731
    x, weight, bias = map(f, (x, weight, bias))
    B, S, C = x.shape
    v = x.view(B, S, groups, C // groups)
    mean = v.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(((v - mean) ** 2).mean((1, 3), keepdim=True) + eps)
    z = ((v - mean) * rstd).reshape(B, S, C)
    # mean and variance are good to a few units of 2^-24 (of the mean's size, and relative); the values that go in are exact
    err = (24 * F32 * ((v.abs() + mean.abs()) * rstd + 1)).reshape(B, S, C)
    if weight is not None:
        z, err = z * weight, err * weight.abs()
    if bias is not None:
        z = z + bias
        err = err + 2 * F32 * (z.abs() + bias.abs())
    y = act64(z, act)
    if act:
        err = 1.2 * err + 2.0 ** -19 * (y.abs() + z.abs())
    return y, err
