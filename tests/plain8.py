"""Plain 64-bit forms of the norms and layers in 8 bits, and the bounds their outputs are judged by (assert_close and act64 of plain64).

  codes    equal: they are those of the real numbers, ties to the even one.  An activation's value is itself rounded, in 64 bits, so where 127 z / max|z|
           lies within 2^-40 of a border between two codes either of them will do
  scales   the norm's statistic is a sum of C squares in fp32: 2 sqrt(C) 2^-24 for its root (four standard deviations of rounding errors that add up like a
           random walk, halved by the root), and 8 operations
  product  the sum is exact; its conversion, the two scales and the bias take an operation each
"""
import torch

from plain64 import F32, act64


def codes64(z, loose=False):
    """(codes, max|z| [..., 1], where either of two codes will do) of z in 64 bits."""
    a = z.abs()
    top = a.amax(-1, keepdim=True)
    safe = torch.where(top > 0, top, torch.ones_like(top))
    low = torch.floor(127 * a / safe).clamp(0, 126)
    over = 254 * a - (2 * low + 1) * top                       # the distance from the border above `low`
    q = torch.where((over > 0) | ((over == 0) & (low % 2 == 1)), low + 1, low)
    q = torch.where(top > 0, q * torch.sign(z), torch.zeros_like(z))
    return q, top, (over.abs() <= 2.0 ** -40 * 254 * top) if loose else torch.zeros_like(z, dtype=torch.bool)


def norm64(x, weight=None, residual=None, eps=1e-6):
    """(y, root [..., 1], h, relative error of what is divided by the root)"""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h = h.cpu()
    f = h.double()
    root = torch.sqrt((f * f).mean(-1, keepdim=True) + eps)
    z = f if weight is None else f * weight.cpu().double()
    return z, root, h, (2 * x.size(-1) ** 0.5 + 8) * F32


def check_codes(codes, scale, z, factor, err, what, loose=False, rowsum=None):
    q, top, either = codes64(z, loose)
    got = codes.cpu().double()
    off = (got != q) & ~(either & ((got - q).abs() == 1))
    assert not off.any(), f"{what}: {int(off.sum())} of {off.numel()} codes differ, the first at {tuple(off.nonzero()[0].tolist())}"
    want = (factor * top / 127)[..., 0]
    assert scale.shape == want.shape, what
    over = (scale.cpu().double() - want).abs() - (err + 3 * F32) * want - 2.0 ** -149
    assert not (over > 0).any(), f"{what}: scales off by {float(over.max()):.3g}"
    if rowsum is not None:
        assert torch.equal(rowsum.cpu().long(), codes.cpu().long().sum(-1)), f"{what}: sums of codes"


def linear8_64(codes, x_scale, w, w_scale, bias=None, act=0, gate=None, residual=None, device="cpu"):
    """(reference, slack)"""
    f = lambda t: None if t is None else t.to(device).double()   # noqa: E731
    codes, x_scale, w, w_scale, bias, gate, residual = map(f, (codes, x_scale, w, w_scale, bias, gate, residual))
    M = codes.shape[0]
    z = (codes @ w.t()) * x_scale[:, None] * w_scale          # (below 2^53: exact before the scales)
    mag = z.abs()
    if bias is not None:
        z, mag = z + bias, mag + bias.abs()
    err = 4 * F32 * mag
    y = act64(z, act)
    if act:
        err = 1.2 * err + 2.0 ** -19 * (y.abs() + z.abs())    # (the slope of each of the activations is at most 1.13)
    if gate is not None:
        g = gate.reshape(-1, gate.shape[-1]).repeat_interleave(M // (gate.numel() // gate.shape[-1]), 0)
        y, err = y * g, err * g.abs() + 2 * F32 * (y * g).abs()
    if residual is not None:
        y = y + residual
        err = err + 2 * F32 * (y.abs() + residual.abs())
    return y, err
