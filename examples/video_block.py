"""A block of a video diffusion transformer and a step of its decoder, with this library's operators where they stand in such a model:

  conditioning   linear           one row per guidance branch -> shifts, scales and gates of the block
  Q, K, V        qlinear (W4A4)   one projection of the modulated tokens
  positions      rope             q and k turned in place, inside the projection's output, by t, h and w of their patch
  attention      plain torch, in 32 bits
  output         qlinear (W4A4)
  feed-forward   linear + linear  kept in 16 bits: GELU in the first one's epilogue, gate and residual in the second one's
  decoder        group_norm       with SiLU, channels last, then a 1 x 1 convolution (linear) added to what went in

python examples/video_block.py [--grid T,H,W] [--width D]     random weights and latents, one block, times per call
"""
import argparse
import os
import sys
import types

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_18663_amd as dvdq   # noqa: E402

HAD = 64            # Hadamard block of the quantized layers
DT = torch.bfloat16


def make_weights(D, heads, C, seed=0, device="cuda"):
    """Random weights of one block of width D and one decoder step of C channels."""
    g = torch.Generator(device=device).manual_seed(seed)

    def randn(*shape, scale=1.0):
        return (scale * torch.randn(shape, generator=g, device=device)).to(DT)

    def quantized(n, k):   # (a model's come from its calibration: dvdq.bgr_quantize)
        codes = torch.randint(-7, 8, (n, k), generator=g, device=device, dtype=torch.int32) & 15
        packed = (codes[:, 0::2] | codes[:, 1::2] << 4).to(torch.uint8).contiguous()
        return {"w": packed, "w_scale": torch.full((n,), k ** -0.5 / 4, device=device), "bias": randn(n, scale=0.1)}

    return {
        "heads": heads,
        "mod_w": randn(6 * D, D, scale=D ** -0.5), "mod_b": randn(6 * D, scale=0.1),
        "qkv": quantized(3 * D, D), "out": quantized(D, D),
        "up_w": randn(4 * D, D, scale=D ** -0.5), "up_b": randn(4 * D, scale=0.1),
        "down_w": randn(D, 4 * D, scale=(4 * D) ** -0.5), "down_b": randn(D, scale=0.1),
        "norm_w": 1 + randn(C, scale=0.1), "norm_b": randn(C, scale=0.1),
        "conv_w": randn(C, C, scale=C ** -0.5), "conv_b": randn(C, scale=0.1),
    }


def make_positions(grid, head_dim, device="cuda"):
    """(positions int32 [tokens, 3], rotated elements per axis, table): made once per resolution."""
    t, h, w = grid
    i = torch.arange(t * h * w, device=device)
    pos = torch.stack([i // (h * w), i // w % h, i % w], -1).to(torch.int32).contiguous()
    hw = head_dim // 3 // 2 * 2
    sections = (head_dim - 2 * hw, hw, hw)
    freq, magnitude = dvdq.rope_frequencies(sections)
    return pos, sections, dvdq.rope_table(max(grid), freq, magnitude, device=device)


def modulated(x, shift, scale):
    x = torch.nn.functional.layer_norm(x.float(), x.shape[-1:])
    return (x * (1 + scale.float()) + shift.float()).to(DT)


def block(x, cond, p, positions, ops=dvdq):
    """x: tokens [T, D], changed in place; cond: [1, D]."""
    pos, sections, table = positions
    T, D = x.shape
    H = p["heads"]
    shift_a, scale_a, gate_a, shift_m, scale_m, gate_m = ops.linear(cond, p["mod_w"], p["mod_b"])[0].chunk(6)
    qkv, _ = dvdq.qlinear(modulated(x, shift_a, scale_a), p["qkv"]["w"], p["qkv"]["w_scale"], HAD, 4, bias=p["qkv"]["bias"])
    q, k, v = qkv.view(T, 3, H, D // H).unbind(1)
    q, k = ops.rope(q, k, table, pos, sections, interleaved=True, q_out=q, k_out=k)
    q, k, v = (t.transpose(0, 1).float().contiguous() for t in (q, k, v))
    a = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) * (D // H) ** -0.5, -1)
    a = torch.bmm(a, v).transpose(0, 1).reshape(T, D).to(DT)
    o, _ = dvdq.qlinear(a, p["out"]["w"], p["out"]["w_scale"], HAD, 4, bias=p["out"]["bias"])
    x += gate_a * o
    h = ops.linear(modulated(x, shift_m, scale_m), p["up_w"], p["up_b"], act=dvdq.ACT_GELU_TANH)
    return ops.linear(h, p["down_w"], p["down_b"], gate=gate_m.contiguous(), residual=x, y=x)


def decoder_step(z, p, ops=dvdq):
    """z: latents [1, T, H, W, C], channels last; a norm, its activation and a 1 x 1 convolution around a residual."""
    C = z.shape[-1]
    h = ops.group_norm(z, 32, p["norm_w"], p["norm_b"], eps=1e-6, act=dvdq.ACT_SILU)
    rows = z.reshape(-1, C)
    return ops.linear(h.view(-1, C), p["conv_w"], p["conv_b"], residual=rows).view(z.shape)


# The same operators in elementary torch operations, in 32 bits, rounded once (to compare with; see also tests/plain64.py)
def _plain_rope(q, k, table, pos, sections, interleaved, q_out, k_out):
    axis = torch.cat([torch.full((r // 2,), a, device=q.device) for a, r in enumerate(sections)])
    cs = table[pos.long()[:, axis], torch.arange(axis.numel(), device=q.device)][:, None]
    for x, out in ((q, q_out), (k, k_out)):
        f = x.float()
        a, b = f[..., 0::2], f[..., 1::2]
        out.copy_(torch.stack([a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]], -1).flatten(-2))
    return q_out, k_out


def _plain_linear(x, w, bias, act=dvdq.ACT_NONE, gate=None, residual=None, y=None):
    z = x.float() @ w.float().t() + bias.float()
    if act == dvdq.ACT_GELU_TANH:
        z = torch.nn.functional.gelu(z, approximate="tanh")
    if gate is not None:
        z = z * gate.float()
    if residual is not None:
        z = z + residual.float()
    return z.to(x.dtype) if y is None else y.copy_(z)


def _plain_group_norm(x, groups, w, b, eps, act):
    f = x.float().reshape(x.shape[0], -1, groups, x.shape[-1] // groups)
    d = f - f.mean((1, 3), keepdim=True)
    z = (d * torch.rsqrt((d * d).mean((1, 3), keepdim=True) + eps)).reshape(x.shape) * w.float() + b.float()
    return (z * torch.sigmoid(z)).to(x.dtype)


PLAIN = types.SimpleNamespace(rope=_plain_rope, linear=_plain_linear, group_norm=_plain_group_norm)


def run(grid, D, heads, C, ops=dvdq, seed=1):
    """(tokens after one block, latents after one decoder step)"""
    p = make_weights(D, heads, C)
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = grid[0] * grid[1] * grid[2]
    x = torch.randn((T, D), generator=g, device="cuda").to(DT)
    cond = torch.randn((1, D), generator=g, device="cuda").to(DT)
    z = torch.randn((1, grid[0], grid[1], grid[2], C), generator=g, device="cuda").to(DT)
    positions = make_positions(grid, D // heads)
    return block(x, cond, p, positions, ops), decoder_step(z, p, ops)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--grid", default="3,30,52")
    ap.add_argument("--width", type=int, default=1536)
    a = ap.parse_args()
    grid, D = tuple(int(v) for v in a.grid.split(",")), a.width
    heads, C = D // 128, 512
    mine, plain = run(grid, D, heads, C), run(grid, D, heads, C, PLAIN)
    for name, u, v in zip(("tokens", "latents"), mine, plain):
        print(f"{name}: {tuple(u.shape)}, against the plain operators {float((u.float() - v.float()).norm() / v.float().norm()):.2e}")
    times = {}

    def timed(name):
        def call(*args, **kw):
            ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            ev[0].record()
            out = getattr(dvdq, name)(*args, **kw)
            ev[1].record()
            times.setdefault(name, []).append(ev)
            return out
        return call
    run(grid, D, heads, C, types.SimpleNamespace(**{f: timed(f) for f in ("rope", "linear", "group_norm")}))
    torch.cuda.synchronize()
    for name, evs in times.items():
        print(name, " ".join(f"{a.elapsed_time(b) * 1e3:.1f}" for a, b in evs), "us")


if __name__ == "__main__":
    main()
