"""Host side of the operators around the quantized layer: refusals before anything touches a GPU, rotary frequencies.  CPU only."""
import ctypes as C
import math

import pytest

import paper_2505_18663_amd as dvdq

FAKE = 0x1000        # never dereferenced: every call below fails validation, or has nothing to do
ODD = 0x1001


def heads(p=FAKE, out=None, n=4, st=(512, 64, 16), ost=None):
    return dvdq._RopeHeads(p, p + (1 << 20) if out is None else out, n, (C.c_int64 * 3)(*st), (C.c_int64 * 3)(*(ost or st)))


def rope(q=None, k=None, B=2, T=8, D=16, table=FAKE, n_pos=10, R=16, pos=FAKE, pb=0, axes=1, sections=None, flags=0, dtype=0):
    sec = None if sections is None else (C.c_int32 * len(sections))(*sections)
    return dvdq.lib().dvdq_rope(C.byref(q or heads()), None if k is None else C.byref(k), B, T, D, table, n_pos, R, pos, pb, axes, sec, flags,
                                dtype, None)


def test_rope_argument_errors():
    assert dvdq.lib().dvdq_rope(None, None, 1, 1, 16, FAKE, 10, 16, FAKE, 0, 1, None, 0, 0, None) == 1
    assert rope(q=heads(p=None, out=FAKE)) == 1 and rope(table=None) == 1 and rope(pos=None) == 1 and rope(axes=2) == 1
    assert rope(B=-1) == 2 and rope(T=-1) == 2 and rope(D=0) == 2 and rope(n_pos=0) == 2
    assert rope(R=15) == 2 and rope(R=18) == 2 and rope(R=0) == 2 and rope(axes=0) == 2 and rope(pb=7) == 2
    assert rope(axes=2, sections=(8, 6)) == 2 and rope(axes=2, sections=(9, 7)) == 2 and rope(axes=2, sections=(-2, 18)) == 2
    assert rope(q=heads(n=0)) == 2 and rope(k=heads(n=0)) == 2
    assert rope(D=1026) == 3 and rope(axes=5, sections=(4, 4, 4, 2, 2)) == 3 and rope(flags=4) == 3 and rope(dtype=3) == 3
    assert rope(T=1 << 24) == 3 and rope(B=1 << 12, T=1 << 12) == 3
    assert rope(q=heads(st=(512, 64, 16), ost=(0, 64, 16))) == 3                       # all batches to one place
    assert rope(q=heads(out=FAKE, ost=(512, 128, 16))) == 3                            # in place with other strides
    assert rope(q=heads(p=ODD)) == 5 and rope(table=0x1008) == 5 and rope(pos=0x1002) == 5 and rope(q=heads(p=0x1002, out=0x9002), dtype=2) == 5
    assert rope(B=0) == 0 and rope(T=0) == 0                                           # nothing to do


def test_rope_table_argument_errors():
    f = dvdq.lib().dvdq_rope_table
    assert f(None, 4, 4, 1.0, FAKE, None) == 1 and f(FAKE, 4, 4, 1.0, None, None) == 1
    assert f(FAKE, 0, 4, 1.0, FAKE, None) == 2 and f(FAKE, 4, 0, 1.0, FAKE, None) == 2
    assert f(FAKE, 4, 513, 1.0, FAKE, None) == 3 and f(FAKE, 1 << 31, 4, 1.0, FAKE, None) == 3
    assert f(0x1008, 4, 4, 1.0, FAKE, None) == 5


def linear(x=FAKE, ldx=64, w=FAKE, ldw=64, bias=None, act=0, gate=None, gr=0, ldg=0, res=None, ldr=0, M=4, N=32, K=64, dtype=0, y=FAKE + 65536,
           ldy=32, ws=FAKE, nws=1 << 40):
    return dvdq.lib().dvdq_linear(x, ldx, w, ldw, bias, act, gate, gr, ldg, res, ldr, M, N, K, dtype, y, ldy, ws, nws, None)


def test_linear_argument_errors():
    assert linear(x=None) == 1 and linear(w=None) == 1 and linear(y=None) == 1
    assert linear(M=-1) == 2 and linear(N=0) == 2 and linear(K=0) == 2
    assert linear(ldx=63) == 2 and linear(ldw=63) == 2 and linear(ldy=31) == 2 and linear(res=FAKE, ldr=31) == 2
    assert linear(gate=FAKE, gr=3, ldg=32) == 2 and linear(gate=FAKE, gr=0, ldg=32) == 2 and linear(gate=FAKE, gr=2, ldg=31) == 2
    assert linear(act=4) == 3 and linear(act=-1) == 3 and linear(dtype=2) == 3 and linear(dtype=-1) == 3
    assert linear(M=1 << 24) == 3 and linear(N=1 << 23, ldy=1 << 23) == 3 and linear(K=1 << 23, ldx=1 << 23, ldw=1 << 23) == 3
    assert linear(res=FAKE + 65536, ldr=40) == 3                                       # y is the residual, in other places
    for name in ("x", "w", "bias", "res", "y"):
        assert linear(**{name: ODD, "ldr": 32}) == 5, name
    assert linear(gate=ODD, gr=1, ldg=32) == 5
    assert linear(M=0) == 0
    assert dvdq.linear_workspace_bytes(0, 4, 4) == 0 and dvdq.linear_workspace_bytes(4, 4, -1) == 0
    M, N, K = 300, 512, 4096
    need = dvdq.linear_workspace_bytes(M, N, K)
    if need:
        assert linear(M=M, N=N, K=K, ldx=K, ldw=K, ldy=N, nws=need - 1) == 4
        assert linear(M=M, N=N, K=K, ldx=K, ldw=K, ldy=N, ws=FAKE + 8) == 5
        assert linear(M=M, N=N, K=K, ldx=K, ldw=K, ldy=N, ws=None) == 1


def test_linear_choice_is_the_same_every_time_and_sizes_the_workspace():
    sizes = {0: (256, 256), 1: (256, 128), 2: (128, 128), 3: (128, 64), 4: (64, 64)}
    for M, N, K in [(1, 64, 8), (16, 512, 4096), (17, 384, 1000), (512, 5120, 4096), (32760, 8960, 1536), (700, 300, 33), (3000, 500, 1157)]:
        need, most = dvdq.linear_workspace_bytes(M, N, K), 0
        for any_ in (False, True):
            c = dvdq.bench_linear_choice(M, N, K, any_)
            assert c == dvdq.bench_linear_choice(M, N, K, any_)
            if c < 0:
                continue
            (bn, bm), parts = sizes[c & 15], (c >> 4) & 255
            tiles = -(-N // bn) * -(-M // bm)
            pad = -(-((M + N) * (-(-K // 64) * 64) * 2) // 256) * 256 if c & 4096 else 0
            most = max(most, pad + (parts * tiles * bn * bm * 4 if parts > 1 else 0))
        assert need == most, (M, N, K)
    assert dvdq.bench_linear_choice(0, 1, 1) == -2


def gn(x=FAKE, B=2, S=10, C=32, xb=320, xr=32, groups=4, w=None, b=None, eps=1e-5, act=0, dtype=0, y=FAKE + 65536, yb=320, yr=32, ws=FAKE, nws=1 << 40):
    return dvdq.lib().dvdq_group_norm(x, B, S, C, xb, xr, groups, w, b, eps, act, dtype, y, yb, yr, ws, nws, None)


def test_group_norm_argument_errors():
    assert gn(x=None) == 1 and gn(y=None) == 1 and gn(ws=None) == 1
    assert gn(B=-1) == 2 and gn(S=-1) == 2 and gn(C=0) == 2 and gn(groups=0) == 2 and gn(groups=5) == 2 and gn(eps=-1.0) == 2
    assert gn(eps=math.nan) == 2 and gn(xr=31) == 2 and gn(yr=31) == 2
    assert gn(C=4100, xr=4100, yr=4100) == 3 and gn(B=65536) == 3 and gn(act=2) == 3 and gn(dtype=3) == 3
    assert gn(yb=0) == 3 and gn(y=FAKE, yr=40) == 3 and gn(y=FAKE, yb=640) == 3
    assert gn(x=ODD) == 5 and gn(w=ODD) == 5 and gn(b=ODD) == 5 and gn(y=ODD) == 5 and gn(ws=0x1008) == 5 and gn(x=0x1002, dtype=2) == 5
    assert gn(nws=dvdq.group_norm_workspace_bytes(2, 10, 32, 4) - 1) == 4
    assert gn(B=0) == 0 and gn(S=0) == 0
    assert dvdq.group_norm_workspace_bytes(1, 1, 32, 5) == 0 and dvdq.group_norm_workspace_bytes(0, 1, 32, 4) == 0


def test_binding_refuses_cpu_tensors():
    import torch
    t = torch.zeros((2, 3, 8))
    for call in (lambda: dvdq.rope(t, None, t, t), lambda: dvdq.linear(t[0], t[0]), lambda: dvdq.group_norm(t, 2)):
        with pytest.raises(TypeError):
            call()


def test_rope_frequencies():
    f, m = dvdq.rope_frequencies(8)
    assert m == 1.0 and f == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-14)
    f, _ = dvdq.rope_frequencies((4, 2), base=100.0)
    assert f == pytest.approx([1.0, 0.1, 1.0], rel=1e-14)
    f, m = dvdq.rope_frequencies(8, scaling="linear", factor=4.0)
    assert m == 1.0 and f == pytest.approx([0.25, 0.025, 0.0025, 0.00025], rel=1e-14)
    # the slowest pair stretched by the factor, the fastest not at all
    f, _ = dvdq.rope_frequencies(64, scaling="ntk", factor=8.0)
    plain, _ = dvdq.rope_frequencies(64)
    assert f[0] == 1.0 and f[-1] == pytest.approx(plain[-1] / 8, rel=1e-12)
    # pairs of many turns stay, pairs of few are divided, the rest lies in between and in order
    f, m = dvdq.rope_frequencies(128, scaling="yarn", factor=16.0, original_length=4096)
    plain, _ = dvdq.rope_frequencies(128)
    assert m == pytest.approx(1 + 0.1 * math.log(16.0))
    ratio = [a / b for a, b in zip(f, plain)]
    turns = [4096 * p / (2 * math.pi) for p in plain]
    assert all(r == 1.0 for r, t in zip(ratio, turns) if t > 40) and all(r == pytest.approx(1 / 16) for r, t in zip(ratio, turns) if t < 0.8)
    assert all(a >= b for a, b in zip(ratio, ratio[1:])) and any(1 / 16 < r < 1 for r in ratio)
    assert dvdq.rope_frequencies(128, scaling="yarn", factor=1.0, original_length=4096)[0] == pytest.approx(plain)
    for bad in (dict(rot_dim=7), dict(rot_dim=()), dict(rot_dim=8, scaling="other"), dict(rot_dim=8, base=1.0), dict(rot_dim=8, factor=0.5),
                dict(rot_dim=8, scaling="yarn", factor=2.0)):
        with pytest.raises(ValueError):
            dvdq.rope_frequencies(**bad)
