"""Host side of the norms and layers in 8 bits: refusals before anything touches a GPU.  CPU only."""
import pytest
import torch

import paper_2505_18663_amd as dvdq

X, R, H, W, Y, S = (0x100000 * i for i in range(1, 7))   # never dereferenced: every call below fails validation, or has nothing to do


def norm(x=X, B=2, S=3, C=16, xs=(48, 16), r=None, rs=(48, 16), h=None, hs=(48, 16), w=W, eps=1e-6, dtype=0, y=Y, ys=(48, 16)):
    return dvdq.lib().dvdq_rms_norm(x, B, S, C, *xs, r, *rs, h, *hs, w, eps, dtype, y, *ys, None)


def norm_quant(x=X, B=2, S=3, C=16, xs=(48, 16), r=None, rs=(48, 16), h=None, hs=(48, 16), w=W, eps=1e-6, dtype=0, c=Y, cs=(48, 16), s=S, sums=None):
    return dvdq.lib().dvdq_rms_norm_quant(x, B, S, C, *xs, r, *rs, h, *hs, w, eps, dtype, c, *cs, s, sums, None)


def quant(x=X, ldx=16, up=None, ldu=0, act=0, M=4, C=16, dtype=0, c=Y, ldc=16, s=S, sums=None):
    return dvdq.lib().dvdq_quant8(x, ldx, up, ldu, act, M, C, dtype, c, ldc, s, sums, None)


def linear(x=X, ldx=64, xs=S, w=W, ldw=64, ws=S, bias=None, act=0, gate=None, gr=0, ldg=0, res=None, ldr=0, M=4, N=32, K=64, dtype=0, y=Y, ldy=32, space=H,
           n=1 << 40):
    return dvdq.lib().dvdq_linear8(x, ldx, xs, w, ldw, ws, bias, act, gate, gr, ldg, res, ldr, M, N, K, dtype, y, ldy, space, n, None)


@pytest.mark.parametrize("f,out", [(norm, "y"), (norm_quant, "c")])
def test_norm_argument_errors(f, out):
    assert f(x=None) == 1 and f(**{out: None}) == 1 and f(r=R) == 1
    assert f(B=-1) == 2 and f(S=-1) == 2 and f(C=0) == 2 and f(eps=-1.0) == 2 and f(eps=float("nan")) == 2 and f(h=H) == 2
    assert f(dtype=3) == 3 and f(dtype=-1) == 3 and f(C=(1 << 22) + 1) == 3 and f(B=1 << 16, S=1 << 15) == 3 and f(B=1 << 32) == 3
    assert f(**{out + "s": (0, 16)}) == 3 and f(**{out + "s": (48, 0)}) == 3            # rows on one another
    assert f(r=R, h=H, hs=(0, 16)) == 3 and f(r=R, h=X, hs=(96, 16)) == 3 and f(r=R, h=R, hs=(48, 32)) == 3
    assert f(r=R, h=Y) == 3 and f(w=Y) == 3 and f(r=R, h=W) == 3                        # outputs over one another, or over what every row needs
    assert f(x=X + 1) == 5 and f(w=W + 1) == 5 and f(r=R + 1, h=H) == 5 and f(r=R, h=H + 1) == 5 and f(x=X + 2, dtype=2) == 5
    assert f(B=0) == 0 and f(S=0) == 0 and f(x=None, B=0) == 0


def test_norm_in_place_only_with_its_own_strides():
    assert norm(y=X, ys=(96, 16)) == 3 and norm(r=R, h=H, y=R, ys=(48, 24)) == 3
    assert norm_quant(c=X) == 3 and norm_quant(r=R, h=H, c=R) == 3 and norm_quant(s=None) == 1
    assert norm(y=Y + 1) == 5 and norm_quant(s=S + 2) == 5 and norm_quant(sums=S + 1) == 5


def test_quant_argument_errors():
    assert quant(x=None) == 1 and quant(c=None) == 1 and quant(s=None) == 1
    assert quant(M=-1) == 2 and quant(C=0) == 2 and quant(ldc=15) == 2
    assert quant(act=4) == 3 and quant(act=-1) == 3 and quant(dtype=3) == 3 and quant(C=(1 << 22) + 1, ldc=1 << 23) == 3 and quant(M=1 << 31) == 3
    assert quant(c=X) == 3 and quant(up=R, ldu=16, c=R) == 3
    assert quant(x=X + 1) == 5 and quant(up=R + 1) == 5 and quant(s=S + 1) == 5 and quant(sums=S + 2) == 5 and quant(x=X + 2, dtype=2) == 5
    assert quant(M=0) == 0 and quant(x=None, M=0) == 0


def test_linear8_argument_errors():
    for name in ("x", "xs", "w", "ws", "y"):
        assert linear(**{name: None}) == 1, name
    assert linear(M=-1) == 2 and linear(N=0) == 2 and linear(K=0) == 2
    assert linear(ldx=63) == 2 and linear(ldw=63) == 2 and linear(ldy=31) == 2 and linear(res=R, ldr=31) == 2
    assert linear(gate=R, gr=3, ldg=32) == 2 and linear(gate=R, gr=0, ldg=32) == 2 and linear(gate=R, gr=2, ldg=31) == 2
    assert linear(act=4) == 3 and linear(act=-1) == 3 and linear(dtype=3) == 3 and linear(dtype=-1) == 3
    assert linear(M=1 << 24) == 3 and linear(N=1 << 23, ldy=1 << 23) == 3 and linear(K=131072, ldx=131072, ldw=131072) == 3
    assert linear(res=Y, ldr=40) == 3 and linear(y=X) == 3 and linear(y=W) == 3 and linear(y=S) == 3 and linear(bias=Y) == 3
    assert linear(gate=Y, gr=2, ldg=32) == 3 and linear(ldy=1 << 27) == 3
    for dtype, odd in ((0, 1), (1, 1), (2, 2)):
        for name in ("bias", "res", "y"):
            assert linear(**{name: H + odd, "ldr": 32, "dtype": dtype}) == 5, name
        assert linear(gate=H + odd, gr=1, ldg=32, dtype=dtype) == 5
    assert linear(xs=S + 2) == 5 and linear(ws=S + 1) == 5
    assert linear(M=0) == 0 and linear(M=0, x=None) == 0
    assert dvdq.linear8_workspace_bytes(0, 4, 4) == 0 and dvdq.linear8_workspace_bytes(4, 4, 131072) == 0
    M, N, K = 300, 512, 4001
    need = dvdq.linear8_workspace_bytes(M, N, K)
    if need:
        size = dict(M=M, N=N, K=K, ldx=K, ldw=K, ldy=N)
        assert linear(**size, n=need - 1) == 4 and linear(**size, space=H + 8) == 5 and linear(**size, space=None) == 1


def test_the_binding_refuses_what_is_not_on_a_gpu():
    x, c, s = torch.zeros(4, 16), torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    for f in (lambda: dvdq.rms_norm(x), lambda: dvdq.rms_norm_quant(x), lambda: dvdq.quant8(x), lambda: dvdq.linear8(c, s, c, s)):
        with pytest.raises(TypeError, match="expected a CUDA/HIP tensor"):
            f()


def test_the_sizes_that_stand_for_each_shape_of_tile_take_it():
    from test_gpu_linear8 import WAYS
    for (shape, parts), (M, N, K) in WAYS.items():
        assert dvdq.bench_linear8_choice(M, N, K) == shape + 16 * parts, (M, N, K)
        bn, bm = {0: (256, 256), 1: (256, 128), 2: (128, 128), 3: (128, 64), 4: (64, 64)}[shape]
        need = -(-M // bm) * -(-N // bn) * parts * bm * bn * 4 if parts > 1 else 0
        assert dvdq.linear8_workspace_bytes(M, N, K) >= need
    assert {shape for shape, _ in WAYS} == set(range(5))
    for M, N, K in ((8, 5120, 13824), (16, 5120, 5120)):    # few tokens: straight from the weights
        assert dvdq.bench_linear8_choice(M, N, K) == dvdq.bench_linear8_choice(M, N, K, True) == -1 and dvdq.linear8_workspace_bytes(M, N, K) == 0


def test_the_workspace_holds_whatever_way_the_addresses_ask_for():
    """Rows that are no whole pieces are copied, or read through registers, in parts of K: the size is for the larger."""
    from test_gpu_linear8 import ROWS
    ways = set()
    for M, N, K in (*ROWS, (40, 48, 1168), (33, 65, 1000)):
        for any_ in (False, True):
            c = dvdq.bench_linear8_choice(M, N, K, any_)
            assert c == dvdq.bench_linear8_choice(M, N, K, any_)
            ways.add((c % 16, min(c // 16 % 256, 2), c >> 12))
            shape, parts, pad = c % 16, c // 16 % 256, bool(c & 4096)
            bn, bm = {0: (256, 256), 1: (256, 128), 2: (128, 128), 3: (128, 64), 4: (64, 64)}[shape]
            need = -(-M // bm) * -(-N // bn) * parts * bm * bn * 4 if parts > 1 else 0
            need += (M + N) * (-(-K // 128) * 128) if pad else 0
            assert dvdq.linear8_workspace_bytes(M, N, K) >= need, (M, N, K)
    assert {(2, 1, 2), (4, 1, 2), (4, 2, 2)} <= ways and any(w[2] == 1 for w in ways)    # through registers as both tiles, whole and in parts; copied
