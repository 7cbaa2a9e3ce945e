"""The product of 8-bit codes and weights with its epilogue, against the formula in 64 bits."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import assert_close
from plain8 import linear8_64

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def ints(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)


def tensor(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def operands(g, M, N, K):
    xs = torch.exp(tensor(g, M, scale=0.3)) / 127
    ws = torch.exp(tensor(g, N, scale=0.3)) / 127 / K ** 0.5
    return ints(g, M, K), xs, ints(g, N, K), ws


def check(args, what, device="cpu", **kw):
    M, N = args[0].shape[0], args[2].shape[0]
    ws = dvdq.linear8_workspace_bytes(M, N, args[0].shape[1])
    space = torch.full((ws + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    y = dvdq.linear8(*args, workspace=space[:ws] if ws else None, **kw)
    assert (space[ws:] == 0xA5).all(), f"{what}: wrote past the workspace"
    kw = {k: v for k, v in kw.items() if k in ("bias", "act", "gate", "residual")}
    ref, slack = linear8_64(*args, device=device, **kw)
    assert_close(y, ref, slack, what)
    return y


# few tokens, every shape of tile, parts of K, one more and one less than a tile, and rows of any length
SIZES = [(1, 1, 1), (1, 64, 64), (2, 9216, 1536), (7, 33, 100), (15, 100, 4097), (16, 128, 256), (16, 129, 8000), (17, 16, 128), (17, 130, 129), (33, 65, 1000),
         (64, 64, 4096), (65, 255, 384), (100, 520, 48), (127, 127, 127), (128, 128, 128), (129, 257, 272), (200, 1000, 16), (256, 256, 2048), (300, 77, 5000),
         (511, 640, 1152), (1000, 300, 333), (2100, 1030, 513), (3000, 96, 80), (4096, 4096, 128)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_sizes(size, dtype):
    M, N, K = size
    g = gen(M + N + K)
    args = operands(g, M, N, K)
    big = M * N * K > 1 << 28
    on = DEV if big else "cpu"
    check(args, f"{size}", on, dtype=dtype)
    gate = tensor(g, N, dtype=dtype) if M % 2 else tensor(g, 2, N, dtype=dtype)
    check(args, f"{size} all", on, dtype=dtype, bias=tensor(g, N, dtype=dtype), act=dvdq.ACT_GELU_TANH, gate=gate, residual=tensor(g, M, N, dtype=dtype))


# a size for each shape of tile (0: 256 x 256 .. 4: 64 x 64), whole and in parts of K (see test_rows8_linear8.py)
WAYS = {(0, 1): (2600, 5120, 784), (0, 3): (2600, 1540, 13824), (1, 1): (12000, 260, 1168), (1, 4): (6200, 136, 8208), (2, 1): (12000, 136, 48),
        (2, 11): (70, 1540, 8208), (3, 1): (70, 9000, 48), (3, 7): (70, 1540, 4112), (4, 1): (40, 48, 48), (4, 4): (40, 48, 2064)}


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("dtype", TYPES)
def test_every_shape_of_tile(way, dtype):
    M, N, K = WAYS[way]
    g = gen(M)
    args = operands(g, M, N, K)
    bias, gate, residual = tensor(g, N, dtype=dtype), tensor(g, 2, N, dtype=dtype), tensor(g, M, N, dtype=dtype)
    for kw in ({}, {"gate": gate}, {"residual": residual}, {"gate": gate, "residual": residual, "act": dvdq.ACT_SILU}, {"gate": residual, "residual": residual}):
        check(args, f"{way} {dtype} {list(kw)}", DEV, dtype=dtype, bias=bias, **kw)


# rows that are no whole pieces: through registers as 128 x 128 and 64 x 64 tiles, whole and in parts, and copied first
ROWS = [(6242, 1160, 1156), (2000, 500, 1000), (417, 200, 136), (188, 1376, 1720), (100, 3000, 3001), (40, 1000, 9001), (2600, 5120, 777), (600, 2000, 4001), (70, 130, 100)]


@pytest.mark.parametrize("size", ROWS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_are_no_whole_pieces(size, dtype):
    M, N, K = size
    g = gen(K)
    args = operands(g, M, N, K)
    check(args, f"{size} {dtype}", DEV, dtype=dtype)
    check(args, f"{size} {dtype} all", DEV, dtype=dtype, bias=tensor(g, N, dtype=dtype), act=dvdq.ACT_GELU, gate=tensor(g, N, dtype=dtype), residual=tensor(g, M, N, dtype=dtype))
    # whole pieces at an address that is none
    x, w = ints(g, M, K + 40)[:, 8:8 + K // 16 * 16], ints(g, N, K + 25)[:, 1:1 + K // 16 * 16]
    check((x, args[1], w, args[3]), f"{size} {dtype} address", DEV, dtype=dtype, residual=tensor(g, M, N, dtype=dtype))


@pytest.mark.parametrize("M", [3, 40, 700])
@pytest.mark.parametrize("act", [0, 1, 2, 3])
def test_epilogues(M, act):
    N, K = 200, 320
    g = gen(act)
    args = operands(g, M, N, K)
    for dtype in TYPES:
        for bias in (None, tensor(g, N, dtype=dtype)):
            for gate in (None, tensor(g, N, dtype=dtype), tensor(g, M, N, dtype=dtype)):
                for residual in (None, tensor(g, M, N, dtype=dtype)):
                    check(args, f"{M} act {act} {dtype} {bias is not None} {gate is None or gate.dim()} {residual is not None}", dtype=dtype,
                          bias=bias, act=act, gate=gate, residual=residual)


def test_gate_rows_that_end_inside_tiles():
    g = gen(2)
    args = operands(g, 570, 300, 256)
    for G in (2, 3, 5, 19, 30, 57, 114, 570):
        check(args, f"{G} rows of the gate", gate=tensor(g, G, 300, dtype=torch.bfloat16), residual=tensor(g, 570, 300, dtype=torch.bfloat16))


@pytest.mark.parametrize("M", [2, 150])
def test_views(M):
    """Rows of any pitch at any address, outputs inside larger tensors, the output in the residual's place."""
    g = gen(3)
    N, K = 96, 257
    for offset, pitch in ((0, 272), (1, 261), (16, 288), (3, 259), (5, 320)):
        x = ints(g, M, pitch)[:, offset:offset + K] if offset + K <= pitch else ints(g, M, pitch + offset)[:, offset:offset + K]
        w = ints(g, N, pitch + offset + 7)[:, offset:offset + K]
        xs, ws = torch.rand((M,), generator=g, device=DEV) / 50, torch.rand((N,), generator=g, device=DEV) / 50
        for k in (K, 256, 240):
            args = (x[:, :k], xs, w[:, :k], ws)
            out = torch.zeros((M, N + 9), dtype=torch.float16, device=DEV)
            check(args, f"offset {offset} pitch {pitch} K {k}", y=out[:, 4:4 + N], residual=tensor(g, M, N + 3, dtype=torch.float16)[:, 1:1 + N])
            assert not out[:, :4].any() and not out[:, 4 + N:].any()
    r = tensor(g, M, N, dtype=torch.bfloat16)
    args = (x, xs, w, ws)
    want = dvdq.linear8(*args, residual=r)
    assert dvdq.linear8(*args, residual=r, y=r) is r and torch.equal(r, want)
    one = ints(g, 1, K).expand(M, K)                                          # one token for all rows: rows that lie on one another are refused
    with pytest.raises(dvdq.DvdqError):
        dvdq.linear8(one, xs, w, ws)


def test_the_largest_sums():
    """K at its limit with every product at its largest: one below 2^31."""
    K = 131071
    for M in (1, 20):
        x = torch.full((M, K), -128, dtype=torch.int8, device=DEV)
        w = torch.full((33, K), -128, dtype=torch.int8, device=DEV)
        w[1] = 127
        y = dvdq.linear8(x, torch.ones(M, device=DEV), w, torch.ones(33, device=DEV), dtype=torch.float32)
        want = torch.full((M, 33), float(128 * 128 * K), device=DEV)
        want[:, 1] = -128.0 * 127 * K
        assert torch.equal(y, want)
    with pytest.raises(dvdq.DvdqError):
        dvdq.linear8(torch.zeros((1, K + 1), dtype=torch.int8, device=DEV), torch.ones(1, device=DEV), torch.zeros((1, K + 1), dtype=torch.int8, device=DEV), torch.ones(1, device=DEV))


def test_nan_and_infinite_scales_stay_in_their_rows():
    g = gen(4)
    for M in (5, 90):
        args = operands(g, M, 70, 96)
        args[1][1] = float("nan")
        args[1][3] = float("inf")
        args[3][2] = float("nan")
        y = dvdq.linear8(*args, bias=torch.ones(70, device=DEV, dtype=torch.bfloat16))
        assert y[1].isnan().all() and y[:, 2].isnan().all()
        rest = y[[i for i in range(M) if i not in (1, 3)]][:, [i for i in range(70) if i != 2]]
        assert rest.isfinite().all() and not y[3].isfinite().any()


def test_sums_are_exact_and_do_not_change():
    g = gen(5)
    for M, N, K in ((6, 500, 2048), (300, 300, 6000), (900, 1100, 640)):
        args = operands(g, M, N, K)
        one = (args[0], torch.ones(M, device=DEV), args[2], torch.ones(N, device=DEV))
        y = dvdq.linear8(*one, dtype=torch.float32)
        assert torch.equal(y.cpu().double(), (args[0].cpu().double() @ args[2].cpu().double().t()).float().double())
        for _ in range(3):
            assert torch.equal(dvdq.linear8(*one, dtype=torch.float32), y)
        assert torch.equal(dvdq.linear8(args[0][1:2], one[1][:1], args[2], one[3], dtype=torch.float32)[0], y[1])


def test_a_run_of_them_together():
    """Residual and norm into codes, the product up with its activation, codes again, the product down into the residual: as a block of a model has them."""
    g = gen(6)
    M, D, F = 333, 384, 1000
    dt = torch.bfloat16
    x, r, nw = tensor(g, M, D, dtype=dt), tensor(g, M, D, dtype=dt), (1 + tensor(g, D, scale=0.2)).to(dt)
    w1, w2, w3 = tensor(g, F, D, scale=D ** -0.5), tensor(g, F, D, scale=D ** -0.5), tensor(g, D, F, scale=F ** -0.5)
    (c1, s1), (c2, s2), (c3, s3) = (dvdq.quant8(w) for w in (w1, w2, w3))
    codes, scale, h = dvdq.rms_norm_quant(x, nw, residual=r)
    both = dvdq.linear8(codes, scale, torch.cat([c1, c2]), torch.cat([s1, s2]))
    mid, mid_scale = dvdq.quant8(both[:, :F], up=both[:, F:], act=dvdq.ACT_SILU)
    y = dvdq.linear8(mid, mid_scale, c3, s3, residual=h)
    # each step from the one before
    ref, slack = linear8_64(mid, mid_scale, c3, s3, residual=h)
    assert_close(y, ref, slack, "down")
    # and the whole against 32 bits without codes: a code is off by half a step of max / 127, 0.3 to 0.5 % of a typical row's norm, in each of five roundings
    f = h.float()
    n = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + 1e-6) * nw.float()
    a, b = n @ w1.t(), n @ w2.t()
    full = (torch.nn.functional.silu(a) * b) @ w3.t()
    off = ((y.float() - f) - full).norm() / full.norm()
    assert off < 0.05, float(off)
    # codes of the norm in the 4-bit layer (W4A8), whose weights have zero-points
    wq, ws, wz = dvdq.bgr_quantize(w1)
    codes, scale, sums = dvdq.rms_norm_quant(h, nw, want_rowsum=True)
    got = dvdq.w4ax_gemm(codes, scale, dvdq.w4_prepack(wq), ws, 8, dvdq.W_NATIVE, w_zero=wz, code_rowsum=sums)
    low, high = (wq & 15).to(torch.int8), (wq >> 4).to(torch.int8)
    w4 = torch.stack([low, high], -1).flatten(1)
    w4 = torch.where(w4 > 7, w4 - 16, w4).double() - wz[:, None].double()
    want = (codes.double() @ w4.t()) * scale.double()[:, None] * ws.double()
    assert ((got.double() - want).norm() / want.norm()) < 2.0 ** -8
    # and codes of the rotating quantizer here
    codes, scale = dvdq.rotate_quant(h, 1, 8)
    assert_close(dvdq.linear8(codes, scale, c1, s1), *linear8_64(codes, scale, c1, s1), "rotate_quant")


@pytest.mark.parametrize("size", [(420000, 5200, 64), (420000, 5200, 72), (40000, 64, 131056), (40000, 64, 131071), (40000, 1000, 131071)])
def test_beyond_32_bits_of_elements(size):
    """Outputs of more than 2^31 elements, codes of more than 2^32 bytes: straight, copied and through registers."""
    M, N, K = size
    g = gen(9)
    codes = torch.empty((M, K), dtype=torch.int8, device=DEV).random_(-127, 128, generator=g)
    _, xs, w, ws = operands(g, 1, N, K)
    xs = torch.exp(tensor(g, M, scale=0.3)) / 127
    y = torch.ones((M, N), dtype=torch.bfloat16, device=DEV)
    gate = tensor(g, N, dtype=torch.bfloat16)
    assert dvdq.linear8(codes, xs, w, ws, gate=gate, residual=y, y=y) is y
    for first in (0, M // 2 - 3, (1 << 31) // N - 3, (1 << 32) // K - 3, M - 50):
        if 0 <= first < M:
            part = slice(first, min(first + 50, M))
            ref, slack = linear8_64(codes[part], xs[part], w, ws, gate=gate, residual=torch.ones_like(y[part]), device=DEV)
            assert_close(y[part], ref, slack, f"{size} from row {first}")
