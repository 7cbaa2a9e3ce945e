"""The 16-bit matrix product and its epilogue against the formula in 64 bits."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import assert_close, linear64

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = {"none": 0, "silu": 1, "gelu_tanh": 2, "gelu": 3}


def inputs(M, N, K, dtype, gate_rows=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda shape, s=1.0: (s * torch.randn(shape, generator=g)).to(dtype).cuda()   # noqa: E731
    return {"x": r((M, K)), "w": r((N, K), K ** -0.5), "bias": r((N,), 0.5), "gate": r((gate_rows, N)) if gate_rows else None,
            "residual": r((M, N))}


def check(got, x, w, bias=None, act=0, gate=None, residual=None, what=""):
    ref, slack = linear64(x, w, bias, act, gate, residual)
    assert_close(got, ref, slack, what)


# sizes at, below and above tiles and slices; single tokens; odd channel counts; long sums
SHAPES = [(1, 1, 1), (1, 64, 8), (2, 9216, 1536), (1, 1, 4096), (3, 257, 100), (7, 130, 72), (16, 512, 512), (17, 384, 1000), (31, 96, 2048),
          (33, 1000, 264), (64, 64, 64), (65, 65, 65), (100, 1160, 1152), (127, 129, 200), (128, 128, 13824), (129, 257, 1157), (200, 4608, 1536),
          (255, 256, 96), (256, 512, 1024), (300, 300, 33), (513, 1156, 1160), (1000, 999, 998), (1560, 520, 4096), (2049, 129, 320),
          (4100, 260, 136), (5000, 768, 72)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_product(shape, dtype):
    t = inputs(*shape, DTYPES[dtype])
    check(dvdq.linear(t["x"], t["w"]), t["x"], t["w"], what="product")
    check(dvdq.linear(t["x"], t["w"], t["bias"], residual=t["residual"]), t["x"], t["w"], t["bias"], residual=t["residual"], what="residual")


# (M, N, K, shape of tile, parts of K, whether workgroups take several tiles), every way an aligned product is taken
WAYS = [(57652, 395, 312, 0, 1, True), (53282, 135, 272, 0, 1, False), (16728, 131, 4320, 0, 3, False), (2116, 7277, 784, 1, 1, True),
        (17948, 142, 624, 1, 1, False), (5694, 134, 3400, 1, 4, False), (33862, 137, 72, 2, 1, True), (18670, 68, 80, 2, 1, False),
        (70, 2705, 1432, 2, 6, False), (7212, 1093, 64, 3, 1, True), (8674, 67, 64, 3, 1, False), (70, 1407, 1296, 3, 6, False),
        (34, 65, 72, 4, 1, False), (36, 67, 744, 4, 3, False)]
TILES = [(256, 256, 1), (256, 128, 1), (128, 128, 2), (128, 64, 2), (64, 64, 4)]    # channels, tokens, workgroups per compute unit


@pytest.mark.parametrize("way", WAYS)
def test_every_way(way):
    M, N, K, shape, parts, several = way
    assert dvdq.bench_linear_choice(M, N, K) == shape + 16 * parts
    bn, bm, per_cu = TILES[shape]
    assert (-(-N // bn) * -(-M // bm) * parts > 256 * per_cu) == several
    g = torch.Generator(device="cuda").manual_seed(7)
    r = lambda *s, k=1.0: (k * torch.randn(s, generator=g, device="cuda")).to(torch.bfloat16)   # noqa: E731
    x, w, bias, gate, res = r(M, K), r(N, K, k=K ** -0.5), r(N), r(2, N), r(M, N)
    got = dvdq.linear(x, w, bias, 1, gate, res)
    ref, slack = linear64(x, w, bias, 1, gate, res, device="cuda")
    assert_close(got, ref, slack, str(way))
    # and once more over the residual, with another gate and no bias
    y = res.clone()
    dvdq.linear(x, w, None, 2, gate[1], y, y=y)
    ref, slack = linear64(x, w, None, 2, gate[1], res, device="cuda")
    assert_close(y, ref, slack, str(way) + " in place")


@pytest.mark.parametrize("shape,way", [((129, 257, 1157), 4 + 16 * 5 + 4096), ((9000, 3000, 203), 2 + 16 + 4096), ((300, 300, 33), 2 + 16 + 8192),
                                       ((100, 1160, 1152), 2 + 16 * 4 + 8192), ((31, 96, 2048), 2 + 16 * 8 + 8192)])
def test_every_way_of_unaligned_rows(shape, way):
    M, N, K = shape
    assert dvdq.bench_linear_choice(M, N, K, True) == way
    g = torch.Generator(device="cuda").manual_seed(8)
    x, w = (torch.randn((n, K + 3), generator=g, device="cuda").to(torch.float16)[:, 1:K + 1] for n in (M, N))
    got = dvdq.linear(x, w)
    ref, slack = linear64(x, w, device="cuda")
    assert_close(got, ref, slack, str(shape))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("shape", [(6, 200, 96), (90, 136, 256), (90, 133, 77), (720, 520, 640), (1026, 300, 1024)])
def test_epilogue(shape, act, dtype):
    M, N, K = shape
    for gate_rows in (1, 2, M):
        t = inputs(M, N, K, DTYPES[dtype], gate_rows)
        for bias in (t["bias"], None):
            for gate in (t["gate"], None):
                for residual in (t["residual"], None):
                    got = dvdq.linear(t["x"], t["w"], bias, ACTS[act], gate, residual)
                    check(got, t["x"], t["w"], bias, ACTS[act], gate, residual,
                          f"bias {bias is not None} gate {gate is not None} residual {residual is not None}")
    one = t["gate"][0]
    assert torch.equal(dvdq.linear(t["x"], t["w"], gate=one), dvdq.linear(t["x"], t["w"], gate=one[None]))


@pytest.mark.parametrize("shape", [(5, 72, 40), (300, 264, 136), (300, 261, 131)])
@pytest.mark.parametrize("odd", [0, 1, 3, 8])
def test_pitches_and_addresses(shape, odd):
    """Views whose rows begin at any element, outputs inside a larger buffer, the residual overwritten by the output."""
    M, N, K = shape
    g = torch.Generator().manual_seed(1)
    xb, wb, yb = (torch.randn((r, c + odd + 5), generator=g).to(torch.bfloat16).cuda() for r, c in ((M, K), (N, K), (M, N)))
    x, w, y = xb[:, odd:odd + K], wb[:, odd:odd + K], yb[:, odd:odd + N]
    vec = torch.randn((2, N + odd), generator=g).to(torch.bfloat16).cuda()
    bias, gate = vec[0, odd:], vec[1, odd:]
    before = yb.clone()
    want = dvdq.linear(x.contiguous(), w.contiguous(), bias.contiguous(), 2, gate.contiguous(), y.contiguous())
    check(want, x, w, bias, 2, gate, y.clone())
    out = dvdq.linear(x, w, bias, 2, gate, residual=y, y=y)
    assert out.data_ptr() == y.data_ptr()
    check(out, x, w, bias, 2, gate, before[:, odd:odd + N])
    assert torch.equal(yb[:, :odd], before[:, :odd]) and torch.equal(yb[:, odd + N:], before[:, odd + N:])


@pytest.mark.parametrize("shape", [(3, 64, 100), (40, 64, 100), (200, 300, 100), (260, 264, 1032), (2, 64, 4000), (260, 264, 1031)])
def test_nan_and_infinities_stay_in_their_rows(shape):
    """What lies beside a row, past K and past M and N, does not enter: not even NaN times nothing."""
    M, N, K = shape
    t = inputs(M, N, K, torch.float16)
    nan = float("nan")
    xb = torch.full((M + 2, K + 9), nan, dtype=torch.float16, device="cuda")
    wb = torch.full((N + 2, K + 9), float("inf"), dtype=torch.float16, device="cuda")
    x, w = xb[1:M + 1, :K], wb[1:N + 1, :K]
    x.copy_(t["x"])
    w.copy_(t["w"])
    got = dvdq.linear(x, w, t["bias"], 1)
    check(got, t["x"], t["w"], t["bias"], 1)
    clean = got.clone()
    x[M // 2, K - 1] = nan
    w[N // 2, 0] = float("inf")
    got = dvdq.linear(x, w, t["bias"])
    rows, cols = torch.arange(M).cuda() != M // 2, torch.arange(N).cuda() != N // 2
    assert bool(got[M // 2].isnan().all()) and not bool(got[:, N // 2].isfinite().any())
    assert torch.equal(dvdq.linear(x, w, t["bias"], 1)[rows][:, cols], clean[rows][:, cols])


def test_overflow_of_fp16_is_infinite():
    x = torch.full((4, 128), 200.0, dtype=torch.float16, device="cuda")
    w = torch.full((8, 128), 200.0, dtype=torch.float16, device="cuda")
    w[3] = -200.0
    y = dvdq.linear(x, w)
    assert bool((y[:, 3] == -float("inf")).all()) and bool((y[:, :3] == float("inf")).all())


@pytest.mark.parametrize("shape", [(2, 4608, 1536), (100, 640, 2048), (512, 512, 4096), (1500, 1152, 1160)])
def test_same_result_every_time_and_workspace_contents_do_not_matter(shape):
    M, N, K = shape
    t = inputs(M, N, K, torch.bfloat16, 1)
    n = dvdq.linear_workspace_bytes(M, N, K)
    want = dvdq.linear(t["x"], t["w"], t["bias"], 2, t["gate"], t["residual"])
    for fill in (0, 255, 127):
        ws = torch.full((max(n, 16),), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(dvdq.linear(t["x"], t["w"], t["bias"], 2, t["gate"], t["residual"], workspace=ws), want)


def test_rows_past_32_bit_offsets():
    """Activations and outputs of more than 2^32 bytes: spot rows against the formula."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    M, N, K = 1 << 20, 2056, 2304
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = (torch.randn((N, K), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)
    gate = torch.randn((4, N), generator=g, device="cuda").to(torch.bfloat16)
    y = dvdq.linear(x, w, gate=gate, residual=None)
    for rows in (slice(0, 3), slice(M // 2 - 2, M // 2 + 2), slice(M - 3, M)):
        r = torch.arange(M)[rows]
        ref, slack = linear64(x[rows], w)
        gr = gate.cpu().double()[r // (M // 4)]
        assert_close(y[rows], ref * gr, slack * gr.abs() + 2.0 ** -22 * (ref * gr).abs(), f"rows {rows}")


def test_nothing_to_do_and_refusals():
    t = inputs(6, 8, 16, torch.bfloat16, 2)
    assert dvdq.linear(t["x"][:0], t["w"], t["bias"]).shape == (0, 8)
    with pytest.raises(TypeError):
        dvdq.linear(t["x"].cpu(), t["w"])
    with pytest.raises(TypeError):
        dvdq.linear(t["x"].float(), t["w"].float())
    with pytest.raises(TypeError):
        dvdq.linear(t["x"], t["w"].half())
    with pytest.raises(TypeError):
        dvdq.linear(t["x"], t["w"], t["bias"].float())
    with pytest.raises(ValueError):
        dvdq.linear(t["x"], t["w"][:, :8])
    with pytest.raises(ValueError):
        dvdq.linear(t["x"], t["w"], t["bias"][:4])
    with pytest.raises(ValueError):
        dvdq.linear(t["x"], t["w"], residual=t["residual"][:3])
    with pytest.raises(ValueError):
        dvdq.linear(t["x"].t().contiguous().t(), t["w"])
    with pytest.raises(ValueError):
        dvdq.linear(t["x"], t["w"], y=torch.empty((6, 9), dtype=torch.bfloat16, device="cuda"))
    for kw, status in ((dict(act=4), 3), (dict(act=-1), 3), (dict(gate=torch.zeros((4, 8), dtype=torch.bfloat16, device="cuda")), 2)):
        with pytest.raises(dvdq.DvdqError) as e:
            dvdq.linear(t["x"], t["w"], **kw)
        assert e.value.status == status


@pytest.mark.parametrize("shape", [(2, 2048, 1536), (512, 640, 4096), (3000, 520, 264)])
def test_streams_and_graph(shape):
    M, N, K = shape
    t = inputs(M, N, K, torch.bfloat16, 1)
    args = (t["w"], t["bias"], 2, t["gate"], t["residual"])
    want = dvdq.linear(t["x"], *args)
    torch.cuda.synchronize()
    n = dvdq.linear_workspace_bytes(M, N, K)
    ws = torch.empty((n,), dtype=torch.uint8, device="cuda") if n else None
    y = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dvdq.linear(t["x"], *args, y=y, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dvdq.linear(t["x"], *args, y=y, workspace=ws)
    for i in range(4):
        t["x"].copy_(torch.roll(t["x"], 1, 0))
        graph.replay()
        eager = dvdq.linear(t["x"], *args)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i
