"""Channels-last group norm against its formula in 64 bits."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import assert_close, group_norm64

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def inputs(B, S, C, dtype, seed=0, offset=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, S, C), generator=g) * torch.exp(0.5 * torch.randn((B, 1, C), generator=g)) + offset * torch.randn((B, 1, C), generator=g)
    return x.to(dtype).cuda(), (1 + 0.2 * torch.randn((C,), generator=g)).to(dtype).cuda(), (0.2 * torch.randn((C,), generator=g)).to(dtype).cuda()


def check(got, x, groups, w=None, b=None, eps=1e-5, act=0, what=""):
    ref, slack = group_norm64(x, groups, w, b, eps, act)
    assert_close(got, ref, slack, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [
    (1, 1, 1, 1), (2, 1, 32, 8), (1, 2, 64, 64), (3, 17, 96, 32), (1, 1560, 512, 32), (2, 1001, 320, 32), (1, 4097, 30, 3),
    (1, 777, 33, 11), (2, 300, 1024, 32), (1, 50, 4096, 32), (1, 40, 2050, 2), (1, 5000, 7, 1), (5, 64, 20, 5), (1, 70000, 16, 4),
    (1, 33000, 128, 1), (4, 2049, 8, 8),
])
def test_against_formula(shape, dtype):
    B, S, C, groups = shape
    x, w, b = inputs(B, S, C, DTYPES[dtype])
    check(dvdq.group_norm(x, groups), x, groups, what="plain")
    check(dvdq.group_norm(x, groups, w, b, eps=1e-6, act=dvdq.ACT_SILU), x, groups, w, b, 1e-6, 1, "affine, silu")
    check(dvdq.group_norm(x, groups, w, None, eps=1e-3), x, groups, w, None, 1e-3, 0, "weight alone")
    check(dvdq.group_norm(x, groups, None, b), x, groups, None, b, what="bias alone")


@pytest.mark.parametrize("offset", [100.0, -3000.0])
@pytest.mark.parametrize("shape", [(1, 900, 64, 8), (1, 90000, 64, 8)])
def test_channels_far_from_zero(shape, offset):
    """All channels of a group a thousand deviations from zero: sums of squares would lose the variance, differences do not."""
    B, S, C, groups = shape
    g = torch.Generator().manual_seed(1)
    x = (offset + torch.randn((B, S, C), generator=g)).cuda()
    x[:, 0] = 0.0                                  # a first row that is nothing like the others
    check(dvdq.group_norm(x, groups), x, groups)


@pytest.mark.parametrize("S", [3, 2000, 40000])
def test_constant_groups(S):
    x = torch.full((2, S, 48), 3.140625, dtype=torch.float32, device="cuda")
    w = torch.full((48,), 2.0, device="cuda")
    b = torch.arange(48, dtype=torch.float32, device="cuda")
    assert torch.equal(dvdq.group_norm(x, 6, w, b), b.expand(2, S, 48))
    # eps = 0 as well: 0 / 0 is NaN by the formula
    assert bool(dvdq.group_norm(x, 6, w, b, eps=0.0).isnan().all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("S", [5, 3000, 50000])
def test_nan_and_infinities_stay_in_their_group(S, bad):
    x, w, b = inputs(2, S, 40, torch.float32)
    for s in (0, S // 2, S - 1):
        y = x.clone()
        y[1, s, 13] = bad
        got = dvdq.group_norm(y, 4, w, b, act=dvdq.ACT_SILU)
        want = dvdq.group_norm(x, 4, w, b, act=dvdq.ACT_SILU)
        assert bool(got[1, :, 10:20].isnan().all())
        keep = torch.ones((40,), dtype=torch.bool)
        keep[10:20] = False
        assert torch.equal(got[0], want[0]) and torch.equal(got[1][:, keep.cuda()], want[1][:, keep.cuda()])


@pytest.mark.parametrize("dtype", DTYPES)
def test_views_and_in_place(dtype):
    dtype = DTYPES[dtype]
    # a channels-last module's tensor, [B, C, T, H, W]
    g = torch.Generator().manual_seed(2)
    m = torch.randn((2, 24, 3, 5, 7), generator=g).to(dtype).cuda().contiguous(memory_format=torch.channels_last_3d)
    got = dvdq.group_norm(m.movedim(1, -1), 6, act=dvdq.ACT_SILU)
    flat = m.movedim(1, -1).reshape(2, 105, 24)
    check(got.reshape(2, 105, 24), flat, 6, act=1)
    assert got.shape == (2, 3, 5, 7, 24)
    # rows that begin at odd elements, channels beside them untouched, in place
    buf = torch.randn((2, 500, 51), generator=g).to(dtype).cuda()
    x = buf[:, :, 1:49]
    before = buf.clone()
    want = dvdq.group_norm(x, 4)
    check(want, x, 4)
    assert dvdq.group_norm(x, 4, y=x).data_ptr() == x.data_ptr()
    assert torch.equal(x, want) and torch.equal(buf[:, :, 49:], before[:, :, 49:]) and torch.equal(buf[:, :, 0], before[:, :, 0])
    # every second batch of a tensor, into a view
    y = torch.zeros((2, 500, 60), dtype=dtype, device="cuda")
    wide = torch.randn((4, 500, 48), generator=g).to(dtype).cuda()
    dvdq.group_norm(wide[::2], 4, y=y[:, :, 5:53])
    check(y[:, :, 5:53], wide[::2].contiguous(), 4)
    assert not y[:, :, :5].any() and not y[:, :, 53:].any()


def test_two_dimensions():
    x, w, b = inputs(6, 1, 64, torch.bfloat16)
    check(dvdq.group_norm(x[:, 0], 4, w, b)[:, None], x, 4, w, b)


@pytest.mark.parametrize("shape", [(1, 100, 64, 8), (2, 30000, 64, 8), (1, 300000, 64, 8)])
def test_workspace_contents_do_not_matter(shape):
    B, S, C, groups = shape
    x, w, b = inputs(B, S, C, torch.bfloat16)
    want = dvdq.group_norm(x, groups, w, b)
    for fill in (0, 255, 127):
        ws = torch.full((dvdq.group_norm_workspace_bytes(B, S, C, groups),), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(dvdq.group_norm(x, groups, w, b, workspace=ws), want)


def test_rows_past_32_bit_offsets():
    """More than 2^32 bytes of input: the last rows are normalized with the statistics of all."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    S, C, groups = (1 << 22) + 3, 520, 4
    x = torch.empty((1, S, C), dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    x[:, -1] = 3.0
    y = dvdq.group_norm(x, groups, eps=0.0)
    for g in range(groups):
        ch = slice(g * 130, g * 130 + 130)
        total = sq = 0.0
        for s in range(0, S, 1 << 19):
            part = x[0, s:s + (1 << 19), ch].double()
            total, sq = total + float(part.sum()), sq + float((part * part).sum())
        mean = total / (S * 130)
        rstd = (sq / (S * 130) - mean * mean) ** -0.5
        for rows in (slice(0, 4), slice(S - 4, S)):
            ref = (x[0, rows, ch].cpu().double() - mean) * rstd
            assert_close(y[0, rows, ch], ref, 1e-5, f"group {g}")


def test_nothing_to_do_and_refusals():
    for shape in ((0, 4, 8), (2, 0, 8), (0, 8)):
        assert dvdq.group_norm(torch.empty(shape, dtype=torch.float16, device="cuda"), 2).shape == shape
    x, w, b = inputs(2, 6, 8, torch.bfloat16)
    with pytest.raises(TypeError):
        dvdq.group_norm(x.cpu(), 2)
    with pytest.raises(TypeError):
        dvdq.group_norm(x, 2, w.float(), b)
    with pytest.raises(ValueError):
        dvdq.group_norm(x, 2, w[:7], b)
    with pytest.raises(ValueError):
        dvdq.group_norm(x.transpose(1, 2), 2)                        # channels not dense
    with pytest.raises(ValueError):
        dvdq.group_norm(x.view(2, 2, 3, 8).transpose(1, 2), 2)       # rows not in order
    for groups, status in ((3, 2), (0, 2), (-2, 2)):
        with pytest.raises(dvdq.DvdqError) as e:
            dvdq.group_norm(x, groups)
        assert e.value.status == status
    for kw, status in ((dict(eps=-1.0), 2), (dict(eps=float("nan")), 2), (dict(act=dvdq.ACT_GELU), 3),
                       (dict(workspace=torch.empty((8,), dtype=torch.uint8, device="cuda")), 4)):
        with pytest.raises(dvdq.DvdqError) as e:
            dvdq.group_norm(x, 2, **kw)
        assert e.value.status == status


@pytest.mark.parametrize("shape", [(1, 400, 64, 8), (1, 60000, 64, 8)])
def test_streams_and_graph(shape):
    B, S, C, groups = shape
    x, w, b = inputs(B, S, C, torch.bfloat16)
    want = dvdq.group_norm(x, groups, w, b, act=dvdq.ACT_SILU)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = torch.empty((dvdq.group_norm_workspace_bytes(B, S, C, groups),), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(x)
    side.wait_stream(torch.cuda.current_stream())
    dvdq.group_norm(x, groups, w, b, act=dvdq.ACT_SILU, y=y, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dvdq.group_norm(x, groups, w, b, act=dvdq.ACT_SILU, y=y, workspace=ws)
    for i in range(4):
        x.copy_(torch.roll(x, 1, 1) * 1.5)
        graph.replay()
        eager = dvdq.group_norm(x, groups, w, b, act=dvdq.ACT_SILU)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i
