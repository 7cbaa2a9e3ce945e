"""Rotary positions against their formula in 64 bits."""
import math

import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import F32, assert_close, rope64

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def inputs(B, T, Hq, Hk, D, sections, dtype, n_pos=97, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((B, T, Hq, D), generator=g).to(dtype).cuda()
    k = torch.randn((B, T, Hk, D), generator=g).to(dtype).cuda()
    freq, mag = dvdq.rope_frequencies(sections)
    table = dvdq.rope_table(n_pos, [f / scale for f in freq], mag)
    pos = torch.randint(0, n_pos, (B, T, len(sections)), generator=g, dtype=torch.int32).cuda()
    return q, k, table, pos


def check(got, x, table, pos, sections, interleaved, inverse=False, what=""):
    ref, mag = rope64(x, table, pos, sections, interleaved, inverse)
    assert_close(got, ref, 3 * F32 * mag, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [
    (1, 1, 1, 1, 2, (2,)), (1, 1, 40, 8, 128, (128,)), (2, 5, 3, 1, 64, (64,)), (1, 130, 12, 12, 128, (44, 42, 42)),
    (2, 33, 4, 4, 128, (16, 56, 56)), (1, 67, 14, 2, 80, (40,)), (3, 7, 5, 3, 72, (54,)), (1, 9, 2, 2, 96, (2, 30, 64)),
    (1, 3, 1, 1, 1024, (1024,)), (1, 17, 7, 1, 66, (22,)), (2, 3, 2, 1, 37, (6, 4, 2, 8)), (1, 4, 2, 2, 256, (250,)),
    (1, 2, 3, 3, 128, (0, 64, 64)),
])
def test_against_formula(shape, interleaved, dtype):
    B, T, Hq, Hk, D, sections = shape
    q, k, table, pos = inputs(B, T, Hq, Hk, D, sections, DTYPES[dtype])
    p = pos if len(sections) > 1 else pos[..., 0].contiguous()
    qo, ko = dvdq.rope(q, k, table, p, sections if len(sections) > 1 else None, interleaved)
    check(qo, q, table, pos, sections, interleaved, what="q")
    check(ko, k, table, pos, sections, interleaved, what="k")
    assert torch.equal(dvdq.rope(q, None, table, p, sections if len(sections) > 1 else None, interleaved), qo)


@pytest.mark.parametrize("interleaved", [False, True])
def test_views_of_a_fused_projection_in_place_and_transposed(interleaved):
    B, T, H, D = 2, 21, 6, 64
    g = torch.Generator().manual_seed(3)
    _, _, table, pos = inputs(B, T, 1, 1, D, (64,), torch.bfloat16)
    pos = pos[..., 0].contiguous()
    qkv = torch.randn((B, T, 3 * H * D + 3), generator=g).to(torch.bfloat16).cuda()     # rows that begin at odd elements
    view = qkv[..., 1:1 + 3 * H * D].unflatten(-1, (3, H, D))
    q, k, v = view[:, :, 0], view[:, :, 1], view[:, :, 2]
    want_q, want_k = dvdq.rope(q, k, table, pos, None, interleaved)
    check(want_q, q, table, pos[..., None], (64,), interleaved)
    # into [batch, heads, tokens, D]
    qt, kt = (torch.empty((B, H, T, D), dtype=q.dtype, device=q.device) for _ in range(2))
    dvdq.rope(q, k, table, pos, None, interleaved, q_out=qt.transpose(1, 2), k_out=kt.transpose(1, 2))
    assert torch.equal(qt.transpose(1, 2), want_q) and torch.equal(kt.transpose(1, 2), want_k)
    # in place: nothing beside q and k changes
    before = qkv.clone()
    dvdq.rope(q, k, table, pos, None, interleaved, q_out=q, k_out=k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    assert torch.equal(qkv[..., 1 + 2 * H * D:], before[..., 1 + 2 * H * D:]) and torch.equal(qkv[..., 0], before[..., 0])
    # part of the head, in place, and only one of the two in place
    t2 = table[:, :9].contiguous()
    want = dvdq.rope(v, None, t2, pos, None, interleaved)
    check(want, v, t2, pos[..., None], (18,), interleaved)
    other = torch.empty_like(want)
    src = v.clone()
    dvdq.rope(v, src, t2, pos, None, interleaved, q_out=v, k_out=other)
    assert torch.equal(v, want) and torch.equal(other, want)
    dvdq.rope(src, None, t2, pos, None, interleaved, q_out=src)
    assert torch.equal(src, want)


def test_three_dimensions_and_shared_positions():
    q, k, table, pos = inputs(1, 13, 4, 2, 64, (64,), torch.float16)
    p = pos[0, :, 0].contiguous()
    want, _ = dvdq.rope(q, k, table, p)
    assert torch.equal(dvdq.rope(q[0], k[0], table, p)[0], want[0])
    q2 = q.expand(3, -1, -1, -1)                       # one tensor for every batch, one row of positions for all
    assert torch.equal(dvdq.rope(q2, None, table, p), want.expand(3, -1, -1, -1))


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_outside_the_table(interleaved):
    sections = (6, 10)
    q, k, table, pos = inputs(1, 8, 2, 1, 24, sections, torch.float32, n_pos=11)
    pos[0, 0], pos[0, 1, 0], pos[0, 2, 1] = -1, -5, -(2 ** 31)
    pos[0, 3, 0], pos[0, 4], pos[0, 5, 1] = 11, 2 ** 31 - 1, 12
    q[0, 0, 0, 1] = float("inf")                       # as they are: no inf * 0
    q[0, 0, 1, 2] = float("nan")
    qo, ko = dvdq.rope(q, k, table, pos, sections, interleaved)
    check(qo, q, table, pos, sections, interleaved)
    check(ko, k, table, pos, sections, interleaved)
    assert torch.equal(ko[0, 0], k[0, 0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(interleaved):
    """Against differences: d/dx sum(w * rope(x)) along a direction, in fp32 where the map is linear."""
    sections = (10, 6)
    x, _, table, pos = inputs(2, 5, 3, 1, 20, sections, torch.float32)
    w = torch.randn(x.shape, generator=torch.Generator().manual_seed(5)).cuda()
    grad = dvdq.rope(w, None, table, pos, sections, interleaved, inverse=True)
    check(grad, w, table, pos, sections, interleaved, inverse=True)
    d = torch.randn(x.shape, generator=torch.Generator().manual_seed(6)).cuda()
    up = dvdq.rope(x + 0.5 * d, None, table, pos, sections, interleaved).double()
    down = dvdq.rope(x - 0.5 * d, None, table, pos, sections, interleaved).double()
    slope = ((up - down) * w.double()).sum()
    # each of the 600 terms is good to a few 2^-24 of |x| + |d| times |w|
    assert abs(float(slope - (grad.double() * d.double()).sum())) <= 16 * F32 * float(((x.abs() + d.abs()) * w.abs()).sum())
    back = dvdq.rope(dvdq.rope(x, None, table, pos, sections, interleaved), None, table, pos, sections, interleaved, inverse=True)
    assert float((back - x).abs().max()) <= 16 * F32 * float(x.abs().max()) * 2


def test_table_in_64_bits_far_into_a_context():
    freq, mag = dvdq.rope_frequencies(64, base=10000.0, scaling="yarn", factor=8.0, original_length=4096)
    n = 1 << 20
    table = dvdq.rope_table(n, freq, mag).cpu()
    for p in (0, 1, 4095, 4096, 999999, n - 1):
        a = torch.tensor(freq, dtype=torch.float64) * p
        ref = mag * torch.stack([a.cos(), a.sin()], -1)
        # one rounding to fp32; the angle in 64 bits is good to 2^-52 of its size
        assert float((table[p].double() - ref).abs().max()) <= 2.0 ** -24 * mag * 1.02 + 2.0 ** -51 * p


def test_one_token_of_a_long_cache_and_long_strides():
    """A token's heads that lie more than 2^31 elements apart, in a buffer as large as a long cache."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    D, far = 64, (1 << 31) + 64
    buf = torch.zeros((2 * far,), dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((3, 2, D), (D, far, 1))
    g = torch.Generator().manual_seed(9)
    q.copy_(torch.randn((3, 2, D), generator=g))
    table = dvdq.rope_table(50, dvdq.rope_frequencies(D)[0])
    pos = torch.tensor([7, 49, 0], dtype=torch.int32, device="cuda")
    want, mag = rope64(q[None], table, pos[None, :, None], (D,), False)
    dvdq.rope(q, None, table, pos, q_out=q)
    assert_close(q, want[0], 3 * F32 * mag[0], "far heads")


def test_nothing_to_do():
    table = dvdq.rope_table(4, [1.0])
    for shape in ((0, 2, 2), (0, 3, 2, 2), (2, 0, 2, 2)):
        q = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        pos = torch.empty(shape[:-2], dtype=torch.int32, device="cuda")
        assert dvdq.rope(q, None, table, pos).shape == shape


def test_refusals():
    q, k, table, pos = inputs(2, 4, 2, 1, 16, (16,), torch.bfloat16)
    pos = pos[..., 0].contiguous()
    with pytest.raises(TypeError):
        dvdq.rope(q.cpu(), None, table, pos)
    with pytest.raises(TypeError):
        dvdq.rope(q.double(), None, table, pos)
    with pytest.raises(TypeError):
        dvdq.rope(q, k.float(), table, pos)
    with pytest.raises(TypeError):
        dvdq.rope(q, k, table, pos.long())
    with pytest.raises(ValueError):
        dvdq.rope(q, k[:, :3], table, pos)
    with pytest.raises(ValueError):
        dvdq.rope(q, k, table, pos[:, :3].contiguous())
    with pytest.raises(ValueError):
        dvdq.rope(q.transpose(-1, -2).contiguous().transpose(-1, -2), k, table, pos)   # the last dimension is not dense
    with pytest.raises(ValueError):
        dvdq.rope(q, k, table, pos, q_out=torch.empty_like(q)[:, :, :1])
    with pytest.raises(dvdq.DvdqError) as e:                                           # table for more than the head
        dvdq.rope(q, k, dvdq.rope_table(97, [1.0] * 9), pos)
    assert e.value.status == 2
    with pytest.raises(dvdq.DvdqError) as e:                                           # sections are not the table's pairs
        dvdq.rope(q, k, table, torch.zeros((2, 4, 2), dtype=torch.int32, device="cuda"), (8, 6))
    assert e.value.status == 2
    with pytest.raises(dvdq.DvdqError) as e:                                           # every batch to the same place
        dvdq.rope(q, None, table, pos, q_out=torch.empty_like(q[:1]).expand(2, -1, -1, -1))
    assert e.value.status == 3


def test_streams_and_graph():
    q, k, table, pos = inputs(1, 300, 6, 6, 128, (44, 42, 42), torch.bfloat16)
    want = dvdq.rope(q, k, table, pos, (44, 42, 42), True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = dvdq.rope(q, k, table, pos, (44, 42, 42), True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = tuple(torch.zeros_like(t) for t in (q, k))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dvdq.rope(q, k, table, pos, (44, 42, 42), True, q_out=out[0], k_out=out[1])
    for i in range(4):
        q.copy_(torch.roll(q, 1, 1))
        graph.replay()
        eager = dvdq.rope(q, k, table, pos, (44, 42, 42), True)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), i
    assert math.isfinite(float(out[0].float().sum()))
