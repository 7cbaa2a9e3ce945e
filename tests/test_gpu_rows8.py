"""Root-mean-square norm, the norm with 8-bit codes, and rows to 8 bits, against the formulas in 64 bits."""
import pytest
import torch

import paper_2505_18663_amd as dvdq
from plain64 import act64, assert_close
from plain8 import check_codes, norm64

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# one element to long rows: each width of the kernels' pieces, one more and one less, rows that need a workgroup and rows that are read again
WIDTHS = [1, 3, 8, 31, 64, 65, 80, 127, 128, 136, 255, 257, 512, 513, 1024, 1533, 1536, 2047, 4096, 4104, 5120, 8192, 8200, 13824, 16384, 16391, 32768, 40001]


def tensor(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows_for(C):
    return 5 if C > 4096 else 67 if C > 300 else 301


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_norm(dtype, C):
    g, M = gen(C), rows_for(C)
    x, w, r = tensor(g, M, C, dtype=dtype, scale=3.0), tensor(g, C, dtype=dtype), tensor(g, M, C, dtype=dtype)
    for weight, residual, eps in ((w, r, 1e-6), (None, None, 1e-5), (w, None, 0.0), (None, r, 1e-2)):
        z, root, h, err = norm64(x, weight, residual, eps)
        what = f"{dtype} C={C} weight={weight is not None} residual={residual is not None}"
        y = dvdq.rms_norm(x, weight, residual=residual, eps=eps)
        if residual is not None:
            y, h_got = y
            assert torch.equal(h_got.cpu(), h), what
        ref = z / root
        assert_close(y, ref, err * ref.abs(), what)
        codes, scale, sums, *more = dvdq.rms_norm_quant(x, weight, residual=residual, eps=eps, want_rowsum=True)
        assert len(more) == (residual is not None) and (not more or torch.equal(more[0].cpu(), h)), what
        check_codes(codes, scale, z, 1 / root, err, what, rowsum=sums)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_quant(dtype, C):
    g, M = gen(C + 1), rows_for(C)
    both = tensor(g, M, 2 * C + 3, dtype=dtype, scale=2.0)
    x, up = both[:, :C], both[:, C + 1:2 * C + 1]               # (views that begin at any element)
    for act in (dvdq.ACT_NONE, dvdq.ACT_SILU, dvdq.ACT_GELU_TANH, dvdq.ACT_GELU):
        for second in (None, up):
            what = f"{dtype} C={C} act={act} up={second is not None}"
            z = act64(x.cpu().double(), act)
            if second is not None:
                z = z * second.cpu().double()
            codes, scale, sums = dvdq.quant8(x, up=second, act=act, want_rowsum=True)
            # (act64 of silu and tanh GELU and erfc are good to 2^-50 of the value)
            check_codes(codes, scale, z, 1.0, 0.0, what, loose=act != 0, rowsum=sums)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 255, 257, 4099, 40000])
def test_any_number_of_rows(M):
    g = gen(M)
    for C in (96, 640):
        x, r, w = tensor(g, M, C, dtype=torch.bfloat16), tensor(g, M, C, dtype=torch.bfloat16), tensor(g, C, dtype=torch.bfloat16)
        z, root, h, err = norm64(x, w, r)
        y, h_got = dvdq.rms_norm(x, w, residual=r)
        assert torch.equal(h_got.cpu(), h)
        assert_close(y, z / root, err * (z / root).abs(), f"{M} x {C}")
        codes, scale, _ = dvdq.rms_norm_quant(x, w, residual=r)
        check_codes(codes, scale, z, 1 / root, err, f"{M} x {C}")
        codes, scale = dvdq.quant8(x, up=r)
        check_codes(codes, scale, x.cpu().double() * r.cpu().double(), 1.0, 0.0, f"{M} x {C}")


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_go_to_the_even_code(dtype):
    half = torch.arange(-126, 127, dtype=torch.float64) + 0.5
    x = torch.cat([half, torch.tensor([127.0])])[None].to(DEV).to(dtype)     # 127 z / max|z| = z, all of them ties
    codes, scale = dvdq.quant8(x)
    assert torch.equal(codes.cpu().double(), torch.round(x.cpu().double())) and float(scale) == 1.0
    codes, scale, h = dvdq.rms_norm_quant(x, torch.full((254,), 0.5, device=DEV, dtype=dtype), residual=torch.zeros_like(x))
    assert torch.equal(codes.cpu().double(), torch.round(x.cpu().double()))
    # 254 z an odd multiple of the maximum, which no code's step divides
    x = torch.tensor([[254.0, 1.0, 3.0, 5.0, 127.0, -129.0]], device=DEV, dtype=dtype)
    assert dvdq.quant8(x)[0].tolist() == [[127, 0, 2, 2, 64, -64]]


def test_values_a_hair_from_a_border():
    """Products that differ from a tie in digits fp32 does not hold."""
    a = torch.tensor([1 + 2.0 ** -23, 1 - 2.0 ** -24, 1.0], dtype=torch.float32)
    x = torch.stack([torch.cat([torch.tensor([254.0]), v.repeat(8) * torch.tensor([1., 3, 5, 7, 33, 65, 129, 251])]) for v in a]).to(DEV)
    up = torch.stack([torch.cat([torch.tensor([1.0]), w.repeat(8)]) for w in (a[1], a[0], a[2])]).to(DEV)
    codes, scale = dvdq.quant8(x, up=up)
    check_codes(codes, scale, x.cpu().double() * up.cpu().double(), 1.0, 0.0, "hair")


@pytest.mark.parametrize("C", [30, 250, 1533, 2048, 5120, 9001, 13824, 16384, 40001])
def test_rows_full_of_values_next_to_borders(C):
    """Every value within a few units of its last digit of the border between two codes, with and without a second factor, behind a norm's weight and behind
    each activation: the codes of 64-bit arithmetic all the same."""
    g = gen(C)
    rows = 6
    k = torch.randint(0, 127, (rows, C), generator=g, device=DEV).double() + 0.5
    sign = torch.randint(0, 2, (rows, C), generator=g, device=DEV) * 2.0 - 1
    off = 1 + torch.randint(-3, 4, (rows, C), generator=g, device=DEV) * 2.0 ** -23
    x = (k * sign * off).float()
    x[:, C // 3] = 127.0
    check_codes(*dvdq.quant8(x), x.cpu().double(), 1.0, 0.0, f"{C}")
    second = torch.exp(0.3 * tensor(g, rows, C))
    y = (x.double() / second.double()).float()                                # the product with `second` is x again, to 24 digits
    y[:, C // 3] = 127.5 / second[:, C // 3]
    check_codes(*dvdq.quant8(y, up=second), y.cpu().double() * second.cpu().double(), 1.0, 0.0, f"{C} up")
    w = second[0].contiguous()
    z, root, _, err = norm64(x / w, w)
    check_codes(*dvdq.rms_norm_quant(x / w, w), z, 1 / root, err, f"{C} norm")
    for act in (dvdq.ACT_SILU, dvdq.ACT_GELU_TANH, dvdq.ACT_GELU):
        a = tensor(g, rows, C, scale=2.0)
        a[:, C // 3] = 9.0
        up = (k * sign / act64(a.double(), act)).float()
        up[:, C // 3] = 127.0 / 9.0
        z = act64(a.cpu().double(), act) * up.cpu().double()
        keep = z.abs() <= z[:, C // 3].abs()[:, None]                         # (a value just above would be the largest)
        z, up = torch.where(keep, z, 0.0 * z), torch.where(keep.to(DEV), up, 0.0 * up)
        check_codes(*dvdq.quant8(a, up=up, act=act), z, 1.0, 0.0, f"{C} act {act}", loose=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", [40, 700, 9000, 40000])
def test_rows_of_zeros_nans_and_infinities(dtype, C):
    g = gen(7)
    x, w = tensor(g, 6, C, dtype=dtype), tensor(g, C, dtype=dtype)
    x[1] = 0
    x[2, C - 1] = float("nan")
    x[3, 0] = float("inf")
    x[4, C // 2] = -float("inf")
    bad = torch.tensor([False, False, True, True, True, False])
    for codes, scale, sums in (dvdq.quant8(x, want_rowsum=True), dvdq.quant8(x, up=x, act=dvdq.ACT_GELU, want_rowsum=True), dvdq.rms_norm_quant(x, w, want_rowsum=True)):
        assert torch.equal(scale.isnan().cpu()[bad], torch.ones(3, dtype=torch.bool)) and not scale.isnan().cpu()[~bad].any()
        assert not codes[bad.to(DEV)].any() and not codes[1].any() and float(scale[1]) == 0.0
        assert torch.equal(sums.cpu().long(), codes.cpu().long().sum(-1)) and codes[0].any() and codes[5].any()
    y = dvdq.rms_norm(x, w)
    assert not y[1].any() and y[2].isnan().all() and y[3, 0].isnan() and not y[3, 1:].any()
    assert dvdq.rms_norm(x, None, eps=0.0)[1].isnan().all()                  # 0 / 0


@pytest.mark.parametrize("act", [dvdq.ACT_SILU, dvdq.ACT_GELU_TANH, dvdq.ACT_GELU])
@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_the_largest_values_in_front_of_an_activation(dtype, act):
    g = gen(12)
    x, big = tensor(g, 4, 300, dtype=dtype), torch.finfo(dtype).max
    x[0, 7], x[1, 8], x[2, 9], x[3, 10] = float("inf"), -float("inf"), -big, big
    codes, scale = dvdq.quant8(x, act=act)
    assert scale[:2].isnan().all() and not codes[:2].any()
    assert torch.isfinite(scale[2:]).all() and int(codes[2, 9]) == 0 and codes[2].any() and int(codes[3, 10]) == 127 and int(codes[3].count_nonzero()) == 1


@pytest.mark.parametrize("dtype", TYPES)
def test_small_and_large_values(dtype):
    """Products that fp32 holds with few digits, and rows whose largest value is far above the others."""
    g = gen(3)
    x = tensor(g, 8, 300, dtype=dtype)
    small = 2.0 ** -14 if dtype == torch.float16 else 2.0 ** -70
    for s in (small, 1.0, 2.0 ** 8):
        a, b = (x.float() * s).to(dtype), (tensor(g, 8, 300) * s).to(dtype)
        a[:, 5] *= 16
        z = a.cpu().double() * b.cpu().double()
        codes, scale = dvdq.quant8(a, up=b)
        check_codes(codes, scale, z, 1.0, 0.0, f"{dtype} {s}")


def test_deep_in_an_activations_tail():
    """Rows whose values all lie where the activation falls like an exponential."""
    g = gen(4)
    for act, at in ((dvdq.ACT_SILU, -30.0), (dvdq.ACT_GELU_TANH, -4.5), (dvdq.ACT_GELU, -5.5)):
        x = at + tensor(g, 40, 500, scale=0.5)
        z = act64(x.cpu().double(), act)
        codes, scale = dvdq.quant8(x, act=act)
        check_codes(codes, scale, z, 1.0, 2.0 ** -24, f"act {act}", loose=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_views_in_place_and_given_outputs(dtype):
    g = gen(5)
    T, H, D = 37, 5, 96
    qkv = tensor(g, T, 3 * H, D, dtype=dtype)
    w = tensor(g, D + 1, dtype=dtype)[1:]
    q, keep = qkv[:, H:2 * H], qkv.clone()
    z, root, _, err = norm64(q.contiguous(), w)
    y = dvdq.rms_norm(q, w, y=q)                                              # heads in place, inside the projection's output
    assert y is q
    assert_close(q, z / root, err * (z / root).abs(), "heads")
    keep[:, H:2 * H] = q
    assert torch.equal(qkv, keep)
    # [B, heads, T, D] from [B, T, heads, D] is no sequence of rows; [B, T, D] views with a batch stride are
    x = tensor(g, 4, 9, 2, 130, dtype=dtype)[:, :, 1, 1:129]
    r = tensor(g, 9, 4, 128, dtype=dtype).transpose(0, 1)
    z, root, h, err = norm64(x.contiguous(), None, r.contiguous())
    out = torch.zeros((4, 9, 140), dtype=dtype, device=DEV)
    codes = torch.full((4, 9, 131), 99, dtype=torch.int8, device=DEV)
    y, h_got = dvdq.rms_norm(x, residual=r, h=r, y=out[..., 2:130])
    assert h_got is r and torch.equal(r.cpu(), h)
    assert_close(y, z / root, err * (z / root).abs(), "views")
    assert not out[..., :2].any() and not out[..., 130:].any()
    got = dvdq.rms_norm_quant(r, codes=codes[..., 1:129], x_scale=torch.empty((4, 9), device=DEV))
    check_codes(got[0], got[1], z, 1 / root, err, "views")
    assert (codes[..., 0] == 99).all() and (codes[..., 129:] == 99).all()
    with pytest.raises(ValueError):
        dvdq.rms_norm(tensor(g, 2, 3, 4, 8).transpose(1, 2))
    # four dimensions that lie in order
    x = tensor(g, 2, 3, 5, 64, dtype=dtype)
    assert torch.equal(dvdq.rms_norm(x), dvdq.rms_norm(x.view(-1, 64)).view(x.shape))
    assert torch.equal(dvdq.rms_norm_quant(x)[1], dvdq.rms_norm_quant(x.view(-1, 64))[1].view(2, 3, 5))
    # rows broadcast over a batch
    one = tensor(g, 1, 64, dtype=dtype)
    assert torch.equal(dvdq.rms_norm(one.expand(7, 64)), dvdq.rms_norm(one).expand(7, 64))


def test_results_do_not_change():
    g = gen(6)
    x = tensor(g, 3000, 1536, dtype=torch.bfloat16)
    first = (dvdq.rms_norm(x), *dvdq.rms_norm_quant(x), *dvdq.quant8(x, act=dvdq.ACT_GELU))
    for _ in range(3):
        for a, b in zip(first, (dvdq.rms_norm(x), *dvdq.rms_norm_quant(x), *dvdq.quant8(x, act=dvdq.ACT_GELU))):
            assert torch.equal(a, b)
    # a row's result is its own: not the number of rows' or its place
    assert torch.equal(dvdq.rms_norm(x[7:8])[0], first[0][7]) and torch.equal(dvdq.rms_norm_quant(x[7:8])[0][0], first[1][7])


def test_nothing_to_do():
    for shape in ((0, 64), (0, 3, 64), (3, 0, 64)):
        x = torch.empty(shape, device=DEV)
        assert dvdq.rms_norm(x).shape == shape and dvdq.rms_norm_quant(x)[1].shape == shape[:-1]
    assert dvdq.quant8(torch.empty((0, 5), device=DEV))[0].shape == (0, 5)


def test_rows_beyond_32_bits_of_elements():
    """Offsets of more than 2^31 elements, and of more than 2^32 bytes in the codes."""
    C, M = 16384, 262200
    x = torch.empty((M, C), dtype=torch.bfloat16, device=DEV)
    x.view(-1).view(torch.int16).fill_(0x3F80)                                # ones
    g = gen(8)
    for at in (0, 131071, 131072, 262143, 262199):
        x[at] = tensor(g, C, dtype=torch.bfloat16)
    codes, scale = dvdq.quant8(x)
    y = dvdq.rms_norm(x, y=x)
    for at in (0, 131071, 131072, 262143, 262199):
        g = gen(8) if at == 0 else g
        row = tensor(g, C, dtype=torch.bfloat16)[None]
        a, b = dvdq.quant8(row)
        assert torch.equal(codes[at], a[0]) and scale[at] == b[0] and torch.equal(y[at], dvdq.rms_norm(row)[0])
    assert int(codes[262144, 5]) == 127 and float(y[262144, 5]) == 1.0
