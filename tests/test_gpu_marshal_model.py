"""The operators around the quantized layer through the native module: the same outputs as through the Python functions' own checks
and ctypes, given outputs, workspaces and streams used, the same refusals."""
import types

import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu


@pytest.fixture
def both(monkeypatch):
    """call(f) -> (f() through the native module, f() without it)"""
    dvdq.lib()
    native = dvdq._marshal
    assert dvdq._marshal.__file__ == dvdq._MARSHAL_PATH   # (else both would go through ctypes)
    taken = []
    watch = types.SimpleNamespace(**{f: (lambda *a, f=f: taken.append(getattr(native, f)(*a)) or taken[-1]) for f in ("rope", "linear", "group_norm")})

    def call(f, plain=True):
        """plain: whether the native module is expected to take the call"""
        monkeypatch.setattr(dvdq, "_marshal", watch)
        first = f()
        assert (taken.pop() is not None) == plain
        monkeypatch.setattr(dvdq, "_marshal", dvdq._Handback)
        return first, f()
    return call


def _equal(pair):
    a, b = pair
    for x, y in zip(a if isinstance(a, tuple) else (a,), b if isinstance(b, tuple) else (b,)):
        assert x.shape == y.shape and x.stride() == y.stride() and x.dtype == y.dtype and torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_rope(dtype, both):
    qkv = torch.randn((2, 9, 12, 32), device="cuda").to(dtype)
    q, k = qkv[:, :, :4], qkv[:, :, 4:8]
    table = dvdq.rope_table(40, dvdq.rope_frequencies((8, 12, 12))[0])
    pos = torch.randint(0, 40, (2, 9, 3), dtype=torch.int32, device="cuda")
    for il in (False, True):
        for inv in (False, True):
            _equal(both(lambda: dvdq.rope(q, k, table, pos, (8, 12, 12), il, inv)))
            _equal(both(lambda: dvdq.rope(q, None, table, pos[0], [8, 12, 12], il, inv)))
            _equal(both(lambda: dvdq.rope(q, k, table, pos[..., 0].contiguous(), None, il, inv)))
            _equal(both(lambda: dvdq.rope(q[0], k[0], table, pos[0, :, 1].contiguous(), None, il, inv)))
    out = torch.empty((2, 4, 9, 32), dtype=dtype, device="cuda")
    a, b = both(lambda: dvdq.rope(q, None, table, pos, (8, 12, 12), q_out=out.transpose(1, 2)))
    assert a.data_ptr() == b.data_ptr() == out.data_ptr()
    _equal(both(lambda: dvdq.rope(q.transpose(1, 2).contiguous().transpose(1, 2), None, table, pos[..., 0].contiguous())))
    assert both(lambda: dvdq.rope(q[:0], None, table, pos[:0, :, 0].contiguous()), plain=False)[0].shape == (0, 9, 4, 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_linear(dtype, both):
    x, w = torch.randn((10, 70), device="cuda").to(dtype)[:, 3:67], torch.randn((24, 64), device="cuda").to(dtype)
    b, g, r = torch.randn((24,), device="cuda").to(dtype), torch.randn((5, 24), device="cuda").to(dtype), torch.randn((10, 30), device="cuda").to(dtype)[:, 2:26]
    _equal(both(lambda: dvdq.linear(x, w)))
    _equal(both(lambda: dvdq.linear(x, w, b, dvdq.ACT_GELU, g, r)))
    _equal(both(lambda: dvdq.linear(x, w, gate=g[0])))
    y, ws = torch.empty((10, 24), dtype=dtype, device="cuda"), torch.empty((1 << 20,), dtype=torch.uint8, device="cuda")
    a, c = both(lambda: dvdq.linear(x, w, b, y=y, workspace=ws))
    assert a is y and c is y
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a, c = both(lambda: dvdq.linear(x, w, b, stream=side))
    side.synchronize()
    assert torch.equal(a, c) and torch.equal(a, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_group_norm(dtype, both):
    x = torch.randn((3, 40, 50), device="cuda").to(dtype)[:, :, 1:49]
    w, b = torch.randn((48,), device="cuda").to(dtype), torch.randn((48,), device="cuda").to(dtype)
    a, c = both(lambda: dvdq.group_norm(x, 6, w, b, act=dvdq.ACT_SILU))
    assert torch.equal(a, c)
    a, c = both(lambda: dvdq.group_norm(x.view(3, 40, 48).unflatten(1, (5, 8)), 6, w, b, eps=1e-6), plain=False)
    assert torch.equal(a, c)
    y, ws = torch.empty((3, 40, 48), dtype=dtype, device="cuda"), torch.empty((1 << 20,), dtype=torch.uint8, device="cuda")
    a, c = both(lambda: dvdq.group_norm(x, 6, None, None, 1e-3, dvdq.ACT_NONE, y, ws))
    assert a is y and c is y


def test_the_same_refusals(both):
    x, w = torch.randn((4, 16), device="cuda").bfloat16(), torch.randn((8, 16), device="cuda").bfloat16()
    table, pos = dvdq.rope_table(4, [1.0, 0.5]), torch.zeros((4,), dtype=torch.int32, device="cuda")
    q = x.view(4, 2, 8)
    for f, error in ((lambda: dvdq.linear(x, w.half()), TypeError), (lambda: dvdq.linear(x, w[:, :8]), ValueError), (lambda: dvdq.linear(x, w, act=9), dvdq.DvdqError),
                     (lambda: dvdq.linear(x.float(), w.float()), TypeError), (lambda: dvdq.group_norm(x[None], 3), dvdq.DvdqError),
                     (lambda: dvdq.group_norm(x[None].double(), 2), TypeError), (lambda: dvdq.group_norm(x[None], 2, w[0, :8]), ValueError),
                     (lambda: dvdq.rope(q, q[:3], table, pos), ValueError), (lambda: dvdq.rope(q, None, table, pos[:3]), ValueError),
                     (lambda: dvdq.rope(q, None, table, pos, (2, 2)), ValueError), (lambda: dvdq.rope(q, None, dvdq.rope_table(4, [1.0] * 5), pos), dvdq.DvdqError)):
        for path in (dvdq._marshal, dvdq._Handback):
            old = dvdq._marshal
            try:
                dvdq._marshal = path
                with pytest.raises(error):
                    f()
            finally:
                dvdq._marshal = old
