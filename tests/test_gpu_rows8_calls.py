"""The norms and layers in 8 bits through the native module and through Python and ctypes; refusals; streams; captured and replayed."""
import types

import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAMES = ("rms_norm", "rms_norm_quant", "quant8", "linear8")


@pytest.fixture
def both(monkeypatch):
    """call(f) -> (f() through the native module, f() without it)"""
    dvdq.lib()
    native = dvdq._marshal
    assert native.__file__ == dvdq._MARSHAL_PATH   # (else both would go through ctypes)
    taken = []
    watch = types.SimpleNamespace(**{f: (lambda *a, f=f: taken.append(getattr(native, f)(*a)) or taken[-1]) for f in NAMES})

    def call(f, plain=True):
        """plain: whether the native module is expected to take the call"""
        monkeypatch.setattr(dvdq, "_marshal", watch)
        first = f()
        assert (taken.pop() is not None) == plain
        monkeypatch.setattr(dvdq, "_marshal", dvdq._Handback)
        return first, f()
    return call


def _equal(pair):
    for x, y in zip(*(v if isinstance(v, tuple) else (v,) for v in pair)):
        assert x.shape == y.shape and x.stride() == y.stride() and x.dtype == y.dtype and torch.equal(x, y)
    assert len(pair[0]) == len(pair[1])
    return pair


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_the_same_outputs_both_ways(dtype, both):
    x, w = torch.randn((9, 5, 70), device=DEV).to(dtype)[..., 3:67], torch.randn(64, device=DEV).to(dtype)
    r = torch.randn((9, 5, 64), device=DEV).to(dtype)
    for t, u in ((x, r), (x[:, 2], r[:, 2])):
        for weight in (None, w):
            _equal(both(lambda: dvdq.rms_norm(t, weight)))
            _equal(both(lambda: dvdq.rms_norm(t, weight, residual=u, eps=1e-3)))
            for sums in (False, True):
                assert len(_equal(both(lambda: dvdq.rms_norm_quant(t, weight, want_rowsum=sums)))[0]) == 2 + sums
                assert len(_equal(both(lambda: dvdq.rms_norm_quant(t, weight, residual=u, want_rowsum=sums)))[0]) == 3 + sums
    _equal(both(lambda: dvdq.rms_norm(r.view(3, 3, 5, 64)), plain=False))
    h, y = torch.empty_like(r), torch.empty_like(r)
    a, b = both(lambda: dvdq.rms_norm(x, w, residual=r, h=h, y=y))
    assert a[0] is y and a[1] is h and b[0] is y and b[1] is h
    c, s, n = torch.empty((9, 5, 64), dtype=torch.int8, device=DEV), torch.empty((9, 5), device=DEV), torch.empty((9, 5), dtype=torch.int32, device=DEV)
    a, b = both(lambda: dvdq.rms_norm_quant(x, w, residual=r, h=h, codes=c, x_scale=s, code_rowsum=n))
    assert all(p is q for p, q in zip(a, (c, s, n, h))) and all(p is q for p, q in zip(b, (c, s, n, h)))
    for up in (None, r[:, 2]):
        for act in range(4):
            _equal(both(lambda: dvdq.quant8(x[:, 2], up=up, act=act)))
            _equal(both(lambda: dvdq.quant8(x[:, 2], up, act, want_rowsum=True)))
    codes, scale = dvdq.quant8(x[:, 2])
    wc, ws = dvdq.quant8(torch.randn((24, 64), device=DEV))
    bias, gate, res = torch.randn(24, device=DEV).to(dtype), torch.randn((3, 24), device=DEV).to(dtype), torch.randn((9, 30), device=DEV).to(dtype)[:, 2:26]
    _equal(both(lambda: (dvdq.linear8(codes, scale, wc, ws, dtype=dtype),)))
    _equal(both(lambda: (dvdq.linear8(codes, scale, wc, ws, bias, dvdq.ACT_GELU, gate, res, dtype=dtype),)))
    _equal(both(lambda: (dvdq.linear8(codes, scale, wc, ws, gate=gate[0], y=torch.empty((9, 24), dtype=dtype, device=DEV)),)))
    y, space = torch.empty((9, 24), dtype=dtype, device=DEV), torch.empty((1 << 20,), dtype=torch.uint8, device=DEV)
    a, b = both(lambda: dvdq.linear8(codes, scale, wc, ws, bias, y=y, workspace=space))
    assert a is y and b is y


def test_the_same_refusals_both_ways():
    x, w = torch.randn((4, 16), device=DEV).bfloat16(), torch.randn(16, device=DEV).bfloat16()
    c, s = dvdq.quant8(x)
    one = torch.ones(3, device=DEV)
    calls = (
        (lambda: dvdq.rms_norm(x[0]), ValueError), (lambda: dvdq.rms_norm(x.double()), TypeError), (lambda: dvdq.rms_norm(x, w[:8]), ValueError),
        (lambda: dvdq.rms_norm(x, w.float()), TypeError), (lambda: dvdq.rms_norm(x, residual=x[:3]), ValueError), (lambda: dvdq.rms_norm(x, h=x), ValueError),
        (lambda: dvdq.rms_norm(x.t()), ValueError), (lambda: dvdq.rms_norm(x, eps=-1.0), dvdq.DvdqError), (lambda: dvdq.rms_norm(x, y=x.float()), TypeError),
        (lambda: dvdq.rms_norm(x, residual=x, y=x, h=x), dvdq.DvdqError), (lambda: dvdq.rms_norm(x[:1].expand(4, 16), y=x[:1].expand(4, 16)), dvdq.DvdqError),
        (lambda: dvdq.rms_norm_quant(x, codes=c[:3]), ValueError), (lambda: dvdq.rms_norm_quant(x, codes=x), TypeError),
        (lambda: dvdq.rms_norm_quant(x, x_scale=s[:3]), ValueError), (lambda: dvdq.rms_norm_quant(x, x_scale=s.half()), TypeError),
        (lambda: dvdq.quant8(x, up=x.half()), TypeError), (lambda: dvdq.quant8(x, act=9), dvdq.DvdqError), (lambda: dvdq.quant8(x[None]), ValueError),
        (lambda: dvdq.quant8(x.long()), TypeError), (lambda: dvdq.quant8(x, codes=c.t()), ValueError),
        (lambda: dvdq.linear8(x, s, c, s), TypeError), (lambda: dvdq.linear8(c, s[:3], c, s), ValueError), (lambda: dvdq.linear8(c, s, c[:, :8], s), ValueError),
        (lambda: dvdq.linear8(c, s, c, one), ValueError), (lambda: dvdq.linear8(c, s, c, s, bias=w[:4].float()), TypeError),
        (lambda: dvdq.linear8(c, s, c, s, residual=x), ValueError), (lambda: dvdq.linear8(c, s, c, s, dtype=torch.int8), TypeError),
        (lambda: dvdq.linear8(c, s, c, s, act=7), dvdq.DvdqError), (lambda: dvdq.linear8(c, s, c, s, gate=x), ValueError),
        (lambda: dvdq.linear8(c, s, c, s, y=torch.empty((4, 5), device=DEV)), ValueError), (lambda: dvdq.linear8(c, s, c, s, workspace=x), TypeError))
    native = dvdq._marshal
    for i, (f, error) in enumerate(calls):
        for path in (native, dvdq._Handback):
            try:
                dvdq._marshal = path
                with pytest.raises(error):
                    f()
                    print("not refused:", i)
            finally:
                dvdq._marshal = native


def test_a_tensor_that_is_not_on_the_current_device_is_refused(monkeypatch):
    x = torch.randn((4, 16), device=DEV)
    c, s = dvdq.quant8(x)
    monkeypatch.setattr(dvdq, "_marshal", dvdq._Handback)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for f in (lambda: dvdq.rms_norm(x), lambda: dvdq.rms_norm_quant(x), lambda: dvdq.quant8(x), lambda: dvdq.linear8(c, s, c, s)):
        with pytest.raises(ValueError, match="current device"):
            f()


def chain(x, r, nw, weights, out):
    """The operators as a block has them, into given tensors."""
    (c1, s1), (c2, s2) = weights
    codes, scale, h = dvdq.rms_norm_quant(x, nw, residual=r)
    up = dvdq.linear8(codes, scale, c1, s1, act=dvdq.ACT_GELU_TANH)
    codes, scale = dvdq.quant8(up)
    dvdq.linear8(codes, scale, c2, s2, residual=h, y=out)
    return dvdq.rms_norm(out, nw)


def inputs(M, D, F):
    g = torch.Generator(device=DEV).manual_seed(M)
    make = lambda *s: torch.randn(s, generator=g, device=DEV)   # noqa: E731
    return make(M, D).bfloat16(), make(M, D).bfloat16(), make(D).bfloat16(), (dvdq.quant8(make(F, D)), dvdq.quant8(make(D, F)))


@pytest.mark.parametrize("M,D,F", [(1, 512, 2048), (130, 512, 2000), (700, 264, 1001)])
def test_captured_and_replayed(M, D, F):
    x, r, nw, weights = inputs(M, D, F)
    out = torch.empty((M, D), dtype=torch.bfloat16, device=DEV)
    want = []
    for seed in range(4):
        x.copy_(torch.randn((M, D), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        want.append((chain(x, r, nw, weights, out).clone(), out.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        chain(x, r, nw, weights, out)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        normed = chain(x, r, nw, weights, out)
    for seed in (0, 1, 2, 3, 1, 0):
        x.copy_(torch.randn((M, D), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(normed, want[seed][0]) and torch.equal(out, want[seed][1])
        chain(x, r, nw, weights, torch.empty_like(out))           # the program's own work between replays


def test_on_a_stream_of_its_own():
    x, r, nw, weights = inputs(300, 512, 2000)
    out = torch.empty((300, 512), dtype=torch.bfloat16, device=DEV)
    want = chain(x, r, nw, weights, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    (c1, s1), (c2, s2) = weights
    native = dvdq._marshal
    for path in (native, dvdq._Handback):
        try:
            dvdq._marshal = path
            for _ in range(5):
                codes, scale, h = dvdq.rms_norm_quant(x, nw, residual=r, stream=side)
                up = dvdq.linear8(codes, scale, c1, s1, act=dvdq.ACT_GELU_TANH, stream=side)
                codes, scale = dvdq.quant8(up, stream=side)
                y = dvdq.rms_norm(dvdq.linear8(codes, scale, c2, s2, residual=h, stream=side), nw, stream=side)
                torch.cuda.current_stream().wait_stream(side)
                assert torch.equal(y, want)
        finally:
            dvdq._marshal = native


def test_two_calls_at_once():
    x, r, nw, weights = inputs(600, 512, 2000)
    outs = [torch.empty((600, 512), dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    want = chain(x, r, nw, weights, outs[0]).clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s, o in zip(streams, outs):
        with torch.cuda.stream(s):
            got.append([chain(x, r, nw, weights, o) for _ in range(4)])
    torch.cuda.synchronize()
    for y in sum(got, []):
        assert torch.equal(y, want)
