"""Calls on another stream than the current one: what they allocate for themselves, and what the caller drops, is not handed out again while
their kernels are still to run."""
import types

import pytest
import torch

import paper_2505_18663_amd as dvdq

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    dvdq.lib()
    assert dvdq._marshal.__file__ == dvdq._MARSHAL_PATH
    if request.param == "python":
        monkeypatch.setattr(dvdq, "_marshal", dvdq._Handback)
    return request.param


def calls():
    """name -> (call(inputs, stream) -> outputs, inputs, bytes of scratch)"""
    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s, k=1.0: (k * torch.randn(s, generator=g, device="cuda")).to(torch.bfloat16)   # noqa: E731
    out = {}
    for name, (M, N, K) in {"parts of K": (512, 640, 4096), "copied rows": (9000, 3000, 203)}.items():
        w = r(N, K, k=K ** -0.5)
        out[name] = (lambda x, st, w=w: (dvdq.linear(x, w, act=dvdq.ACT_SILU, stream=st),), [r(M, K) for _ in range(2)], dvdq.linear_workspace_bytes(M, N, K))
    out["three launches"] = (lambda x, st: (dvdq.group_norm(x, 8, stream=st),), [r(1, 60000, 64) for _ in range(2)], dvdq.group_norm_workspace_bytes(1, 60000, 64, 8))
    out["one launch"] = (lambda x, st: (dvdq.group_norm(x, 8, stream=st),), [r(1, 400, 64) for _ in range(2)], dvdq.group_norm_workspace_bytes(1, 400, 64, 8))
    pos = torch.arange(300, dtype=torch.int32, device="cuda")
    table = dvdq.rope_table(300, dvdq.rope_frequencies(64)[0])
    out["rope"] = (lambda x, st: dvdq.rope(x[:, :4], x[:, 4:], table, pos, stream=st), [r(300, 6, 64) for _ in range(2)], 0)
    return out


def test_what_is_dropped_is_not_handed_out(path):
    for name, (call, inputs, scratch) in calls().items():
        assert scratch > 0 or name == "rope"
        want = [call(x, None) for x in inputs]
        sizes = [scratch] + [t.numel() * t.element_size() for t in want[0]]
        sides = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        got = []
        for x, side in zip(inputs, sides):
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)               # the calls' kernels are still to run when they return
            got.append(call(x, side))
            call(x, side)                                   # and one whose outputs are dropped at once
        others = [torch.full((n,), 201, dtype=torch.uint8, device="cuda") for n in sizes * 4 if n]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b)), name
        assert all(bool((t == 201).all()) for t in others), name


def _owner(t):
    """handle of the stream whose memory a tensor has"""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def test_new_tensors_belong_to_the_stream_of_the_call(path):
    side, current = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    for name, (call, inputs, _) in calls().items():
        torch.cuda.synchronize()
        for stream, owner in ((side, side), (types.SimpleNamespace(cuda_stream=side.cuda_stream), side), (None, current), (current, current)):
            for t in call(inputs[0], stream):
                assert _owner(t) == owner.cuda_stream, name
        with torch.cuda.stream(side):
            for stream, owner in ((None, side), (side, side), (current, current)):
                for t in call(inputs[0], stream):
                    assert _owner(t) == owner.cuda_stream, name
        torch.cuda.synchronize()
    assert torch.cuda.current_stream() == current
    table = dvdq.rope_table(64, dvdq.rope_frequencies(32)[0], stream=side)
    assert _owner(table) == side.cuda_stream
    side.synchronize()
    assert torch.equal(table, dvdq.rope_table(64, dvdq.rope_frequencies(32)[0]))


def test_in_a_graph_on_a_forked_stream(path):
    """A capture that forks to another stream: scratch and outputs are the graph's, replays give the eager result."""
    call, inputs, _ = calls()["parts of K"]
    x = inputs[0]
    call(x, None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        y, = call(x, side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        x.copy_(torch.roll(x, 1, 0))
        graph.replay()
        eager, = call(x, None)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i
