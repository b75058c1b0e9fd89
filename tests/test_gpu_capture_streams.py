"""Captured calls on two streams that are joined by events, and calls behind a replayed graph.

A layer's first kernel reads its input before it waits for the launch before it, so inside a graph it may hang on another
kernel's node by a programmatic edge only where that is sound: not behind a contraction that releases the next launch early,
nor behind a cache or attention kernel."""
import ctypes as C

import pytest
import torch

from paper_2504_18415_b200 import hbl
from states_ref import fill, heads, make_batch

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def edges(graph):
    """(kernel, kernel, programmatic) of the graph's edges, by the files that the kernels are in."""
    L, h, n = C.CDLL("libcuda.so.1"), C.c_void_p(graph.raw_cuda_graph()), C.c_size_t(0)
    assert L.cuGraphGetEdges_v2(h, None, None, None, C.byref(n)) == 0
    ends, data = [(C.c_void_p * n.value)() for _ in range(2)], (C.c_ubyte * (8 * n.value))()       # data: from, to, type, 5 unused
    assert L.cuGraphGetEdges_v2(h, *ends, data, C.byref(n)) == 0

    def name(node):
        kind, params, text = C.c_int(), (C.c_ubyte * 256)(), C.c_char_p()
        assert L.cuGraphNodeGetType(C.c_void_p(node), C.byref(kind)) == 0
        if kind.value != 0:
            return "not a kernel"
        assert L.cuGraphKernelNodeGetParams_v2(C.c_void_p(node), params) == 0
        assert L.cuFuncGetName(C.byref(text), C.c_void_p.from_buffer(params)) == 0
        return text.value.decode()

    return [(name(a), name(b), data[8 * i + 2] == 1) for i, (a, b) in enumerate(zip(*ends))]


class Layers:
    """x -> first -> y (on one stream) -> second -> z (on another), each a call of the library."""

    def __init__(self, kind, T):
        g = gen(T)
        self.hidden, self.T = 2048, T
        self.W = [hbl.hbl_quantize_weights(torch.randn(2048, 2048, device="cuda", generator=g) * 0.02) for _ in range(2)]
        self.x = torch.randn(T, 2048, device="cuda", generator=g).bfloat16()
        self.y, self.z = torch.empty_like(self.x), torch.empty_like(self.x)
        self.ws = [hbl.new_workspace(hbl.hbl_workspace_bytes(T, 2048, 2048)) for _ in range(2)]
        self.kind, self.other = kind, torch.cuda.Stream()
        self.cache = hbl.KvCache.empty(-(-T // 64) + 8, 64, 16, 128, 4)
        fill(g, self.cache)
        self.batch, _ = make_batch(g, self.cache, [T], [T + 100])
        self.scratch = hbl.new_workspace(max(1, hbl.hbl_attention_workspace_bytes(self.cache, self.batch, 16)))

    def first(self):
        if self.kind == "attention":
            hbl.hbl_attention(self.cache, self.batch, self.x.view(self.T, 16, 128), out=self.y.view(self.T, 16, 128), workspace=self.scratch)
        else:
            hbl.hbl_forward(self.x, *self.W[0], 2048, 4, True, y=self.y, workspace=self.ws[0], path=self.kind)

    def second(self):
        hbl.hbl_forward(self.y, *self.W[1], 2048, 4, True, y=self.z, workspace=self.ws[1])

    def run(self):
        self.first()
        done = torch.cuda.Event()
        done.record()
        with torch.cuda.stream(self.other):
            self.other.wait_event(done)
            self.second()
            back = torch.cuda.Event()
            back.record()
        torch.cuda.current_stream().wait_event(back)

    def result(self):
        """With everything waited for."""
        self.first()
        torch.cuda.synchronize()
        self.second()
        torch.cuda.synchronize()
        return self.z.clone()


KINDS = [("attention", 1), ("attention", 40), ("attention", 600), (hbl.PATH_AUTO, 16), (hbl.PATH_STREAM_OVERLAP, 128), (hbl.PATH_TENSOR, 600)]


@pytest.mark.parametrize("kind,T", KINDS)
def test_a_layer_on_another_stream_waits_for_the_whole_kernel_it_follows(kind, T):
    l = Layers(kind, T)
    l.run()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        l.run()
    found = edges(graph)
    early = [e for e in found if e[2] and any(s in e[0] for s in ("hbl_attn", "hbl_gemm_stream")) and "hbl_act" in e[1]]
    assert not early and any("hbl_act" in b for _, b, _ in found)
    graph.instantiate()
    for i in range(20):
        l.x.normal_(generator=gen(i))
        l.z.fill_(7.0)
        graph.replay()
        got = l.z.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, l.result())
    assert hbl.hbl_check_status() == 0


def test_a_chain_on_one_stream_keeps_its_early_starts():
    """Calls in the back-to-back mode, captured: the next quantizer still begins beside the contraction."""
    T = 16
    g = gen(3)
    W = hbl.hbl_quantize_weights(torch.randn(2048, 2048, device="cuda", generator=g) * 0.02)
    xs = [torch.randn(T, 2048, device="cuda", generator=g).bfloat16() for _ in range(4)]
    ys = [torch.empty_like(x) for x in xs]
    ws = hbl.new_workspace(hbl.hbl_workspace_bytes(T, 2048, 2048))

    def run():
        for x, y in zip(xs, ys):
            hbl.hbl_forward(x, *W, 2048, 4, True, y=y, workspace=ws, path=hbl.PATH_STREAM_OVERLAP)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        run()
    found = edges(graph)
    assert len(found) == 7 and all(early for _, _, early in found)
    want = [y.clone() for y in ys]
    graph.instantiate()
    for y in ys:
        y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ys, want)) and hbl.hbl_check_status() == 0


@pytest.mark.parametrize("kind,T", KINDS)
def test_a_call_behind_a_replayed_graph(kind, T):
    """The graph ends in a kernel that lets the next launch begin early; the call behind the replay is not part of the graph."""
    l = Layers(kind, T)
    l.result()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l.first()
    torch.cuda.synchronize()
    for i in range(20):
        l.x.normal_(generator=gen(i))
        want = l.result()
        l.y.fill_(3.0)
        l.z.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        l.second()
        assert torch.equal(l.z, want)
    assert hbl.hbl_check_status() == 0
