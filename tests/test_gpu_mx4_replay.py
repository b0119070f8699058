"""The layer that quantizes its rows itself, captured and on two streams, in the product's launch and through the workspace; the norm's 4-bit rows of a replay, every byte."""
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV
from test_gpu_mx4_layer import Layer, bytes_of

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
SHAPES = [(1, 528, 272), (16, 784, 528), (40, 528, 1040), (1100, 1376, 2064)]


def row_bytes(rows, K):
    """Codes and scales of a buffer, without what it is rounded up by."""
    return -(-rows // 16) * 16 * (-(-K // 256) * 256) * 17 // 32


class Rows(Layer):
    """And y2 = Q(x) W^T by the call that quantizes x."""

    def __init__(self, T, d, N, seed=0, workspace=None):
        super().__init__(T, d, N, seed)
        self.linear_work = bytes_of(ssg.ssg_mx4_linear_workspace_bytes(T, d)) if workspace is None else workspace
        self.y2, self.y3 = torch.full((T, N), float("nan"), dtype=BF, device=DEV), torch.full((T, N), float("nan"), device=DEV)

    def run(self):
        out = super().run()
        T, d, N = self.T, self.d, self.N
        ssg.ssg_mx4_linear(self.x, ssg.SSG_BF16, T, d, d, ssg.SSG_MX_FLOOR, self.q, N, self.y2, ssg.SSG_BF16, N, self.linear_work)
        ssg.ssg_mx4_linear(self.kept, ssg.SSG_F32, T, d, d, ssg.SSG_MX_CEIL, self.q, N, self.y3, ssg.SSG_F32, N, self.linear_work)
        return out + [self.y2, self.y3]

    def renew(self, seed):
        gen = torch.Generator().manual_seed(seed)
        self.x.copy_(torch.randn(self.T, self.d, generator=gen).to(BF))
        self.dy.copy_(torch.randn(self.T, self.N, generator=gen).to(BF))

    def clear(self, out):
        for t in out:
            t.fill_(0x5A if t.dtype == torch.uint8 else float("nan"))


def same(out, want, T, d):
    n = row_bytes(T, d)
    return all(torch.equal(a[:n], b[:n]) if a.dtype == torch.uint8 else torch.equal(a, b) for a, b in zip(out, want))


def captured(layer):
    layer.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.run()
    return graph, out


@pytest.mark.parametrize("T,d,N", SHAPES)
def test_replays(T, d, N):
    """New inputs, every output cleared before, eager work of another layer between: the eager bits every time."""
    m, other, ref = Rows(T, d, N, 1), Rows(T, d, N, 2), Rows(T, d, N, 1)
    graph, out = captured(m)
    for i in range(4):
        m.renew(10 + i)
        ref.renew(10 + i)
        m.clear(out)
        m.linear_work.fill_(0xA5)
        graph.replay()
        other.run()
        want = ref.run()
        torch.cuda.synchronize()
        assert same(out, want, T, d)


@pytest.mark.parametrize("T,d,N", SHAPES)
def test_two_graphs_with_one_workspace(T, d, N):
    """One after the other on a stream."""
    a = Rows(T, d, N, 1)
    b = Rows(T, d, N, 2, a.linear_work)
    b.work, b.work_norm = a.work, a.work_norm
    ra, rb = Rows(T, d, N, 1), Rows(T, d, N, 2)
    graphs = captured(a), captured(b)
    for i in range(3):
        for m, r in ((a, ra), (b, rb)):
            m.renew(20 + i)
            r.renew(20 + i)
        for graph, out in graphs:
            a.clear(out)
        for graph, _ in graphs if i % 2 == 0 else graphs[::-1]:
            graph.replay()
        want = ra.run(), rb.run()
        torch.cuda.synchronize()
        assert all(same(out, w, T, d) for (_, out), w in zip(graphs, want))


@pytest.mark.parametrize("T,d,N", [(3, 2736, 2064), (300, 1040, 2064)])
def test_two_streams(T, d, N):
    layers, refs = [Rows(T, d, N, s) for s in (1, 2)], [Rows(T, d, N, s) for s in (1, 2)]
    want = [[t.clone() for t in r.run()] for r in refs]
    torch.cuda.synchronize()
    outs, streams = [None, None], [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i] = layers[i].run()
    torch.cuda.synchronize()
    assert all(same(out, w, T, d) for out, w in zip(outs, want))


def test_both_ways_of_quantizing_are_reached():
    def tags(T, d, N):
        m = Rows(T, d, N)
        ssg.ssg_profile_select(-1)
        ssg.ssg_profile_enable(4)
        try:
            ssg.ssg_mx4_linear(m.x, ssg.SSG_BF16, T, d, d, 0, m.q, N, m.y2, ssg.SSG_BF16, N, m.linear_work)
            return ssg.ssg_profile_read(4)[1]
        finally:
            ssg.ssg_profile_enable(0)

    assert [tags(*s) for s in SHAPES] == [[56], [56], [55, 56], [55, 56]]
