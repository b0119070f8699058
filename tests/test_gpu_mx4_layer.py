"""Norm, quantized rows and products together, as a pre-norm linear layer runs them: forward and backward, eager, captured and on two streams."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, f32
from oracle import mx4, norm

pytestmark = pytest.mark.gpu
EPS = 1e-5


def bytes_of(n):
    return torch.full((max(n, 256),), 0xA5, dtype=torch.uint8, device=DEV)


class Layer:
    """x, residual -> residual_out = x + residual; y = Q(norm(residual_out)) W^T, all buffers its own."""

    def __init__(self, T, d, N, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.T, self.d, self.N = T, d, N
        self.x, self.r = (torch.randn(T, d, generator=gen).to(torch.bfloat16).to(DEV), torch.randn(T, d, generator=gen).to(DEV))
        self.w = (1 + 0.1 * torch.randn(d, generator=gen)).to(torch.bfloat16).to(DEV)
        self.W = (torch.randn(N, d, generator=gen) * d ** -0.5).to(torch.bfloat16).to(DEV)
        self.dy, self.ds = (torch.randn(T, N, generator=gen).to(torch.bfloat16).to(DEV), torch.randn(T, d, generator=gen).to(DEV))
        self.q, self.qt, self.rows = bytes_of(ssg.ssg_mx4_bytes(N, d)), bytes_of(ssg.ssg_mx4_bytes(d, N)), bytes_of(ssg.ssg_mx4_bytes(T, d))
        self.desc = ssg.make_rmsnorm_desc(T, d, EPS, residual=1, r_dtype=ssg.SSG_F32, y_format=ssg.SSG_NORM_MX4)
        self.plain = ssg.make_rmsnorm_desc(T, d, EPS, x_dtype=ssg.SSG_F32, y_format=ssg.SSG_NORM_F32)
        self.work, self.work_norm = bytes_of(ssg.ssg_mx4_linear_bwd_workspace_bytes(T, N, d)), bytes_of(ssg.ssg_rmsnorm_bwd_workspace_bytes(self.desc))
        new = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
        self.kept, self.rstd, self.h, self.y, self.dh, self.dW, self.dr, self.dw = (new(T, d), new(T), new(T, d), new(T, N), new(T, d), new(N, d), new(T, d), new(d))
        self.dx = torch.full((T, d), float("nan"), dtype=torch.bfloat16, device=DEV)

    def run(self):
        T, d, N = self.T, self.d, self.N
        ssg.ssg_mx4_quantize(self.W, ssg.SSG_BF16, N, d, d, 0, 0, self.q)
        ssg.ssg_mx4_quantize(self.W, ssg.SSG_BF16, d, N, d, 1, 0, self.qt)
        ssg.ssg_rmsnorm_fwd(self.desc, self.x, self.r, self.w, self.kept, self.rows, None, None, self.rstd)
        ssg.ssg_mx4_gemm(self.rows, T, self.q, N, d, self.y, ssg.SSG_F32, N)
        ssg.ssg_rmsnorm_fwd(self.plain, self.kept, None, self.w, None, self.h, None, None, None)     # what the weights' gradient reads
        ssg.ssg_mx4_linear_bwd(self.dy, ssg.SSG_BF16, N, self.h, ssg.SSG_F32, d, T, N, d, 0, self.qt, self.dh, ssg.SSG_F32, d, self.dW, ssg.SSG_F32, d, self.work)
        ssg.ssg_rmsnorm_bwd(self.desc, self.dh, ssg.SSG_F32, d, self.kept, self.rstd, self.w, self.ds, self.dx, self.dr, self.dw, self.work_norm)
        return [self.kept, self.rstd, self.rows, self.y, self.dh, self.dW, self.dx, self.dr, self.dw]


@pytest.mark.parametrize("T,d,N", [(1, 272, 528), (5, 1040, 272), (75, 528, 1040), (300, 2736, 1040), (1100, 1376, 2064)])
def test_layer(T, d, N):
    """Every stage against the oracle, from what the stage before left."""
    m = Layer(T, d, N)
    m.run()
    u = 2.0 ** -23
    s, g, rstd = f32(m.kept), f32(m.w), f32(m.rstd)
    assert np.array_equal(s, f32(m.x) + f32(m.r))
    y32 = norm.quantized_rows(s, rstd, g)
    a, w = mx4.values(*mx4.quantize(y32)), mx4.values(*mx4.quantize(f32(m.W)))
    # sums of d, N, T terms in fp32, each addition off by at most 2^-23 of a partial sum
    assert (np.abs(f32(m.y) - a @ w.T) <= d * u * (np.abs(a) @ np.abs(w).T)).all()
    h = f32(m.h)
    assert (np.abs(h - y32) <= 64 * u * np.abs(y32)).all()
    dy = f32(m.dy)
    dyr, dyc, hc, wt = (mx4.values(*mx4.quantize(v)) for v in (dy, dy.T, h.T, f32(m.W).T))
    assert (np.abs(f32(m.dh) - dyr @ wt.T) <= N * u * (np.abs(dyr) @ np.abs(wt).T)).all()
    assert (np.abs(f32(m.dW) - dyc @ hc.T) <= T * u * (np.abs(dyc) @ np.abs(hc).T)).all()
    ds, dw = norm.backward(f32(m.dh), s, rstd, g)
    n = np.abs(s.astype(np.float64) * rstd[:, None])
    b = np.abs(f32(m.dh).astype(np.float64) * g)
    off = rstd[:, None] * (3 * b + 64 * n * (b * n).mean(-1, keepdims=True)) * u
    assert (np.abs(f32(m.dr) - (ds + f32(m.ds))) <= off + u * np.abs(ds + f32(m.ds))).all()
    assert (np.abs(f32(m.dw) - dw) <= (T + 2) * u * (np.abs(f32(m.dh).astype(np.float64)) * n).sum(0)).all()
    assert torch.equal(m.dx, m.dr.to(torch.bfloat16))


def test_norm_feeds_the_8_bit_products():
    T, d, N = 64, 528, 272
    gen = torch.Generator().manual_seed(3)
    x, w = torch.randn(T, d, generator=gen).to(torch.bfloat16).to(DEV), torch.ones(d, dtype=torch.bfloat16, device=DEV)
    W = (torch.randn(N, d, generator=gen) * d ** -0.5).to(torch.bfloat16).to(DEV)
    y, want = torch.empty(T, N, device=DEV), torch.empty(T, N, device=DEV)
    # int8 rows: the same bits as the norm in fp32 and the linear layer that quantizes it
    h, rstd = torch.empty(T, d, device=DEV), torch.empty(T, device=DEV)
    ssg.ssg_rmsnorm_fwd(ssg.make_rmsnorm_desc(T, d, EPS, y_format=ssg.SSG_NORM_F32), x, None, w, None, h, None, None, rstd)
    q, qw = bytes_of(ssg.ssg_i8_bytes(T, d)), bytes_of(ssg.ssg_i8_bytes(N, d))
    ssg.ssg_i8_quantize(W, ssg.SSG_BF16, N, d, d, qw)
    rstd2 = torch.empty(T, device=DEV)
    ssg.ssg_rmsnorm_fwd(ssg.make_rmsnorm_desc(T, d, EPS, y_format=ssg.SSG_NORM_I8), x, None, w, None, q, None, None, rstd2)
    ssg.ssg_i8_gemm(q, T, qw, N, d, y, ssg.SSG_F32, N)
    same = rstd == rstd2                                     # (a row's squares may be added in another order)
    ssg.ssg_i8_linear(h, ssg.SSG_F32, T, d, d, qw, N, want, ssg.SSG_F32, N, bytes_of(ssg.ssg_i8_linear_workspace_bytes(T, d)))
    assert int(same.sum()) > 0 and torch.equal(y[same], want[same])
    # E4M3 under a given scale: the codes of ssg_quantize, the range by ssg_amax of the rows' ranges
    scale, amax = torch.tensor([60.0], device=DEV), torch.empty(T, device=DEV)
    codes = torch.empty(T, d, dtype=torch.uint8, device=DEV)
    ssg.ssg_rmsnorm_fwd(ssg.make_rmsnorm_desc(T, d, EPS, y_format=ssg.SSG_NORM_E4M3), x, None, w, None, codes, scale, amax, rstd2)
    ref, top, top_ref = torch.empty_like(codes), torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    ssg.ssg_quantize(h, ssg.SSG_F32, T, d, ssg.SSG_E4M3, ssg.SSG_SCALE_GIVEN, ssg.SSG_ROUND_EXACT_DIV, ref, None, scale, None)
    ssg.ssg_amax(amax, ssg.SSG_F32, T, top)
    ssg.ssg_amax(h, ssg.SSG_F32, T * d, top_ref)
    assert torch.equal(rstd, rstd2) and torch.equal(codes, ref) and torch.equal(top, top_ref)


@pytest.mark.parametrize("T,d,N", [(1, 528, 272), (40, 528, 1040), (1100, 1376, 2064)])
def test_captured(T, d, N):
    """A graph's replays on new inputs, with eager work of another layer in between, give the eager bits every time."""
    m, other, ref = Layer(T, d, N, 1), Layer(T, d, N, 2), Layer(T, d, N, 1)
    m.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.run()
    for i in range(4):
        for layer in (m, ref):
            gen = torch.Generator().manual_seed(10 + i)
            layer.x.copy_(torch.randn(T, d, generator=gen).to(torch.bfloat16))
            layer.dy.copy_(torch.randn(T, N, generator=gen).to(torch.bfloat16))
        for t in out:
            t.zero_() if t.dtype == torch.uint8 else t.fill_(float("nan"))
        graph.replay()
        other.run()
        want = ref.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want) if a.dtype != torch.uint8)
        n = ssg.ssg_mx4_bytes(T, d) // 256 * 256
        assert torch.equal(m.rows[:n // 2], ref.rows[:n // 2])


def test_two_streams():
    """Two layers at once on streams of their own: the bits of one after the other."""
    a, b, ra, rb = Layer(300, 1040, 2064, 1), Layer(300, 1040, 2064, 2), Layer(300, 1040, 2064, 1), Layer(300, 1040, 2064, 2)
    want = [[t.clone() for t in ra.run()], [t.clone() for t in rb.run()]]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for layer, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                layer.run()
    torch.cuda.synchronize()
    for layer, w in zip((a, b), want):
        got = [layer.kept, layer.rstd, layer.rows, layer.y, layer.dh, layer.dW, layer.dx, layer.dr, layer.dw]
        assert all(torch.equal(x, y) for x, y in zip(got, w))
