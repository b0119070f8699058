"""The mixture's forward on the GPU: every stage against the oracle continued from the GPU's own stored operands, and the whole."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, bf16_ulp, f32
from oracle import i8, route

pytestmark = pytest.mark.gpu


def weights_of(rows, K, seed):
    W = torch.randn(rows, K, generator=torch.Generator().manual_seed(seed)) * K ** -0.5
    codes, scales = i8.quantize(W.numpy())
    q = torch.empty(ssg.ssg_i8_bytes(rows, K), dtype=torch.uint8, device=DEV)
    ssg.ssg_i8_quantize(W.to(DEV), ssg.SSG_F32, rows, K, K, q)
    return q, codes, scales


def read(work, ptr, count, dtype):
    at = ptr - work.data_ptr()
    return work[at:at + count * torch.empty((), dtype=dtype).element_size()].view(dtype)


class Layer:
    def __init__(self, T, E, k, d, f, y_dtype=torch.bfloat16, logits_dtype=torch.float32, seed=0, **more):
        self.T, self.E, self.k, self.d, self.f, self.y_dtype = T, E, k, d, f, y_dtype
        self.route = ssg.make_route_desc(T, E, k, logits_dtype=ssg.SSG_BF16 if logits_dtype == torch.bfloat16 else ssg.SSG_F32, **more)
        self.desc = ssg.make_moe_desc(self.route, d, f, ssg.SSG_F32 if y_dtype == torch.float32 else ssg.SSG_BF16)
        gen = torch.Generator().manual_seed(seed)
        self.x = torch.randn(T, d, generator=gen).to(torch.bfloat16).to(DEV)
        self.logits = torch.randn(T, E, generator=gen).to(logits_dtype).to(DEV)
        self.W1, self.W2, self.W3 = weights_of(E * f, d, 1), weights_of(E * f, d, 2), weights_of(E * d, f, 3)
        self.work = torch.full((ssg.ssg_moe_workspace_bytes(self.desc),), 0xC3, dtype=torch.uint8, device=DEV)

    def run(self, bias=None):
        y = torch.full((self.T, self.d), 9.0, dtype=self.y_dtype, device=DEV)
        ssg.ssg_moe_fwd(self.desc, self.x, self.logits, bias, self.W1[0], self.W2[0], self.W3[0], y, self.work)
        return y

    def check(self, y):
        v = ssg.ssg_moe_view_workspace(self.desc, self.work)
        E, k, d, f = self.E, self.k, self.d, self.f
        ids = read(self.work, v.ids, self.T * k, torch.int32).view(self.T, k).cpu().numpy()
        w = read(self.work, v.weights, self.T * k, torch.float32).view(self.T, k).cpu().numpy().astype(np.float64)
        if v.offsets is None:                                  # up to four tokens: no order of dispatch, nothing quantized is stored
            assert self.T <= 4 and v.rows == self.T * k
            live, flat = self.T * k, ids.reshape(-1)
            place = np.where(flat >= 0, np.arange(live), -1)
            rows_of = [np.nonzero(flat == e)[0] for e in range(E)]
            source, real = np.arange(live), flat >= 0
        else:
            counts, offsets, place, source = route.dispatch(ids, E, 16, v.rows)
            for name, ref, n in (("counts", counts, E), ("offsets", offsets, E + 1), ("place", place, self.T * k), ("source", source, v.rows)):
                assert np.array_equal(read(self.work, getattr(v, name), n, torch.int32).cpu().numpy(), ref), name
            live = int(offsets[-1])
            rows_of = [np.arange(offsets[e], offsets[e] + counts[e]) for e in range(E)]
            real = source[:live] >= 0

        def quantized(ptr, K, want, name):
            if ptr is None:
                return
            wide, up = -(-K // 128) * 128, -(-v.rows // 16) * 16
            codes = read(self.work, ptr, live * wide, torch.uint8).cpu().numpy()
            at = -(-up * wide // 256) * 256
            scales = read(self.work, ptr + at, live, torch.float32).cpu().numpy()
            assert np.array_equal(codes, i8.layout(want[0])) and np.array_equal(scales, want[1]), name

        x = f32(self.x)[np.maximum(source[:live], 0) // k] * real[:, None]
        xq, sx = i8.quantize(x)
        quantized(v.x_q, d, (xq, sx), "quantized x")
        h = read(self.work, v.h, live * f, torch.bfloat16).view(live, f).float().cpu().numpy()
        h[~real] = 0 if v.offsets is None else h[~real]        # (rows of no expert are not written)
        hq, sh = i8.quantize(h)
        quantized(v.h_q, f, (hq, sh), "quantized h")
        o = None if v.o is None else read(self.work, v.o, live * d, self.y_dtype).view(live, d).float().cpu().numpy()
        expected = np.zeros((live, d))
        for e, r in enumerate(rows_of):
            if not len(r):
                continue
            part = [(c[e * n:(e + 1) * n], t[e * n:(e + 1) * n]) for (_, c, t), n in ((self.W1, f), (self.W2, f), (self.W3, d))]
            u, g = (i8.matmul(xq[r], sx[r], *part[i]).astype(np.float64) for i in (0, 1))
            ref = u * g / (1 + np.exp(-g))
            # u and g are the GPU's own bits; their SwiGLU product is good to 6 ulp of binary32, then rounded to bf16
            assert (np.abs(h[r] - ref) <= bf16_ulp(ref) * (0.5 + 2.0 ** -12)).all()
            expected[r] = torch.from_numpy(i8.matmul(hq[r], sh[r], *part[2])).to(self.y_dtype).float().numpy()
            assert o is None or np.array_equal(o[r], expected[r]), f"results of expert {e}"
        p = place.reshape(self.T, k)
        terms = np.where((p >= 0)[:, :, None], w[:, :, None] * expected[np.maximum(p, 0)], 0.0) if live else np.zeros((self.T, k, d))
        ref, size = terms.sum(1), np.abs(terms).sum(1)
        tol = k * 2.0 ** -24 * size + (0.5 * bf16_ulp(ref) if self.y_dtype == torch.bfloat16 else 0.0)
        assert (np.abs(f32(y) - ref) <= tol * (1 + 2.0 ** -10)).all()


@pytest.mark.parametrize("T", [1, 3, 16, 40, 150, 700])
@pytest.mark.parametrize("E,k,d,f", [(1, 1, 64, 48), (4, 2, 128, 208), (7, 3, 272, 80), (70, 5, 96, 64)])
def test_stages(T, E, k, d, f):
    layer = Layer(T, E, k, d, f)
    layer.check(layer.run())


@pytest.mark.parametrize("T,E,k,d,f", [(1, 8, 2, 1024, 2736), (600, 3, 2, 1040, 528), (1500, 2, 2, 272, 400), (2100, 1, 1, 336, 272)])
@pytest.mark.parametrize("y_dtype", [torch.bfloat16, torch.float32])
def test_stages_larger(T, E, k, d, f, y_dtype):
    layer = Layer(T, E, k, d, f, y_dtype=y_dtype, logits_dtype=torch.bfloat16)
    layer.check(layer.run())


@pytest.mark.parametrize("up,down,T,E,k,d,f", [(256, 128, 3100, 2, 1, 528, 2064), (128, 128, 3700, 2, 1, 528, 2064), (128, 256, 3700, 2, 1, 4096, 528), (128, 128, 2500, 5, 2, 400, 1552),
                                               (128, 128, 900, 6, 2, 1040, 784), (0, 0, 90, 40, 5, 272, 336)])
def test_stages_in_every_kernel(up, down, T, E, k, d, f):
    assert ssg.ssg_i8_gemm_plan(T * k, f, d, E, 1).tile == up and ssg.ssg_i8_gemm_plan(T * k, d, f, E, 0).tile == down
    layer = Layer(T, E, k, d, f)
    layer.logits[:, 0] += 0.7                                   # rows of every remainder, one expert with more
    layer.check(layer.run())


def test_a_token_that_is_not_finite_stays_its_own():
    for T in (3, 60):
        layer = Layer(T, 6, 2, 64, 48)
        clean = layer.run().clone()
        layer.x[1, 5] = torch.nan
        y = layer.run()
        others = torch.arange(T, device=DEV) != 1
        assert torch.isnan(y[1]).all() and torch.equal(y[others], clean[others])


def test_groups_bias_and_padding_tokens():
    layer = Layer(90, 16, 4, 128, 96, score=ssg.SSG_ROUTE_SIGMOID, groups=4, top_groups=2, group_top=2, scale=2.5)
    layer.logits[::4] = -torch.inf
    bias = (torch.arange(16) % 5 * 1e-2).to(DEV)
    y = layer.run(bias)
    layer.check(y)
    assert (y[::4] == 0).all()


@pytest.mark.parametrize("T", [5, 300])
def test_experts_without_rows_and_one_with_all(T):
    layer = Layer(T, 12, 2, 64, 64)
    layer.logits[:, 5] = 50.0
    layer.logits[:, 11] = 40.0
    layer.check(layer.run())
    layer.logits[:] = -torch.inf
    y = layer.run()
    layer.check(y)
    assert (y == 0).all()


def test_whole_against_binary64():
    """From the inputs alone, with the definition's roundings (codes, bf16 h) in binary64.  A code of h can fall to the other side of a rounding boundary
    where its products' scales round differently: a step of amax / 127 in one of f terms, and o is rounded to bf16 on the way."""
    T, E, k, d, f = 64, 6, 2, 256, 336
    layer = Layer(T, E, k, d, f)
    y = f32(layer.run())
    ids, w, _ = route.choose(f32(layer.logits).astype(np.float64), k)
    xq, sx = i8.quantize(f32(layer.x))
    ref = np.zeros((T, d))
    for t in range(T):
        for e, weight in zip(ids[t], w[t]):
            part = [(c[e * n:(e + 1) * n].astype(np.float64), s[e * n:(e + 1) * n].astype(np.float64)) for (_, c, s), n in ((layer.W1, f), (layer.W2, f), (layer.W3, d))]
            u, g = (part[i][0] @ xq[t] * float(sx[t]) * part[i][1] for i in (0, 1))
            h = torch.from_numpy(u * g / (1 + np.exp(-g))).to(torch.bfloat16).float().numpy()
            hq, sh = i8.quantize(h[None])
            ref[t] += weight * (part[2][0] @ hq[0]) * float(sh[0]) * part[2][1]
    # two roundings to bf16 of 2^-9 each, at most, in norm; a code's step is 1/127 of the row's largest in a sum of 336
    assert np.linalg.norm(y - ref) <= 2 * 2.0 ** -9 * np.linalg.norm(ref)


@pytest.mark.parametrize("E,k,d,f", [(1, 1, 64, 48), (9, 2, 1040, 528), (16, 4, 96, 2064), (24, 8, 272, 336), (20, 3, 64, 1040), (40, 20, 80, 64),
                                     (33, 17, 64, 208), (6, 6, 8208, 16)])
@pytest.mark.parametrize("y_dtype", [torch.bfloat16, torch.float32])
def test_few_tokens(E, k, d, f, y_dtype):
    for T in (1, 2, 4):
        layer = Layer(T, E, k, d, f, y_dtype=y_dtype, seed=T)
        if E > 8:
            layer.logits[:, : E - k + 1] = -torch.inf           # the last choice of every token has no expert
        layer.check(layer.run())


@pytest.mark.parametrize("T", [5, 40, 300])
@pytest.mark.parametrize("y_dtype", [torch.bfloat16, torch.float32])
def test_a_token_does_not_depend_on_the_batch(T, y_dtype):
    layer = Layer(T, 8, 3, 272, 208, y_dtype=y_dtype, score=ssg.SSG_ROUTE_SIGMOID, scale=1.5)
    whole, x, z = layer.run(), layer.x, layer.logits
    for first, n in ((0, 1), (3, 2), (T - 4, 4), (0, 5)):
        part = Layer(n, 8, 3, 272, 208, y_dtype=y_dtype, score=ssg.SSG_ROUTE_SIGMOID, scale=1.5)
        part.x, part.logits = x[first:first + n].contiguous(), z[first:first + n].contiguous()
        assert torch.equal(part.run(), whole[first:first + n])


def test_another_stream_and_a_graph():
    layer = Layer(50, 8, 2, 128, 96)
    first = layer.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = layer.run()
    side.synchronize()
    assert torch.equal(y, first)
    logits = [layer.logits.clone(), layer.logits.flip(0).clone()]
    eager = []
    for z in logits:
        layer.logits.copy_(z)
        eager.append(layer.run())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.run()
    for i in (0, 1, 0, 1):
        layer.logits.copy_(logits[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[i])
        assert torch.equal(layer.run(), eager[i])


def test_no_tokens():
    layer = Layer(0, 4, 2, 64, 48)
    layer.run()
