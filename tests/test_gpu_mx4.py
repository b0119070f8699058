"""4-bit floating point on the GPU: codes and scales bit for bit against the oracle, products of operands whose sums are exact bit for bit,
others within the error of a sum in fp32."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, f32
from oracle import mx4

pytestmark = pytest.mark.gpu
SSG = {torch.bfloat16: ssg.SSG_BF16, torch.float32: ssg.SSG_F32}
BOTH = [torch.bfloat16, torch.float32]


def buffer(rows, K, fill=0xA5):
    return torch.full((ssg.ssg_mx4_bytes(rows, K),), fill, dtype=torch.uint8, device=DEV)


def parts(q, rows, K):
    up, wide = -(-rows // 16) * 16, -(-K // 256) * 256
    raw = q.cpu().numpy()
    return raw[:up * wide // 2], raw[up * wide // 2:up * wide // 2 + up * wide // 32]


def same_layout(q, rows, K, codes, scales):
    got, want = parts(q, rows, K), mx4.layout(codes, scales)
    return np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def spread(rows, cols, seed):
    """Magnitudes over many binades, ties and saturating values among them."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen) * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=gen).float())
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -5.0])[torch.randint(0, 10, (rows, cols), generator=gen)]
    x = torch.where(torch.rand(rows, cols, generator=gen) < 0.2, ties, x)
    return torch.where(torch.rand(rows, cols, generator=gen) < 0.02, torch.zeros(()), x)


def wide(x, gap, fill=7.0):
    """x inside a wider matrix."""
    out = torch.full((x.shape[0], x.shape[1] + gap), fill, dtype=x.dtype)
    out[:, :x.shape[1]] = x
    return out.to(DEV)


@pytest.mark.parametrize("rule", [ssg.SSG_MX_FLOOR, ssg.SSG_MX_CEIL])
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("rows,K,gap", [(1, 16, 0), (1, 4096, 0), (15, 48, 8), (16, 256, 0), (17, 272, 16), (75, 2736, 0), (100, 1040, 8), (300, 528, 0), (1030, 4096, 8), (9000, 272, 0)])
def test_quantize_rows(rule, dtype, rows, K, gap):
    x = spread(rows, K, rows + K).to(dtype)
    x[rows // 2, :32] = 0
    q = buffer(rows, K)
    ssg.ssg_mx4_quantize(wide(x, gap), SSG[dtype], rows, K, K + gap, 0, rule, q)
    codes, scales = mx4.quantize(f32(x), rule == ssg.SSG_MX_CEIL)
    assert same_layout(q, rows, K, codes, scales)


@pytest.mark.parametrize("rule", [ssg.SSG_MX_FLOOR, ssg.SSG_MX_CEIL])
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("rows,K,gap", [(16, 1, 0), (16, 31, 8), (32, 33, 0), (48, 255, 8), (272, 256, 0), (144, 257, 16), (1040, 777, 0), (2064, 70, 8)])
def test_quantize_columns(rule, dtype, rows, K, gap):
    x = spread(K, rows, rows + K).to(dtype)
    q = buffer(rows, K)
    ssg.ssg_mx4_quantize(wide(x, gap), SSG[dtype], rows, K, rows + gap, 1, rule, q)
    codes, scales = mx4.quantize(f32(x).T, rule == ssg.SSG_MX_CEIL)
    assert same_layout(q, rows, K, codes, scales)


@pytest.mark.parametrize("transposed", [0, 1])
@pytest.mark.parametrize("dtype", BOTH)
def test_extremes(dtype, transposed):
    """Blocks with NaN and infinities, of zeros, of the smallest and the largest numbers."""
    x = torch.ones(16, 256)
    x[0, 3], x[1, 40], x[2, 255] = torch.nan, torch.inf, -torch.inf
    x[3] = 0.0
    x[4, :64] = 3.3e38
    x[4, 64:96] = torch.linspace(-3.38e38, 3.38e38, 32)
    x[5] = 2.0 ** -126
    x[5, ::2] = 2.0 ** -128
    x[6, :32] = 2.0 ** -133
    x[6, 32:64] = 1.5 * 2.0 ** -125
    x[7] = -0.0
    x = x.to(dtype)
    for rule in (ssg.SSG_MX_FLOOR, ssg.SSG_MX_CEIL):
        q = buffer(16, 256)
        ssg.ssg_mx4_quantize((x.t() if transposed else x).contiguous().to(DEV), SSG[dtype], 16, 256, 16 if transposed else 256, transposed, rule, q)
        codes, scales = mx4.quantize(f32(x), rule == ssg.SSG_MX_CEIL)
        assert same_layout(q, 16, 256, codes, scales)
        out = torch.empty(16, 256, device=DEV)
        ssg.ssg_mx4_dequantize(q, 16, 256, out, ssg.SSG_F32, 256)
        assert np.array_equal(out.cpu().numpy().astype(np.float64), mx4.values(codes, scales), equal_nan=True)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("rows,K", [(1, 1), (5, 16), (16, 31), (17, 300), (40, 1025), (1030, 4085), (9000, 300)])
def test_dequantize(dtype, rows, K):
    """Exact in both types, for every code and scale; what lies between rows and behind the last one stays."""
    rng = np.random.default_rng(rows + K)
    codes, scales = rng.integers(0, 16, (rows, K), np.uint8), rng.integers(0, 253, (rows, -(-K // 32)), np.uint8)
    scales[:, 0] = np.array([0, 1, 252, 255])[np.arange(rows) % 4]
    c, s = mx4.layout(codes, scales)
    q = buffer(rows, K)
    q[:c.size + s.size] = torch.from_numpy(np.concatenate([c, s])).to(DEV)
    ld = K + -K % 8 + 8
    out = torch.full((rows + 1, ld), 5.0, dtype=dtype, device=DEV)
    ssg.ssg_mx4_dequantize(q, rows, K, out, SSG[dtype], ld)
    got = f32(out)
    assert np.array_equal(got[:rows, :K].astype(np.float64), mx4.values(codes, scales), equal_nan=True)
    assert (got[:rows, K:] == 5).all() and (got[rows] == 5).all()


@pytest.mark.parametrize("rows,K", [(1, 16), (16, 256), (17, 48), (75, 2736), (33, 272)])
def test_pack(rows, K):
    rng = np.random.default_rng(rows)
    codes, scales = rng.integers(0, 16, (rows, K), np.uint8), rng.integers(0, 256, (rows, -(-K // 32)), np.uint8)
    q = buffer(rows, K)
    packed = torch.from_numpy(mx4.nibbles(codes)).to(DEV)
    ssg.ssg_mx4_pack(packed, torch.from_numpy(scales).to(DEV), rows, K, q)
    assert same_layout(q, rows, K, codes, scales)
    back, s = torch.zeros_like(packed), torch.zeros(rows, -(-K // 32), dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_unpack(q, rows, K, back, s)
    assert torch.equal(back, packed) and np.array_equal(s.cpu().numpy(), scales)


def operand(rows, K, seed, low, high):
    """A random operand with scales 2^low to 2^high and its values."""
    rng = np.random.default_rng(seed)
    codes, scales = rng.integers(0, 16, (rows, K), np.uint8), rng.integers(127 + low, 128 + high, (rows, -(-K // 32)), np.uint8)
    c, s = mx4.layout(codes, scales)
    q = buffer(rows, K, 0)
    q[:c.size + s.size] = torch.from_numpy(np.concatenate([c, s])).to(DEV)
    return q, mx4.values(codes, scales)


def as_type(exact, dtype):
    return f32(torch.from_numpy(exact).to(dtype))


def product(qa, M, qb, N, K, dtype, gap=0):
    out = torch.full((M + 1, N + gap), 3.0, dtype=dtype, device=DEV)
    ssg.ssg_mx4_gemm(qa, M, qb, N, K, out, SSG[dtype], N + gap)
    got = f32(out)
    assert (got[:, N:] == 3).all() and (got[M] == 3).all(), "written outside the result"
    return got[:M, :N]


# Terms are multiples of 1/4 and at most 36 (with scales of 1 and 2: 144), so that up to K = 11008 every partial sum is a whole number of
# quarters below 144 K * 4 < 2^23: exact in fp32 in any order, and the result is the exact sum rounded once.
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (2, 48, 256), (4, 1040, 4112), (5, 16, 272), (16, 272, 48), (17, 48, 528), (33, 1040, 1040), (64, 272, 2736), (65, 16, 1),
                                   (129, 144, 33), (130, 272, 255), (300, 528, 1376), (257, 1040, 300), (700, 2064, 777), (512, 512, 11008)])
def test_exact_products(dtype, M, N, K):
    qa, a = operand(M, K, M + K, 0, 1)
    qb, b = operand(N, K, N + K + 1, 0, 1)
    assert np.array_equal(product(qa, M, qb, N, K, dtype, gap=8), as_type(a @ b.T, dtype))


@pytest.mark.parametrize("M,N,K", [(3, 48, 4112), (40, 272, 2736), (300, 528, 1376), (1100, 1040, 640)])
def test_products_with_scales_far_apart(M, N, K):
    """K terms added in fp32 in some order, each addition off by at most 2^-23 of a partial sum, which is at most the sum of the terms' magnitudes."""
    qa, a = operand(M, K, 1, -12, 12)
    qb, b = operand(N, K, 2, -12, 12)
    got = product(qa, M, qb, N, K, torch.float32).astype(np.float64)
    assert (np.abs(got - a @ b.T) <= K * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()
    assert np.array_equal(got, product(qa, M, qb, N, K, torch.float32).astype(np.float64)), "another call, other bits"


@pytest.mark.parametrize("M", [2, 20, 40, 300])
def test_products_with_no_number(M):
    """A block that is no number makes its row or column NaN and nothing else."""
    K, N = 528, 272
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(1))
    w = torch.randn(N, K, generator=torch.Generator().manual_seed(2))
    x[1, 500], w[33, 7] = torch.nan, torch.inf
    qa, qb = buffer(M, K), buffer(N, K)
    ssg.ssg_mx4_quantize(x.to(DEV), ssg.SSG_F32, M, K, K, 0, 0, qa)
    ssg.ssg_mx4_quantize(w.to(DEV), ssg.SSG_F32, N, K, K, 0, 0, qb)
    got = np.isnan(product(qa, M, qb, N, K, torch.float32))
    want = np.zeros((M, N), bool)
    want[1], want[:, 33] = True, True
    assert np.array_equal(got, want)


def exact_rows(rows, K, seed, dtype):
    """Rows whose values in 4 bits have scales 1 and 2 only."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.rand(rows, K, generator=gen) * 12 - 6
    x[:, ::32] = torch.where(torch.rand(rows, -(-K // 32), generator=gen) < 0.5, 4.0, 8.0)
    return x.to(dtype)


@pytest.mark.parametrize("rule", [ssg.SSG_MX_FLOOR, ssg.SSG_MX_CEIL])
@pytest.mark.parametrize("x_dtype", BOTH)
@pytest.mark.parametrize("y_dtype", BOTH)
@pytest.mark.parametrize("M,N,K,gap", [(0, 16, 32, 0), (1, 16, 16, 0), (1, 1040, 4096, 8), (2, 48, 4112, 0), (3, 272, 48, 8), (4, 528, 11008, 0), (5, 272, 1376, 0), (16, 48, 80, 8), (40, 1040, 528, 0),
                                       (333, 1040, 2736, 0)])
def test_linear(rule, x_dtype, y_dtype, M, N, K, gap):
    x = exact_rows(M, K, M + N, x_dtype) if M else torch.zeros(0, K, dtype=x_dtype)
    qw, w = operand(N, K, 5, 0, 1)
    y = torch.full((M + 1, N + gap), 3.0, dtype=y_dtype, device=DEV)
    work = torch.full((ssg.ssg_mx4_linear_workspace_bytes(M, K),), 0xA5, dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_linear(wide(x, gap), SSG[x_dtype], M, K, K + gap, rule, qw, N, y, SSG[y_dtype], N + gap, work)
    got = f32(y)
    want = as_type(mx4.values(*mx4.quantize(f32(x), rule == ssg.SSG_MX_CEIL)) @ w.T, y_dtype) if M else np.zeros((0, N), np.float32)
    assert np.array_equal(got[:M, :N], want) and (got[:, N:] == 3).all() and (got[M] == 3).all()


@pytest.mark.parametrize("x_dtype,y_dtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("M,N,K", [(5, 48, 16), (7, 4096, 5264), (7, 4112, 5264), (8, 272, 528), (9, 4096, 4096), (9, 16, 4112), (13, 1040, 2736), (16, 16, 2304), (16, 272, 2320), (16, 528, 784)])
def test_linear_of_few_rows(x_dtype, y_dtype, M, N, K):
    """On both sides of where the product's own launch quantizes the rows."""
    test_linear(ssg.SSG_MX_CEIL, x_dtype, y_dtype, M, N, K, 8)


@pytest.mark.parametrize("M", [1, 4, 9, 16])
def test_token_with_no_number(M):
    x = torch.ones(M, 512)
    x[M - 1, 300] = torch.inf
    qw, _ = operand(48, 512, 5, 0, 1)
    y = torch.empty(M, 48, device=DEV)
    ssg.ssg_mx4_linear(x.to(DEV), ssg.SSG_F32, M, 512, 512, 0, qw, 48, y, ssg.SSG_F32, 48, buffer(M, 512))
    bad = torch.isnan(y).cpu()
    assert bad[M - 1].all() and not bad[:M - 1].any()


@pytest.mark.parametrize("which", ["both", "dx", "dW"])
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("M,N,K,gap", [(0, 16, 32, 0), (1, 16, 16, 0), (5, 48, 272, 8), (31, 272, 48, 0), (33, 144, 528, 8), (256, 272, 1040, 0), (300, 1040, 272, 8), (777, 2064, 1376, 0)])
def test_linear_bwd(which, dtype, M, N, K, gap):
    dy, x = exact_rows(M, N, 1, dtype), exact_rows(M, K, 2, dtype)
    if M:
        # blocks along the rows, too: scales of 1 and 2
        dy[::32], x[::32] = (torch.where(torch.rand(-(-M // 32), n, generator=torch.Generator().manual_seed(3)) < 0.5, 4.0, 8.0).to(dtype) for n in (N, K))
    codes, scales = (np.random.default_rng(4).integers(0, 16, (K, N), np.uint8), np.full((K, -(-N // 32)), 127, np.uint8))
    qt = buffer(K, N, 0)
    c, s = mx4.layout(codes, scales)
    qt[:c.size + s.size] = torch.from_numpy(np.concatenate([c, s])).to(DEV)
    dx = torch.full((M + 1, K + gap), 3.0, dtype=dtype, device=DEV) if which != "dW" else None
    dW = torch.full((N + 1, K + gap), 3.0, dtype=torch.float32, device=DEV) if which != "dx" else None
    work = torch.full((ssg.ssg_mx4_linear_bwd_workspace_bytes(M, N, K),), 0xA5, dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_linear_bwd(wide(dy, gap), SSG[dtype], N + gap, wide(x, gap) if dW is not None else None, SSG[dtype], K + gap, M, N, K, 0,
                           qt if dx is not None else None, dx, SSG[dtype], K + gap, dW, ssg.SSG_F32, K + gap, work)
    want_dx, want_dW = mx4.linear_bwd(f32(dy), f32(x), (codes, scales)) if M else (np.zeros((0, K)), np.zeros((N, K)))
    for out, want, t in ((dx, want_dx, dtype), (dW, want_dW, torch.float32)):
        if out is not None:
            got = f32(out)
            assert np.array_equal(got[:-1, :K], as_type(want, t)) and (got[:, K:] == 3).all() and (got[-1] == 3).all()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("M,N,K", [(3, 768, 1120), (61, 1696, 2192), (256, 4096, 2064), (740, 2352, 1120), (1776, 1216, 128), (700, 64, 4112), (105, 4864, 384)])
def test_linear_bwd_in_one_launch(dtype, M, N, K):
    """Either product's sum the longer, from one tile to more than the chip holds; the last one in two launches."""
    test_linear_bwd("both", dtype, M, N, K, 8)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("M,N,K", [(1570, 4112, 8032), (4096, 4096, 4096), (3300, 2416, 11136), (1570, 7600, 8032)])
def test_linear_bwd_in_large_tiles(dtype, M, N, K):
    """Both products, of one and of several rounds of large tiles and of different numbers of them, against each alone (every sum is exact, see above)."""
    assert ssg.ssg_mx4_gemm_plan(M, K, N).tile == ssg.ssg_mx4_gemm_plan(N, K, M).tile == 256
    dy, x = exact_rows(M, N, 1, dtype), exact_rows(M, K, 2, dtype)
    dy[::32], x[::32] = (torch.where(torch.rand(-(-M // 32), n, generator=torch.Generator().manual_seed(3)) < 0.5, 4.0, 8.0).to(dtype) for n in (N, K))
    dy, x, qt = dy.to(DEV), x.to(DEV), buffer(K, N)
    ssg.ssg_mx4_quantize(exact_rows(K, N, 5, torch.float32).to(DEV), ssg.SSG_F32, K, N, N, 0, 0, qt)
    work = buffer(1, 1).new_full((ssg.ssg_mx4_linear_bwd_workspace_bytes(M, N, K),), 0xA5)

    def run(with_dx, with_dW):
        dx, dW = torch.full((M + 1, K), 3.0, dtype=dtype, device=DEV), torch.full((N + 1, K), 3.0, device=DEV)
        ssg.ssg_mx4_linear_bwd(dy, SSG[dtype], N, x, SSG[dtype], K, M, N, K, 0, qt, dx if with_dx else None, SSG[dtype], K, dW if with_dW else None, ssg.SSG_F32, K, work)
        return dx, dW

    dx, dW = run(True, True)
    assert torch.equal(dx, run(True, False)[0]) and torch.equal(dW, run(False, True)[1])
    assert bool((dx[M] == 3).all()) and bool((dW[N] == 3).all())


@pytest.mark.parametrize("M,K", [(1, 92160), (1, 92416), (1, 94208), (2, 46080), (3, 30976), (4, 23040), (4, 23056)])
def test_long_rows_of_few_tokens(M, K):
    """On both sides of what a workgroup quantizes itself.  Scales of 1: terms of at most 36, whole numbers of quarters, whose sums stay below 2^24 quarters."""
    gen = torch.Generator().manual_seed(K)
    x = (torch.rand(M, K, generator=gen) * 12 - 6).to(torch.bfloat16)
    x[:, ::32] = 5.0
    qw, w = operand(32, K, 5, 0, 0)
    y = torch.empty(M, 32, device=DEV)
    ssg.ssg_mx4_linear(x.to(DEV), ssg.SSG_BF16, M, K, K, 0, qw, 32, y, ssg.SSG_F32, 32, buffer(M, K))
    assert np.array_equal(f32(y), as_type(mx4.values(*mx4.quantize(f32(x))) @ w.T, torch.float32))


@pytest.mark.parametrize("dy_dtype,x_dtype,dx_dtype,dw_dtype", [(torch.bfloat16, torch.float32, torch.float32, torch.bfloat16),
                                                                 (torch.float32, torch.bfloat16, torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("rule", [ssg.SSG_MX_FLOOR, ssg.SSG_MX_CEIL])
@pytest.mark.parametrize("M,N,K", [(45, 48, 272), (700, 1040, 528), (2100, 2064, 1376)])
def test_linear_bwd_of_mixed_types(dy_dtype, x_dtype, dx_dtype, dw_dtype, rule, M, N, K):
    """Sums of N, and of M, terms in fp32, each addition off by at most 2^-23 of a partial sum; results in bf16 rounded once more, by half a step."""
    dy, x = spread(M, N, 1).to(dy_dtype), spread(M, K, 2).to(x_dtype)
    W = spread(K, N, 3)
    qt = buffer(K, N, 0)
    ssg.ssg_mx4_quantize(W.to(DEV), ssg.SSG_F32, K, N, N, 0, rule, qt)
    dx, dW = torch.empty(M, K, dtype=dx_dtype, device=DEV), torch.empty(N, K, dtype=dw_dtype, device=DEV)
    work = torch.full((ssg.ssg_mx4_linear_bwd_workspace_bytes(M, N, K),), 0xA5, dtype=torch.uint8, device=DEV)
    ssg.ssg_mx4_linear_bwd(dy.to(DEV), SSG[dy_dtype], N, x.to(DEV), SSG[x_dtype], K, M, N, K, rule, qt, dx, SSG[dx_dtype], K, dW, SSG[dw_dtype], K, work)
    ceil = rule == ssg.SSG_MX_CEIL
    a, b, wt = (mx4.values(*mx4.quantize(v, ceil)) for v in (f32(dy), f32(dy).T, f32(W)))
    xt = mx4.values(*mx4.quantize(f32(x).T, ceil))
    for out, t, p, q, n in ((dx, dx_dtype, a, wt, N), (dW, dw_dtype, b, xt, M)):
        want, off = p @ q.T, n * 2.0 ** -23 * (np.abs(p) @ np.abs(q).T)
        assert (np.abs(f32(out) - want) <= off + (2.0 ** -8 * (np.abs(want) + off) if t == torch.bfloat16 else 0)).all()


@pytest.mark.parametrize("low_a,high_a,low_b,high_b", [(-127, -107, 105, 125), (105, 125, -127, -107), (-127, -100, -40, 0), (-70, -66, -70, -66), (-127, -100, -127, -100)])
@pytest.mark.parametrize("M,N,K", [(3, 48, 4112), (40, 272, 2736), (300, 528, 1376), (1100, 1040, 640)])
def test_products_over_the_range_of_scales(M, N, K, low_a, high_a, low_b, high_b):
    """As with scales far apart; a partial sum below 2^-126 is rounded to a multiple of 2^-149, or away, with half of that beside the rest."""
    qa, a = operand(M, K, 1, low_a, high_a)
    qb, b = operand(N, K, 2, low_b, high_b)
    got = product(qa, M, qb, N, K, torch.float32).astype(np.float64)
    assert (np.abs(got - a @ b.T) <= K * (2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 2.0 ** -150)).all()


def test_values_beyond_the_types():
    """Bytes that only another program's scales have: values behind the largest number are infinite, 255 is no number."""
    codes, scales = np.tile(np.arange(16, dtype=np.uint8), (4, 2)), np.array([[252], [253], [254], [255]], np.uint8)
    c, s = mx4.layout(codes, scales)
    q = buffer(4, 32, 0)
    q[:c.size + s.size] = torch.from_numpy(np.concatenate([c, s])).to(DEV)
    for dtype in BOTH:
        out = torch.empty(4, 32, dtype=dtype, device=DEV)
        ssg.ssg_mx4_dequantize(q, 4, 32, out, SSG[dtype], 32)
        with np.errstate(over="ignore"):
            assert np.array_equal(f32(out), mx4.values(codes, scales).astype(np.float32), equal_nan=True)
