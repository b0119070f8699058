"""Rows in 8-bit integers and their products on the GPU, bit for bit against the oracle's binary32 steps on exact sums."""
import numpy as np
import pytest
import torch

import paper_2409_12517_amd as ssg
from gpu_util import DEV, f32
from oracle import i8

pytestmark = pytest.mark.gpu
SSG = {torch.bfloat16: ssg.SSG_BF16, torch.float32: ssg.SSG_F32}


def buffer(rows, K, fill=0xA5):
    return torch.full((ssg.ssg_i8_bytes(rows, K),), fill, dtype=torch.uint8, device=DEV)


def rows_of(rows, K, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=gen) * torch.exp2(torch.randint(-8, 9, (rows, 1), generator=gen).float())
    return x.to(dtype)


def parts(q, rows, K):
    """codes in the layout, scales, of a buffer."""
    up, wide = -(-rows // 16) * 16, -(-K // 128) * 128
    raw = q.cpu().numpy()
    at = -(-up * wide // 256) * 256
    return raw[:up * wide], raw[at:at + 4 * up].view(np.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 15, 16, 17, 100])
@pytest.mark.parametrize("K", [16, 64, 80, 336, 1040, 4096, 4112, 11008, 28672])
def test_quantize(dtype, rows, K):
    x = rows_of(rows, K, dtype, rows + K)
    x[rows // 2] = 0
    q = buffer(rows, K)
    ssg.ssg_i8_quantize(x.to(DEV), SSG[dtype], rows, K, K, q)
    codes, scales = i8.quantize(f32(x))
    got, s = parts(q, rows, K)
    assert np.array_equal(got, i8.layout(codes))
    assert np.array_equal(s[:rows], scales) and not s[rows:].any()
    out, sc = torch.empty(rows, K, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    ssg.ssg_i8_unpack(q, rows, K, out, sc)
    assert np.array_equal(out.cpu().numpy(), codes) and np.array_equal(sc.cpu().numpy(), scales)
    back = buffer(rows, K, 0x5A)
    ssg.ssg_i8_pack(out, sc, rows, K, back)
    assert all(np.array_equal(a, b) for a, b in zip(parts(back, rows, K), (got, s)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_extremes(dtype):
    """Rows with infinities, NaN, the smallest and the largest numbers, ties between two codes."""
    K = 48
    x = torch.zeros(9, K)
    x[0, 3], x[1, 40], x[2, 0] = torch.inf, torch.nan, -torch.inf
    x[3] = 1e-38
    x[4, :2] = torch.tensor([1e-40, -5e-41])
    x[5] = 3.3e38
    x[6, :5] = torch.tensor([127.0, 0.5, 1.5, -2.5, 126.5])
    x[7, 47] = -1.0
    x[8] = -2.0 ** -126
    x = x.to(dtype)
    q = buffer(9, K)
    ssg.ssg_i8_quantize(x.to(DEV), SSG[dtype], 9, K, K, q)
    codes, scales = i8.quantize(f32(x))
    got, s = parts(q, 9, K)
    assert np.array_equal(got, i8.layout(codes)) and np.array_equal(s[:9], scales, equal_nan=True)
    assert np.isnan(s[:3]).all() and np.isfinite(s[3:]).all()


def test_quantize_strided_rows():
    wide = rows_of(37, 400, torch.bfloat16, 1).to(DEV)
    q, part = buffer(37, 208), wide[:, 16:224]
    ssg.ssg_i8_quantize(part, ssg.SSG_BF16, 37, 208, 400, q)
    codes, scales = i8.quantize(f32(part))
    got, s = parts(q, 37, 208)
    assert np.array_equal(got, i8.layout(codes)) and np.array_equal(s[:37], scales)


def product(M, N, K, c_dtype, seed=0, ldc=None, full_range=False):
    gen = np.random.default_rng(seed)
    lo = -128 if full_range else -127
    a, b = gen.integers(lo, 128, (M, K), dtype=np.int8), gen.integers(lo, 128, (N, K), dtype=np.int8)
    sa, sb = np.exp(gen.normal(size=M)).astype(np.float32) * np.float32(1e-2), np.exp(gen.normal(size=N)).astype(np.float32) * np.float32(1e-3)
    qa, qb = buffer(M, K), buffer(N, K)
    ssg.ssg_i8_pack(torch.from_numpy(a).to(DEV), torch.from_numpy(sa).to(DEV), M, K, qa)
    ssg.ssg_i8_pack(torch.from_numpy(b).to(DEV), torch.from_numpy(sb).to(DEV), N, K, qb)
    ldc = ldc or N
    C = torch.full((M, ldc), 7.0, dtype=c_dtype, device=DEV)
    ssg.ssg_i8_gemm(qa, M, qb, N, K, C, SSG[c_dtype], ldc)
    want = torch.from_numpy(i8.matmul(a, sa, b, sb)).to(c_dtype)
    assert torch.equal(C[:, :N].cpu(), want)
    assert (C[:, N:] == 7.0).all()


@pytest.mark.parametrize("M", [1, 16, 17, 32, 33, 48, 64, 65, 100, 128, 129, 200, 255, 257, 300])
@pytest.mark.parametrize("N,K", [(16, 16), (48, 64), (128, 80), (272, 336), (144, 1040), (400, 640)])
def test_product_over_sizes(M, N, K):
    product(M, N, K, torch.float32, M + N)


@pytest.mark.parametrize("K", [16, 64, 128, 192, 256, 320, 384, 448, 512, 576, 1088])
@pytest.mark.parametrize("M", [7, 40, 90, 513, 1100])
def test_product_over_steps_of_k(M, K):
    product(M, 528, K, torch.bfloat16, K)


@pytest.mark.parametrize("M,N,K", [(1, 11008, 4096), (5, 2736, 4112), (513, 2064, 1360), (2049, 1024, 688), (1296, 1552, 2064), (777, 4096, 512),
                                   (3000, 2736, 272)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product_large(M, N, K, dtype):
    product(M, N, K, dtype, 3)


@pytest.mark.parametrize("tile,M,N,K", [(256, 4096, 4096, 336), (256, 3970, 4096, 1040), (256, 3900, 4080, 656), (256, 7960, 4080, 784), (256, 8030, 4096, 400),
                                        (128, 4200, 4080, 400), (128, 9000, 2064, 272), (128, 4170, 4112, 784), (128, 1290, 2064, 1040)])
def test_product_in_tiles(tile, M, N, K):
    """Whole tiles, tiles with more and with no more than half of their rows, a last column tile of one block; several tiles to a workgroup."""
    assert ssg.ssg_i8_gemm_plan(M, N, K).tile == tile
    product(M, N, K, torch.bfloat16, M)
    product(M, N, K, torch.float32, K)


def test_product_strided_result_and_the_lowest_code():
    product(70, 48, 96, torch.bfloat16, ldc=64)
    product(300, 208, 96, torch.float32, ldc=256)
    product(40, 32, 4096, torch.float32, full_range=True)


def test_largest_sums_stay_exact():
    K = 131056
    for sign in (1, -1):
        a = torch.full((3, K), -128, dtype=torch.int8, device=DEV)
        b = torch.full((16, K), -128 if sign > 0 else 127, dtype=torch.int8, device=DEV)
        qa, qb = buffer(3, K), buffer(16, K)
        ssg.ssg_i8_pack(a, torch.ones(3, device=DEV), 3, K, qa)
        ssg.ssg_i8_pack(b, torch.ones(16, device=DEV), 16, K, qb)
        C = torch.empty(3, 16, device=DEV)
        ssg.ssg_i8_gemm(qa, 3, qb, 16, K, C, ssg.SSG_F32, 16)
        assert (C.double() == float(np.float32((128 * 128 if sign > 0 else -128 * 127) * K))).all()


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("y_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,N", [(1, 16, 16), (2, 528, 48), (4, 14352, 32), (4, 16384, 16), (1, 28672, 64), (1, 64, 16), (1, 2736, 1040), (3, 4096, 528), (8, 11008, 256), (16, 1040, 272), (17, 80, 48), (33, 336, 272), (260, 1040, 784)])
def test_linear(x_dtype, y_dtype, M, K, N):
    x, W = rows_of(M, K + 8, x_dtype, M).to(DEV), rows_of(N, K, torch.bfloat16, N).to(DEV)
    x[M // 2] = 0
    q = buffer(N, K)
    ssg.ssg_i8_quantize(W, ssg.SSG_BF16, N, K, K, q)
    work = torch.empty(ssg.ssg_i8_linear_workspace_bytes(M, K), dtype=torch.uint8, device=DEV)
    y = torch.full((M, N + 16), 3.0, dtype=y_dtype, device=DEV)
    ssg.ssg_i8_linear(x, SSG[x_dtype], M, K, K + 8, q, N, y, SSG[y_dtype], N + 16, work)
    (a, sa), (b, sb) = i8.quantize(f32(x)[:, :K]), i8.quantize(f32(W))
    assert torch.equal(y[:, :N].cpu(), torch.from_numpy(i8.matmul(a, sa, b, sb)).to(y_dtype))
    assert (y[:, N:] == 3.0).all()


def test_a_row_that_is_not_finite_stays_its_own():
    M, K, N = 20, 128, 32
    x = rows_of(M, K, torch.float32, 5)
    x[4, 7], x[17, 0] = torch.nan, torch.inf
    q, work = buffer(N, K), buffer(M, K)
    W = rows_of(N, K, torch.float32, 6)
    ssg.ssg_i8_quantize(W.to(DEV), ssg.SSG_F32, N, K, K, q)
    y = torch.empty(M, N, device=DEV)
    ssg.ssg_i8_linear(x.to(DEV), ssg.SSG_F32, M, K, K, q, N, y, ssg.SSG_F32, N, work)
    bad = torch.zeros(M, dtype=torch.bool)
    bad[[4, 17]] = True
    assert torch.isnan(y.cpu()[bad]).all() and torch.isfinite(y.cpu()[~bad]).all()


def test_no_rows():
    q = buffer(16, 64)
    ssg.ssg_i8_linear(None, ssg.SSG_BF16, 0, 64, 64, q, 16, None, ssg.SSG_BF16, 16, None)
    ssg.ssg_i8_quantize(None, ssg.SSG_BF16, 0, 64, 64, None)


def test_another_stream_and_a_graph():
    M, K, N = 100, 320, 272
    W = rows_of(N, K, torch.bfloat16, 1).to(DEV)
    q, work = buffer(N, K), buffer(M, K)
    ssg.ssg_i8_quantize(W, ssg.SSG_BF16, N, K, K, q)
    xs = [rows_of(M, K, torch.bfloat16, s).to(DEV) for s in (2, 3)]

    def run(x, work):
        y = torch.empty(M, N, device=DEV)
        ssg.ssg_i8_linear(x, ssg.SSG_BF16, M, K, K, q, N, y, ssg.SSG_F32, N, work)
        return y

    eager = [run(x, work).clone() for x in xs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = run(xs[0], buffer(M, K))
    side.synchronize()
    assert torch.equal(y, eager[0])
    fixed = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = run(fixed, work)
    for i in (1, 0, 1):
        fixed.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[i])
        assert torch.equal(run(xs[i], buffer(M, K)), eager[i])
