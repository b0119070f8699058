// Products of matrices in microscaled 4-bit floating point:
//
//   C[m,n] = sum over blocks b of 32 along K of  Xa[m,b] Xb[n,b] sum_{k in b} a[m,k] b[n,k]           sums in fp32
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 32 codes and one scale of each operand from a lane, so the scales cost no instruction of their
// own.  Both operands lie in blocks of 16 rows by 128 codes in the order in which a wave holds them (see Mx4RowsArgs): a block is one 1 KB
// load, to LDS or straight to registers, with nothing to permute and no LDS bank conflicts; the scales of two blocks are 128 bytes.
// The order in which a result's terms are added, and so its last bits, is that of the kernel that it runs in, and the same in every call.
#include <cmath>

#include "ssg_gemm_tile.h"
#include "ssg_lds_load.h"
#include "ssg_mx4.h"

namespace ssg {

namespace {

struct Mx4Params {
    const uint8_t *A, *B, *sa, *sb;
    void *C;
    int64_t M, N, ldc;
    int KB;                      // blocks of 128 along K, an even number
    int c_f32;
    int tiles_n;
};

typedef int v4i_t __attribute__((ext_vector_type(4)));
typedef float v4f_t __attribute__((ext_vector_type(4)));
// the weights' fragment first: a lane then holds row l & 15 of C and, in its four registers, columns 4 (l >> 4) .. + 3.  STEP: which byte of
// the scales' words, that of the first or the second block of a pair.
template <int STEP> __device__ __forceinline__ v4f_t mfma_mx4(const v4i_t &w, uint32_t sw, const v4i_t &x, uint32_t sx, const v4f_t &c) {
    constexpr int kE2M1 = 4;
    const v8i a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, kE2M1, kE2M1, STEP, (int)sw, STEP, (int)sx);
}

// Tile number v of rows * tiles_n: the column tiles of one row tile after the other in groups of four row tiles, and eight contiguous
// ranges of that order for the eight XCDs.
struct Mx4Tile { int rb, cb; };                          // first row block and column block
__device__ __forceinline__ Mx4Tile find_tile(const Mx4Params &p, int row_blocks, int col_blocks, int rows, int v) {
    const int all = rows * p.tiles_n, full = all & ~7;
    const int t = v < full ? (v & 7) * (full >> 3) + (v >> 3) : v;
    constexpr int kGroup = 4;
    const int group = t / (kGroup * p.tiles_n), in_group = t - group * (kGroup * p.tiles_n);
    const int height = rows - group * kGroup < kGroup ? rows - group * kGroup : kGroup;
    return {__builtin_amdgcn_readfirstlane((group * kGroup + in_group % height) * row_blocks), __builtin_amdgcn_readfirstlane(in_group / height * col_blocks)};
}

// Four neighbouring columns of a row.
__device__ __forceinline__ void store4(const Mx4Params &p, int64_t row, int64_t col, const v4f_t &v) {
    if (row >= p.M) return;
    if (p.c_f32) *reinterpret_cast<float4 *>(static_cast<float *>(p.C) + row * p.ldc + col) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.C) + row * p.ldc + col) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// ---- few rows ------------------------------------------------------------------------------------------
// RB blocks of 16 rows by CB blocks of 16 columns to a workgroup, whose waves share K out in pairs of blocks and add their sums in LDS, wave after
// wave.  Both operands come straight from memory in the order of the lanes, U pairs' loads at a time.
template <int RB, int CB, int WAVES> __global__ __launch_bounds__(64 * WAVES) void mx4_few_kernel(Mx4Params p) {
    __shared__ v4f_t part[WAVES][RB * CB][64];
    const int row_blocks = (int)((p.M + 15) / 16), col_blocks = (int)(p.N / 16), pairs = p.KB / 2;
    const Mx4Tile tile = find_tile(p, RB, CB, (row_blocks + RB - 1) / RB, blockIdx.x);
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint8_t *a_src[RB], *b_src[CB], *sa_src[RB], *sb_src[CB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int64_t rb = tile.rb + r < row_blocks ? tile.rb + r : row_blocks - 1;
        a_src[r] = p.A + rb * p.KB * 1024 + l * 16;
        sa_src[r] = p.sa + rb * pairs * 128 + l * 2;
    }
#pragma unroll
    for (int c = 0; c < CB; ++c) {
        const int64_t cb = tile.cb + c < col_blocks ? tile.cb + c : col_blocks - 1;
        b_src[c] = p.B + cb * p.KB * 1024 + l * 16;
        sb_src[c] = p.sb + cb * pairs * 128 + l * 2;
    }
    const int share = (pairs + WAVES - 1) / WAVES;
    const int p1 = (w + 1) * share < pairs ? (w + 1) * share : pairs;
    v4f_t acc[RB][CB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[r][c] = v4f_t{0, 0, 0, 0};
    auto steps = [&](auto count, int at) {
        constexpr int U = decltype(count)::value;
        v4i_t fa[U][2][RB], fb[U][2][CB];
        uint32_t xa[U][RB], xb[U][CB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int c = 0; c < CB; ++c) {
#pragma unroll
                for (int h = 0; h < 2; ++h) fb[u][h][c] = __builtin_nontemporal_load(reinterpret_cast<const v4i_t *>(b_src[c] + (int64_t)(at + u) * 2048 + h * 1024));
                xb[u][c] = *reinterpret_cast<const uint16_t *>(sb_src[c] + (int64_t)(at + u) * 128);
            }
#pragma unroll
            for (int r = 0; r < RB; ++r) {
#pragma unroll
                for (int h = 0; h < 2; ++h) fa[u][h][r] = *reinterpret_cast<const v4i_t *>(a_src[r] + (int64_t)(at + u) * 2048 + h * 1024);
                xa[u][r] = *reinterpret_cast<const uint16_t *>(sa_src[r] + (int64_t)(at + u) * 128);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    acc[r][c] = mfma_mx4<0>(fb[u][0][c], xb[u][c], fa[u][0][r], xa[u][r], acc[r][c]);
                    acc[r][c] = mfma_mx4<1>(fb[u][1][c], xb[u][c], fa[u][1][r], xa[u][r], acc[r][c]);
                }
    };
    constexpr int U = RB + CB > 4 ? 2 : 4;
    int at = w * share;
    for (; at + U <= p1; at += U) steps(std::integral_constant<int, U>{}, at);
    for (; at < p1; ++at) steps(std::integral_constant<int, 1>{}, at);
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < CB; ++c) part[w][r * CB + c][l] = acc[r][c];
    __syncthreads();
    for (int i = w; i < RB * CB; i += WAVES) {
        const int rb = tile.rb + i / CB, cb = tile.cb + i % CB;
        if (rb >= row_blocks || cb >= col_blocks) continue;
        v4f_t v = part[0][i][l];
#pragma unroll
        for (int x = 1; x < WAVES; ++x) v += part[x][i][l];
        store4(p, (int64_t)rb * 16 + (l & 15), (int64_t)cb * 16 + (l >> 4) * 4, v);
    }
}

// ---- up to four rows, quantized on the way ------------------------------------------------------------------
// A block of x has its scale to itself, so a lane forms the codes that it multiplies from 32 values of its row in its own registers, and nothing is
// exchanged before the products.  16 columns to a workgroup, whose waves share K out.
template <bool BF16, int WAVES> __global__ __launch_bounds__(64 * WAVES) void mx4_token_kernel(Mx4TokenArgs a) {
    __shared__ v4f_t part[WAVES][64];
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = l >> 4;
    const int pairs = (int)(mx4_width(a.K) / 256), share = (pairs + WAVES - 1) / WAVES;
    const int p1 = (w + 1) * share < pairs ? (w + 1) * share : pairs;
    const uint8_t *b = a.B + (int64_t)blockIdx.x * pairs * 2048 + l * 16, *sb = a.sb + (int64_t)blockIdx.x * pairs * 128 + l * 2;
    const bool live = (l & 15) < a.rows;
    const uint8_t *x = static_cast<const uint8_t *>(a.x) + (live ? l & 15 : 0) * a.ld * (BF16 ? 2 : 4);
    v4f_t acc = {0, 0, 0, 0};
    for (int at = w * share; at < p1; ++at) {
        v4i_t f[2];
        Mx4Block<BF16> v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) f[h] = __builtin_nontemporal_load(reinterpret_cast<const v4i_t *>(b + (int64_t)at * 2048 + h * 1024));
        const uint32_t sw = *reinterpret_cast<const uint16_t *>(sb + (int64_t)at * 128);
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h].load(x, (int64_t)at * 256 + h * 128 + g * 32, a.K, live);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t byte = mx4_scale_byte(v[h].top_bits(), a.ceil);
            const uint4 q = v[h].codes(byte);
            const v4i_t codes = {(int)q.x, (int)q.y, (int)q.z, (int)q.w};
            acc = h == 0 ? mfma_mx4<0>(f[h], sw, codes, byte, acc) : mfma_mx4<0>(f[h], sw >> 8, codes, byte, acc);
        }
    }
    part[w][l] = acc;
    __syncthreads();
    if (w != 0 || !live) return;
    v4f_t v = part[0][l];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += part[i][l];
    const int64_t at = (l & 15) * a.ldc + (int64_t)blockIdx.x * 16 + g * 4;
    if (a.c_f32) *reinterpret_cast<float4 *>(static_cast<float *>(a.C) + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.C) + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

enum Mx4Form { FEW_16, FEW_32, FEW_64 };
Mx4Form choose_form(const Mx4GemmArgs &a) {
    const int64_t cols16 = a.N / 16;
    if (a.M <= 16 || (a.M + 15) / 16 * cols16 <= 256) return FEW_16;
    if (a.M <= 32 || (a.M + 31) / 32 * cols16 <= 256) return FEW_32;
    return FEW_64;
}

}  // namespace

I8Plan mx4_gemm_plan(const Mx4GemmArgs &a) {
    const Mx4Form form = choose_form(a);
    return {0, form == FEW_64 ? 64 : form == FEW_32 ? 32 : 16, form == FEW_64 ? 32 : 16};
}

void launch_mx4_gemm(const Mx4GemmArgs &a, hipStream_t st) {
    if (a.M == 0) return;
    const Mx4Form form = choose_form(a);
    Mx4Params p;
    p.A = a.A; p.B = a.B; p.sa = a.sa; p.sb = a.sb; p.C = a.C; p.M = a.M; p.N = a.N; p.ldc = a.ldc; p.KB = (int)(mx4_width(a.K) / 128); p.c_f32 = a.c_f32;
    auto go = [&](auto kernel, int rows, int cols, int threads) {
        p.tiles_n = (int)((a.N + cols - 1) / cols);
        hipLaunchKernelGGL(kernel, dim3((unsigned)((a.M + rows - 1) / rows * p.tiles_n)), dim3(threads), 0, st, p);
    };
    profile_before(kTagMx4Gemm, st);
    if (form == FEW_16) go(mx4_few_kernel<1, 1, 8>, 16, 16, 512);
    else if (form == FEW_32) go(mx4_few_kernel<2, 1, 4>, 32, 16, 256);
    else go(mx4_few_kernel<4, 2, 8>, 64, 32, 512);
    profile_after(st);
}

bool mx4_token_ok(int64_t M, int64_t, int64_t) { return M <= kMx4TokenRows; }

void launch_mx4_token(const Mx4TokenArgs &a, hipStream_t st) {
    profile_before(kTagMx4Gemm, st);
    const dim3 blocks((unsigned)(a.N / 16));
    if (a.bf16) hipLaunchKernelGGL((mx4_token_kernel<true, 8>), blocks, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((mx4_token_kernel<false, 8>), blocks, dim3(512), 0, st, a);
    profile_after(st);
}

}  // namespace ssg
