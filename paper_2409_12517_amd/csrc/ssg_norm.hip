// Root-mean-square norm with the residual's addition, and its gradient:
//
//   s = x + r, rounded to r's type and kept;  rstd = 1 / sqrt(mean(s^2) + eps);  y = (s rstd) g,  g = w_offset + w
//   ds = rstd (a - n mean(a n)) + ds_in,  a = dy g,  n = s rstd;  dw = sum over rows of dy n
//
// everything in fp32.  y leaves in bf16 or fp32, as E4M3 codes under a given scale, or as rows in 8-bit integers or microscaled 4-bit floating
// point in the layout of the products that read them.
#include "ssg_device.h"
#include "ssg_i8.h"
#include "ssg_internal.h"
#include "ssg_mx4.h"

namespace ssg {

namespace {

// Eight neighbouring values of a row in their type.
template <bool BF16> struct Raw8 {
    uint4 v[BF16 ? 1 : 2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (auto &q : v) q = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load(const void *rows, int64_t at) {
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(rows) + at * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) v[i] = p[i];
    }
    __device__ __forceinline__ float value(int i) const {
        const uint4 q = v[BF16 ? 0 : i / 4];
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        if (!BF16) return __uint_as_float(words[i % 4]);
        return __uint_as_float(i % 2 ? words[i / 2] & 0xffff0000u : words[i / 2] << 16);
    }
};
__device__ __forceinline__ uint4 as_bf16(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void store8(void *rows, int64_t at, int bf16, const float (&v)[8]) {
    if (bf16) {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(rows) + at) = as_bf16(v);
    } else {
        *reinterpret_cast<float4 *>(static_cast<float *>(rows) + at) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(static_cast<float *>(rows) + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
}
// g of eight columns
__device__ __forceinline__ void factors8(const void *w, int w_bf16, float w_offset, int64_t col, float (&g)[8]) {
    if (!w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    } else if (w_bf16) {
        Raw8<true> raw;
        raw.load(w, col);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = __fadd_rn(w_offset, raw.value(j));
    } else {
        Raw8<false> raw;
        raw.load(w, col);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = __fadd_rn(w_offset, raw.value(j));
    }
}

// How a block's threads share ROWS rows: CL neighbouring threads have neighbouring runs of eight columns of a row, then come the rows, then
// the rest of the columns; a thread has HELD runs.  Either a row's threads are CL neighbours of one wave, or every wave has all the rows.
template <int THREADS, int ROWS, int CL> struct Share {
    static constexpr int kThreads = THREADS, kRows = ROWS, kCols = THREADS / ROWS, kWaves = THREADS / 64;
    static constexpr bool kOneWave = kCols == CL;
    static_assert(CL <= 64 && (kOneWave || CL * ROWS <= 64), "see above");
    static __device__ __forceinline__ int row() { return threadIdx.x / CL % ROWS; }
    static __device__ __forceinline__ int col() { return (int)threadIdx.x / (CL * ROWS) * CL + threadIdx.x % CL; }
    // op over a row's threads, in every one of them; part: the block's scratch of this call alone
    template <class T, class Op> static __device__ __forceinline__ T over_row(T v, T (*part)[ROWS], Op op) {
#pragma unroll
        for (int d = 1; d < CL; d *= 2) v = op(v, __shfl_xor(v, d, 64));
        if constexpr (!kOneWave) {
#pragma unroll
            for (int d = CL * ROWS; d < 64; d *= 2) v = op(v, __shfl_xor(v, d, 64));
            if constexpr (kWaves > 1) {
                if ((threadIdx.x & 63) < CL * ROWS && threadIdx.x % CL == 0) part[threadIdx.x / 64][row()] = v;
                __syncthreads();
                v = part[0][row()];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) v = op(v, part[w][row()]);
            }
        }
        return v;
    }
};
struct Sum { __device__ float operator()(float a, float b) const { return __fadd_rn(a, b); } };
struct Larger { __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; } };

enum { OUT_ROWS, OUT_I8, OUT_MX4 };

// RES: 0 no residual, 1 in bf16, 2 in fp32.  OUT_I8 and OUT_MX4 write the rows and columns that fill the layout up, too.
// One pass: a row stays in registers between its squares and its results.  Bound by memory: 16384 x 4096 bf16 with a bf16 residual to bf16, 537 MB, 94 us,
// 5.7 TB/s; 131072 x 128 13 us; 4096 x 4096 with an fp32 residual into 4 bits, 177 MB, 42 us, 4.2 TB/s; one row of 4096 3.7 us, a launch and the row's latency.
template <bool XBF16, int RES, int OUT, class SHARE, int HELD> __global__ __launch_bounds__(SHARE::kThreads) void norm_kernel(NormArgs a) {
    constexpr int ROWS = SHARE::kRows;
    __shared__ float sums[2][SHARE::kWaves][ROWS];
    __shared__ uint32_t tops[SHARE::kWaves][ROWS];
    const int64_t row = block_of_many() * ROWS + SHARE::row();
    if (OUT == OUT_ROWS && row - SHARE::row() >= a.T) return;
    if (OUT != OUT_ROWS && row - SHARE::row() >= i8_up(a.T, 16)) return;
    const bool live = row < a.T;
    Raw8<XBF16> x[HELD];
    Raw8<RES != 2> r[HELD];
    auto col_of = [&](int i) { return (int64_t)(SHARE::col() + i * SHARE::kCols) * 8; };
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        x[i].clear();
        if (RES) r[i].clear();
        if (live && col_of(i) < a.d) {
            x[i].load(a.x, row * a.ldx + col_of(i));
            if (RES) r[i].load(a.r, row * a.ldr + col_of(i));
        }
    }
    float s[HELD][8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] = RES ? __fadd_rn(x[i].value(j), r[i].value(j)) : x[i].value(j);
        if (RES == 1) {                                      // what is kept is what is normed
            Raw8<true> kept;
            kept.v[0] = as_bf16(s[i]);
            if (live && col_of(i) < a.d) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.r_out) + row * a.ldr + col_of(i)) = kept.v[0];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] = kept.value(j);
        }
        if (RES == 2 && live && col_of(i) < a.d) store8(a.r_out, row * a.ldr + col_of(i), 0, s[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = __fmaf_rn(s[i][j], s[i][j], sum);
    }
    sum = SHARE::over_row(sum, sums[0], Sum{});
    float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)a.d), a.eps)));
    // Squares beyond fp32, or something that is no number: again with 2^-80 s (the same answer in every wave, which all have the same rows, and
    // in every lane of a row).
    const bool over = !(sum < __uint_as_float(0x7f800000u));
    if (__builtin_expect(SHARE::kOneWave ? over : __any(over), 0)) {
        float small = 0.0f;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = __fmul_rn(s[i][j], 0x1p-80f);
                small = __fmaf_rn(v, v, small);
            }
        small = SHARE::over_row(small, sums[1], Sum{});
        if (over) rstd = __fmul_rn(0x1p-80f, __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(small, (float)a.d))));
    }
    if (a.rstd && live && SHARE::col() == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if (!live || col_of(i) >= a.d) continue;             // (s is zero there)
        float g[8];
        factors8(a.w, a.w_bf16, a.w_offset, col_of(i), g);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] = __fmul_rn(__fmul_rn(s[i][j], rstd), g[j]);
    }
    if constexpr (OUT == OUT_ROWS) {
        if (a.form == NORM_E4M3) {
            const float scale = *a.y_scale;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                if (live && col_of(i) < a.d) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(s[i][j], scale);
                    *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.y) + row * a.ldy + col_of(i)) =
                        make_uint2(satcast_pk4<kE4M3>(v[0], v[1], v[2], v[3]), satcast_pk4<kE4M3>(v[4], v[5], v[6], v[7]));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) top = Larger{}(top, abs_bits_ignore_nan(s[i][j]));
            }
            if (a.amax) {
                top = SHARE::over_row(top, tops, Larger{});
                if (live && SHARE::col() == 0) a.amax[row] = __uint_as_float(top);
            }
        } else {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (live && col_of(i) < a.d) store8(a.y, row * a.ldy + col_of(i), a.form == NORM_BF16, s[i]);
        }
    } else if constexpr (OUT == OUT_I8) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = Larger{}(top, __float_as_uint(s[i][j]) & 0x7fffffffu);
        top = SHARE::over_row(top, tops, Larger{});
        const I8Scale q = i8_scale(top);
        if (SHARE::col() == 0) static_cast<float *>(a.y_scales)[row] = q.scale;
        const int64_t padded = i8_width(a.d);
        uint8_t *out = static_cast<uint8_t *>(a.y) + (row / 16 * padded + row % 16) * 16;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int64_t col = col_of(i);
            if (col >= padded) continue;
            uint2 codes = make_uint2(0, 0);
            if (q.factor != 0.0f) codes = make_uint2(i8_codes4(s[i][0], s[i][1], s[i][2], s[i][3], q.factor), i8_codes4(s[i][4], s[i][5], s[i][6], s[i][7], q.factor));
            *reinterpret_cast<uint2 *>(out + col / 16 * 256 + col % 16) = codes;
        }
    } else {
        const int64_t padded = mx4_width(a.d);
        uint8_t *scales = static_cast<uint8_t *>(a.y_scales);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int64_t col = col_of(i);
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = Larger{}(top, __float_as_uint(s[i][j]) & 0x7fffffffu);
            top = quad_max(top);                             // (four neighbouring threads have the four runs of a block)
            if (col >= padded) continue;
            const uint32_t byte = mx4_scale_byte(top, a.ceil);
            const uint32_t codes = byte == 255u ? 0u : mx4_codes8(s[i], mx4_scale(byte));
            const int64_t block = row / 16 * (padded / 128) + col / 128;
            const int lane = (int)(col % 128 / 32 * 16 + row % 16);
            *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(a.y) + block * 1024 + lane * 16 + col % 32 / 2) = codes;
            if (col % 32 == 0) scales[block / 2 * 128 + lane * 2 + col % 256 / 128] = (uint8_t)byte;
        }
    }
}

dim3 grid_of_blocks(int64_t blocks) {                        // of up to 1024 threads (see grid_of_many)
    constexpr int64_t kRow = (int64_t)1 << 21;
    return blocks <= kRow ? dim3((unsigned)blocks) : dim3((unsigned)kRow, (unsigned)((blocks + kRow - 1) / kRow));
}

template <int N> constexpr std::integral_constant<int, N> kHeld{};

// Shares by a row's runs of eight.  Rows of the layouts go four to a block, whose pieces of 64 bytes then lie side by side (16384 x 4096 in 4 bits without a
// residual: one row to a block 55 us, two 49 to 51, four 48.6, eight 46 but 14 % more where there are few), fewer where there are few rows (300 rows
// with a residual: four 6.9 us, two 5.4).  More threads with fewer runs each start sooner: 1024 threads with two runs 131.6 us for 16384 x 4096 with an fp32
// residual, 512 with four 134, 256 with eight 153.

template <bool XBF16, int RES> void launch_norm_as(const NormArgs &a, hipStream_t st) {
    auto go = [&](auto kernel, auto share) {
        using S = decltype(share);
        const int64_t rows = a.form >= NORM_I8 ? i8_up(a.T, 16) : a.T;
        hipLaunchKernelGGL(kernel, grid_of_blocks((rows + S::kRows - 1) / S::kRows), dim3(S::kThreads), 0, st, a);
    };
    if (a.form == NORM_I8 || a.form == NORM_MX4) {
        const int64_t runs = (a.form == NORM_I8 ? i8_width(a.d) : mx4_width(a.d)) / 8;
        auto form = [&](auto out) {
            constexpr int OUT = decltype(out)::value;
            auto as = [&](auto share, auto held) { go(norm_kernel<XBF16, RES, OUT, decltype(share), decltype(held)::value>, share); };
            if constexpr (OUT == OUT_I8)                     // (4 bits fill rows up to 32 runs)
                if (runs <= 16) return as(Share<256, 16, 4>{}, kHeld<1>);
            if (runs <= 32) as(Share<256, 8, 4>{}, kHeld<1>);
            else if (runs <= 64) as(Share<256, 4, 4>{}, kHeld<1>);
            else if (runs <= 128) as(Share<256, 4, 4>{}, kHeld<2>);
            else if (runs <= 256) as(Share<512, 4, 4>{}, kHeld<2>);
            else if (runs <= 512 && a.T <= 512) as(Share<512, 2, 4>{}, kHeld<2>);
            else if (runs <= 512) as(Share<1024, 4, 4>{}, kHeld<2>);
            else if (runs <= 768) as(Share<1024, 4, 4>{}, kHeld<3>);
            else if (runs <= 1024) as(Share<1024, 4, 4>{}, kHeld<4>);
            else if (runs <= 1536) as(Share<1024, 2, 4>{}, kHeld<3>);
            else if (runs <= 2048) as(Share<1024, 2, 4>{}, kHeld<4>);
            else as(Share<1024, 1, 64>{}, kHeld<4>);
        };
        if (a.form == NORM_I8) form(std::integral_constant<int, OUT_I8>{});
        else form(std::integral_constant<int, OUT_MX4>{});
        return;
    }
    const int64_t runs = a.d / 8;
    auto as = [&](auto share, auto held) { go(norm_kernel<XBF16, RES, OUT_ROWS, decltype(share), decltype(held)::value>, share); };
    if (runs <= 8) as(Share<256, 32, 8>{}, kHeld<1>);
    else if (runs <= 16) as(Share<256, 16, 16>{}, kHeld<1>);
    else if (runs <= 32) as(Share<256, 8, 32>{}, kHeld<1>);
    else if (runs <= 64) as(Share<256, 4, 64>{}, kHeld<1>);
    else if (runs <= 128) as(Share<256, 4, 64>{}, kHeld<2>);
    else if (runs <= 256) as(Share<256, 1, 64>{}, kHeld<1>);
    else if (runs <= 512) as(Share<256, 1, 64>{}, kHeld<2>);
    else if (runs <= 768) as(Share<256, 1, 64>{}, kHeld<3>);
    else if (runs <= 1024) as(Share<256, 1, 64>{}, kHeld<4>);
    else if (runs <= 1536) as(Share<512, 1, 64>{}, kHeld<3>);
    else if (runs <= 2048) as(Share<512, 1, 64>{}, kHeld<4>);
    else as(Share<1024, 1, 64>{}, kHeld<4>);
}

// ---- the gradient ------------------------------------------------------------------------------------------
// A block takes rows by a fixed stride and keeps its columns' sums of dy n in registers; they leave as one row of `partial`.  Bound by memory: 16384 x 4096
// bf16 with the residual's gradient, 671 MB, 125 us, 5.4 TB/s; 1023 x 2736 in fp32, 56 MB, 13 us, and 4 for the second launch.  A thread has one run of a row
// where 1024 threads reach (1023 x 2736: 512 threads with one run 15.2 us for both launches, 256 with two 16.5).  Blocks for one round of the chip:
// 512 up to 6144 columns, of up to 768 threads, 256 of wider rows, of 1024 threads or of 512 with several runs each (16384 x 4096 bf16: 256 blocks 115 us, 512 76, 1024 83; 4096 x 11008: 256 60, 512 66, 1024 75).
template <bool DYBF16, bool SBF16, class SHARE, int HELD> __global__ __launch_bounds__(SHARE::kThreads) void norm_bwd_kernel(NormBwdArgs a) {
    constexpr int ROWS = SHARE::kRows, C = SHARE::kCols;
    __shared__ float sums[2][SHARE::kWaves][ROWS];
    __shared__ __attribute__((aligned(16))) float fold[ROWS == 1 ? 1 : SHARE::kThreads * 8];
    auto col_of = [&](int i) { return (int64_t)(SHARE::col() + i * C) * 8; };
    float g[HELD][8], dw[HELD][8];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[i][j] = dw[i][j] = 0.0f;
        if (col_of(i) < a.d) factors8(a.w, a.w_bf16, a.w_offset, col_of(i), g[i]);
    }
    int parity = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.T; row0 += (int64_t)gridDim.x * ROWS, parity ^= 1) {
        const int64_t row = row0 + SHARE::row();
        const bool live = row < a.T;
        Raw8<DYBF16> dy[HELD];
        Raw8<SBF16> s[HELD], ds[HELD];
        const float rstd = live ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            dy[i].clear();
            s[i].clear();
            ds[i].clear();
            if (live && col_of(i) < a.d) {
                dy[i].load(a.dy, row * a.lddy + col_of(i));
                s[i].load(a.s, row * a.lds + col_of(i));
                if (a.ds) ds[i].load(a.ds, row * a.lds + col_of(i));
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = __fmul_rn(s[i].value(j), rstd), d = dy[i].value(j);
                dw[i][j] = __fmaf_rn(d, n, dw[i][j]);
                sum = __fmaf_rn(__fmul_rn(d, g[i][j]), n, sum);
            }
        const float mean = __fdiv_rn(SHARE::over_row(sum, sums[parity], Sum{}), (float)a.d);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (!live || col_of(i) >= a.d) continue;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = __fmul_rn(s[i].value(j), rstd);
                v[j] = __fmaf_rn(rstd, __fmaf_rn(-n, mean, __fmul_rn(dy[i].value(j), g[i][j])), ds[i].value(j));
            }
            if (a.dx) store8(a.dx, row * a.lddx + col_of(i), a.dx_bf16, v);
            if (a.dr) store8(a.dr, row * a.lds + col_of(i), SBF16, v);
        }
    }
    if (!a.dw) return;
    float *out = gridDim.x == 1 ? a.dw : a.partial + (int64_t)blockIdx.x * a.d;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if constexpr (ROWS == 1) {
            if (col_of(i) < a.d) store8(out, col_of(i), 0, dw[i]);
        } else {
            store8(fold, (SHARE::row() * C + SHARE::col()) * 8, 0, dw[i]);
            __syncthreads();
            for (int e = threadIdx.x; e < C * 8; e += SHARE::kThreads) {
                float v = fold[e];
                for (int r = 1; r < ROWS; ++r) v = __fadd_rn(v, fold[r * C * 8 + e]);
                if ((int64_t)i * C * 8 + e < a.d) out[i * C * 8 + e] = v;
            }
            __syncthreads();
        }
    }
}

// The blocks' rows added up, 32 columns to a block, whose half waves share the rows out.
constexpr int kDwCols = 32, kDwShares = 32;
__global__ __launch_bounds__(kDwCols * kDwShares) void norm_dw_kernel(const float *partial, int64_t blocks, int64_t d, float *dw) {
    __shared__ float part[kDwShares][kDwCols];
    const int c = threadIdx.x % kDwCols, share = threadIdx.x / kDwCols;
    const int64_t col = (int64_t)blockIdx.x * kDwCols + c;
    float v = 0.0f;
    if (col < d) {
#pragma unroll 16
        for (int64_t b = share; b < blocks; b += kDwShares) v = __fadd_rn(v, partial[b * d + col]);
    }
    part[share][c] = v;
    __syncthreads();
    if (share != 0 || col >= d) return;
#pragma unroll
    for (int i = 1; i < kDwShares; ++i) v = __fadd_rn(v, part[i][c]);
    dw[col] = v;
}

int64_t bwd_rows(int64_t d) { return d <= 64 ? 32 : d <= 128 ? 16 : d <= 256 ? 8 : d <= 512 ? 4 : d <= 1024 ? 2 : 1; }

template <bool DYBF16, bool SBF16> void launch_norm_bwd_as(const NormBwdArgs &a, hipStream_t st) {
    const int64_t runs = a.d / 8;
    auto as = [&](auto share, auto held) {
        using S = decltype(share);
        hipLaunchKernelGGL((norm_bwd_kernel<DYBF16, SBF16, S, decltype(held)::value>), dim3((unsigned)norm_bwd_blocks(a.T, a.d)), dim3(S::kThreads), 0, st, a);
    };
    if (runs <= 8) as(Share<256, 32, 8>{}, kHeld<1>);
    else if (runs <= 16) as(Share<256, 16, 16>{}, kHeld<1>);
    else if (runs <= 32) as(Share<256, 8, 32>{}, kHeld<1>);
    else if (runs <= 64) as(Share<256, 4, 64>{}, kHeld<1>);
    else if (runs <= 128) as(Share<256, 2, 32>{}, kHeld<1>);
    else if (runs <= 256) as(Share<256, 1, 64>{}, kHeld<1>);
    else if (runs <= 512) as(Share<512, 1, 64>{}, kHeld<1>);
    else if (runs <= 768) as(Share<768, 1, 64>{}, kHeld<1>);
    else if (runs <= 1024) as(Share<1024, 1, 64>{}, kHeld<1>);
    else if (runs <= 1536) as(Share<512, 1, 64>{}, kHeld<3>);
    else if (runs <= 2048) as(Share<512, 1, 64>{}, kHeld<4>);
    else as(Share<1024, 1, 64>{}, kHeld<4>);
}

}  // namespace

void launch_norm(const NormArgs &a, hipStream_t st) {
    if (a.T == 0) return;
    profile_before(kTagNorm, st, (double)a.T * a.d * ((a.x_bf16 ? 2 : 4) + (a.r ? 2 * (a.r_bf16 ? 2 : 4) : 0) + (a.form == NORM_BF16 ? 2 : a.form == NORM_F32 ? 4 : a.form == NORM_MX4 ? 17 / 32. : 1)));
    auto residual = [&](auto x) {
        constexpr bool X = decltype(x)::value;
        if (!a.r) launch_norm_as<X, 0>(a, st);
        else if (a.r_bf16) launch_norm_as<X, 1>(a, st);
        else launch_norm_as<X, 2>(a, st);
    };
    if (a.x_bf16) residual(std::true_type{});
    else residual(std::false_type{});
    profile_after(st);
}

int64_t norm_bwd_blocks(int64_t T, int64_t d) {
    const int64_t rows = bwd_rows(d);
    return std::max<int64_t>(1, std::min<int64_t>((T + rows - 1) / rows, d <= 6144 ? 512 : 256));
}

void launch_norm_bwd(const NormBwdArgs &a, hipStream_t st) {
    profile_before(kTagNormBwd, st, (double)a.T * a.d * ((a.dy_bf16 ? 2 : 4) + (a.s_bf16 ? 2 : 4) * (1 + (a.ds != nullptr) + (a.dr != nullptr)) + (a.dx ? (a.dx_bf16 ? 2 : 4) : 0)));
    if (a.dy_bf16 && a.s_bf16) launch_norm_bwd_as<true, true>(a, st);
    else if (a.dy_bf16) launch_norm_bwd_as<true, false>(a, st);
    else if (a.s_bf16) launch_norm_bwd_as<false, true>(a, st);
    else launch_norm_bwd_as<false, false>(a, st);
    if (a.dw && norm_bwd_blocks(a.T, a.d) > 1) hipLaunchKernelGGL(norm_dw_kernel, dim3((unsigned)((a.d + kDwCols - 1) / kDwCols)), dim3(kDwCols * kDwShares), 0, st, a.partial, norm_bwd_blocks(a.T, a.d), a.d, a.dw);
    profile_after(st);
}

}  // namespace ssg
