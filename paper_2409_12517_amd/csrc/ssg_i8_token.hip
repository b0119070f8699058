// Products in 8-bit integers for up to four tokens: what is quantized on the way stays on the chip.
//
// A decode step is bound by the weights' bytes and, where those are few, by launches, so a workgroup quantizes the rows it needs
// itself, while its first weights are on their way: the same codes and scales as ssg_i8_rows.hip gives, and the same results as the
// other kernels, bit for bit (sums of integers, then the same operations).
//   i8_token_kernel   up to four rows by 16 columns of one matrix, or one row by 16 columns of the two matrices of the expert that
//                     an assignment (token, choice) names, with the SwiGLU product; waves share K out
//   i8_mix_kernel     16 columns of a token's result: its experts side by side, a few waves each, and their weighted sum
// One token: 11008 x 4096 9.4 us, 4.8 TB/s (13.6 in two launches); 8 experts of d = 2048, f = 1376 9 to 11 and 11 us for 45 and
// 23 MB (43 us a call in five launches, 25 in three).  What bounds them now is the start and the end of a single
// round of workgroups: x and the first weights from memory, two barriers, the sums in LDS; in the mix kernel also that one token has d / 16
// workgroups, 128 on 256 compute units there.
#include "ssg_gemm_tile.h"
#include "ssg_i8.h"

namespace ssg {

namespace {

typedef int v4i_t __attribute__((ext_vector_type(4)));
// Steps of 64 whose weights a wave loads before it multiplies; beyond its share it loads the last one again.  Microseconds, one token, by the
// steps that are a wave's share:
//   mix kernel                  3     6     8    11    16    22    28    32       token kernel   2 matrices: 4     8    16   1 matrix: 4     8    16    28
//    8 at once                8.2   8.9   8.2  12.2  12.8  16.3  20.4  18.4        4 at once             6.9  17.2  14.7            6.8   5.5   8.8  12.3
//   12                        9.2  10.2   9.0  11.5  15.2  17.1  21.9  19.9        8                     7.5  16.8  13.8            8.3   6.0   8.3  12.6
//   16                       10.8  11.7  10.5  13.1  13.8  19.5  21.0  20.5       12                     8.5  19.8  16.2            9.6   6.7   9.3  13.4
constexpr int kAtOnce = 8;

// The products of this wave's steps [k0, k1) of 64 along K: weights from `b` (1 KB a step), codes of lane l & 15's row from LDS at
// `codes`, where step k0 lies first: kAtOnce at a time, beyond the end the last step again, times zero.
template <int NB> struct Stream {
    const uint8_t *b[NB];
    int k0, k1;
    v4i_t w[kAtOnce][NB];
    __device__ __forceinline__ void load(int k) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int at = k + u < k1 ? k + u : (k1 > 0 ? k1 - 1 : 0);
#pragma unroll
            for (int c = 0; c < NB; ++c) w[u][c] = __builtin_nontemporal_load(reinterpret_cast<const v4i_t *>(b[c] + (int64_t)at * 1024));
        }
    }
    __device__ __forceinline__ void multiply(int k, const uint8_t *codes, v4i_t (&acc)[NB]) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const bool in = k + u < k1;
            const v4i_t x = *reinterpret_cast<const v4i_t *>(codes + (in ? k + u - k0 : 0) * 64) & (in ? -1 : 0);
#pragma unroll
            for (int c = 0; c < NB; ++c) acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][c], x, acc[c], 0, 0, 0);
        }
    }
};

template <bool BF16, bool DUAL, int WAVES, int ROWS> __global__ __launch_bounds__(64 * WAVES) void i8_token_kernel(I8TokenArgs a) {
    constexpr int NB = DUAL ? 2 : 1, kThreads = 64 * WAVES;
    extern __shared__ __attribute__((aligned(16))) uint8_t codes[];          // rows of Kp
    __shared__ v4i_t part[WAVES][NB][64];
    __shared__ uint32_t maxima[WAVES][ROWS];
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col_blocks = (int)(a.N / 16), KB = (int)(i8_width(a.K) / 64), Kp = KB * 64;
    const int pair = a.ids ? blockIdx.x / col_blocks : 0, cb = blockIdx.x % col_blocks;
    const int expert = a.ids ? __builtin_amdgcn_readfirstlane(a.ids[pair]) : 0;
    if (expert < 0) return;
    const int64_t from = a.ids ? pair / a.k : 0;
    const int share = (KB + WAVES - 1) / WAVES;
    Stream<NB> s;
    s.k0 = w * share < KB ? w * share : KB;
    s.k1 = s.k0 + share < KB ? s.k0 + share : KB;
#pragma unroll
    for (int c = 0; c < NB; ++c) s.b[c] = (c == 0 ? a.B : a.B2) + ((int64_t)expert * col_blocks + cb) * KB * 1024 + l * 16;
    s.load(s.k0);

    const int runs = (int)(a.K / 16), padded = Kp / 16;
    const uint8_t *src = static_cast<const uint8_t *>(a.src) + from * a.ld * (BF16 ? 2 : 4);
    const int64_t row_bytes = a.ld * (BF16 ? 2 : 4);
    uint32_t top[ROWS] = {};
    I8Run<BF16> held[ROWS];                            // this thread's first run of each row
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        held[r].clear();
        if (r < a.rows && tid < runs) held[r].load(src + r * row_bytes, tid);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        top[r] = held[r].max_bits(0);
        if (r < a.rows)
            for (int c = tid + kThreads; c < runs; c += kThreads) {
                I8Run<BF16> run;
                run.load(src + r * row_bytes, c);
                top[r] = run.max_bits(top[r]);
            }
        top[r] = wave_max_u32(I8Run<BF16>::as_f32_bits(top[r]));
        if (l == 0) maxima[w][r] = top[r];
    }
    __syncthreads();
    float scale[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) m = m > maxima[i][r] ? m : maxima[i][r];
        const I8Scale q = i8_scale(m);
        scale[r] = q.scale;
        if (r >= a.rows) continue;
        held[r].opaque();
        if (tid < padded) *reinterpret_cast<uint4 *>(codes + r * Kp + tid * 16) = held[r].codes(q.factor);
        for (int c = tid + kThreads; c < padded; c += kThreads) {
            I8Run<BF16> run;
            run.clear();
            if (c < runs) run.load(src + r * row_bytes, c);
            *reinterpret_cast<uint4 *>(codes + r * Kp + c * 16) = run.codes(q.factor);
        }
    }
    __syncthreads();
    v4i_t acc[NB] = {};
    // rows of C beyond a.rows are computed from the first row's codes and not stored
    const uint8_t *mine = codes + ((l & 15) < a.rows ? l & 15 : 0) * Kp + (l >> 4) * 16 + s.k0 * 64;
    if (s.k0 < s.k1) {
        s.multiply(s.k0, mine, acc);
        for (int k = s.k0 + kAtOnce; k < s.k1; k += kAtOnce) {
            s.load(k);
            s.multiply(k, mine, acc);
        }
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) part[w][c][l] = acc[c];
    __syncthreads();
    if (w != 0 || (l & 15) >= a.rows) return;
    v4i_t sum[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        sum[c] = part[0][c][l];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) sum[c] += part[i][c][l];
    }
    const int64_t col = (int64_t)cb * 16 + (l >> 4) * 4, row = a.ids ? pair : l & 15;
    float sa = scale[0];
#pragma unroll
    for (int r = 1; r < ROWS; ++r) sa = (l & 15) == r ? scale[r] : sa;
    const float4 s1 = *reinterpret_cast<const float4 *>(a.sb + (int64_t)expert * a.N + col);
    float v[4] = {(float)sum[0][0] * sa * s1.x, (float)sum[0][1] * sa * s1.y, (float)sum[0][2] * sa * s1.z, (float)sum[0][3] * sa * s1.w};
    if (DUAL) {
        const float4 s2 = *reinterpret_cast<const float4 *>(a.sb2 + (int64_t)expert * a.N + col);
        const v4i_t g = sum[NB - 1];
        v[0] = swiglu_f32(v[0], (float)g[0] * sa * s2.x);
        v[1] = swiglu_f32(v[1], (float)g[1] * sa * s2.y);
        v[2] = swiglu_f32(v[2], (float)g[2] * sa * s2.z);
        v[3] = swiglu_f32(v[3], (float)g[3] * sa * s2.w);
    }
    if (a.c_f32) *reinterpret_cast<float4 *>(static_cast<float *>(a.C) + row * a.ldc + col) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.C) + row * a.ldc + col) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// y[t, 16 columns]: kMixWaves waves, `split` of them to an expert, each with a share of K; h row t k + j is the expert's input.
constexpr int kMixWaves = 16;
template <bool O_F32, bool Y_F32> __global__ __launch_bounds__(64 * kMixWaves) void i8_mix_kernel(I8MixArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t codes[];          // kMixWaves shares
    __shared__ v4i_t part[kMixWaves][4];
    __shared__ float result[kMaxChosen][16], weight[kMaxChosen];
    __shared__ int chosen[kMaxChosen];
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col_blocks = (int)(a.N / 16), KB = (int)(i8_width(a.K) / 64);
    const int t = blockIdx.x / col_blocks, cb = blockIdx.x % col_blocks;
    const int split = a.split, share = (KB + split - 1) / split, at_once = kMixWaves / split;
    const int runs = (int)(a.K / 16);
    uint8_t *mine = codes + w * share * 64;
    if (tid < a.k) {
        chosen[tid] = a.ids[t * a.k + tid];
        weight[tid] = a.weights[t * a.k + tid];
    }
    for (int j0 = 0; j0 < a.k; j0 += at_once) {
        const int j = j0 + w / split;
        const int expert = w / split < at_once && j < a.k ? __builtin_amdgcn_readfirstlane(a.ids[t * a.k + j]) : -1;
        float scale = 0.0f;
        if (expert >= 0) {
            Stream<1> s;
            s.k0 = w % split * share < KB ? w % split * share : KB;
            s.k1 = s.k0 + share < KB ? s.k0 + share : KB;
            s.b[0] = a.B + ((int64_t)expert * col_blocks + cb) * KB * 1024 + l * 16;
            s.load(s.k0);
            const uint8_t *src = static_cast<const uint8_t *>(a.h) + ((int64_t)t * a.k + j) * a.K * 2;
            // the whole row's maximum in every wave, its own share's codes, of which the first run of each lane stays
            I8Run<true> held;
            held.clear();
            if (s.k0 * 4 + l < s.k1 * 4 && s.k0 * 4 + l < runs) held.load(src, s.k0 * 4 + l);
            uint32_t top = 0;
            for (int c = l; c < runs; c += 64) {
                I8Run<true> run;
                run.load(src, c);
                top = run.max_bits(top);
            }
            const I8Scale q = i8_scale(wave_max_u32(I8Run<true>::as_f32_bits(top)));
            scale = q.scale;
            held.opaque();
            if (s.k0 * 4 + l < s.k1 * 4) *reinterpret_cast<uint4 *>(mine + l * 16) = held.codes(q.factor);
            for (int c = s.k0 * 4 + l + 64; c < s.k1 * 4; c += 64) {
                I8Run<true> run;
                run.clear();
                if (c < runs) run.load(src, c);
                *reinterpret_cast<uint4 *>(mine + (c - s.k0 * 4) * 16) = run.codes(q.factor);
            }
            __threadfence_block();
            __builtin_amdgcn_wave_barrier();
            v4i_t acc[1] = {};
            const uint8_t *x = mine + (l >> 4) * 16;    // (all 16 rows the same: only one is used)
            if (s.k0 < s.k1) {
                s.multiply(s.k0, x, acc);
                for (int k = s.k0 + kAtOnce; k < s.k1; k += kAtOnce) {
                    s.load(k);
                    s.multiply(k, x, acc);
                }
            }
            if ((l & 15) == 0) part[w][l >> 4] = acc[0];
        }
        __syncthreads();
        if (expert >= 0 && w % split == 0 && (l & 15) == 0) {
            v4i_t sum = part[w][l >> 4];
            for (int i = 1; i < split; ++i) sum += part[w + i][l >> 4];
            const float4 sb = *reinterpret_cast<const float4 *>(a.sb + (int64_t)expert * a.N + cb * 16 + (l >> 4) * 4);
            float v[4] = {(float)sum[0] * scale * sb.x, (float)sum[1] * scale * sb.y, (float)sum[2] * scale * sb.z, (float)sum[3] * scale * sb.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)                 // in the type that it has where it goes through memory: a token's bits do not depend on its batch
                result[j][(l >> 4) * 4 + i] = O_F32 ? v[i] : bf16_bits_to_f32(f32_to_bf16_bits(v[i]));
        }
        __syncthreads();
    }
    if (tid >= 16) return;
    float y = 0.0f;
    for (int j = 0; j < a.k; ++j)
        if (chosen[j] >= 0) y = __fmaf_rn(weight[j], result[j][tid], y);
    const int64_t at = (int64_t)t * a.N + cb * 16 + tid;
    if (Y_F32) static_cast<float *>(a.y)[at] = y;
    else static_cast<uint16_t *>(a.y)[at] = (uint16_t)f32_to_bf16_bits(y);
}

}  // namespace

void launch_i8_token(const I8TokenArgs &a, hipStream_t st) {
    const bool dual = a.B2 != nullptr;
    const unsigned blocks = (unsigned)((a.ids ? a.pairs : 1) * (a.N / 16));
    const unsigned lds = (unsigned)(a.rows * i8_width(a.K));
    profile_before(dual ? kTagI8Swiglu : kTagI8Gemm, st);
    // one matrix has few workgroups, which take more waves each
    auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), lds, st, a); };
    auto rows = [&](auto count) {
        constexpr int ROWS = decltype(count)::value;
        if (a.bf16) go(i8_token_kernel<true, false, 8, ROWS>, 512);
        else go(i8_token_kernel<false, false, 8, ROWS>, 512);
    };
    if (dual) go(i8_token_kernel<true, true, 4, 1>, 256);
    else if (a.rows == 1) rows(std::integral_constant<int, 1>{});
    else rows(std::integral_constant<int, kTokenRows>{});
    profile_after(st);
}

// waves to an expert
static int mix_split(int k) {
    int split = 1;
    while (2 * split * k <= kMixWaves) split *= 2;
    return split;
}
static int64_t mix_lds(int64_t K, int k) { const int64_t KB = i8_width(K) / 64, s = mix_split(k); return kMixWaves * ((KB + s - 1) / s) * 64; }

// One token always.  More where every compute unit has one workgroup to quantize them for, and K enough that the launch saved is not spent
// on it: 4 tokens, 4096 x 11008 14.7 us and 15.4 in two launches, 1040 x 2736 6.6 and 7.2; 2752 x 1024 6.5 and 6.0, 11008 x 4096 17.2 and 13.7
// (2 tokens there 13.5 and 13.6, in fp32 18.7 and 14.1; 8 tokens of 4096 x 4096 11.0 and 8.5).
bool i8_token_ok(int64_t T, int64_t N, int64_t K) {
    return T * i8_width(K) <= kTokenLds && (T == 1 || (T <= kTokenRows && N <= 4096 && K >= 2048));
}
bool i8_mix_ok(int64_t T, int64_t d, int64_t f, int k) { return T <= kTokenRows && i8_width(d) <= kTokenLds && mix_lds(f, k) <= kMixLds; }

void launch_i8_mix(I8MixArgs a, hipStream_t st) {
    a.split = mix_split(a.k);
    const unsigned blocks = (unsigned)(a.T * (a.N / 16)), lds = (unsigned)mix_lds(a.K, a.k);
    profile_before(kTagI8Gemm, st);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * kMixWaves), lds, st, a); };
    if (a.y_f32) go(i8_mix_kernel<true, true>);
    else if (a.o_f32) go(i8_mix_kernel<true, false>);
    else go(i8_mix_kernel<false, false>);
    profile_after(st);
}

}  // namespace ssg
