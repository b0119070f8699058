// Products in 8-bit integers with a scale for each token and channel, for one matrix of weights or for those of E experts:
//
//   C[m,n] = (sum_k a[m,k] b[n,k]) sa[m] sb[n]            the sum exact, in 32-bit integers (K <= 131072)
//   h[m,n] = u g sigma(g),  u and g two such products      the gate/up form, h rounded to bf16
//
// Both operands lie in blocks of 16 rows by 64 codes in the order in which a wave holds them (see I8RowsArgs), so a block
// is one 1 KB load, to LDS or straight to registers, with nothing to permute and no LDS bank conflicts.
// With experts the rows of C are sorted by expert and every expert's start at a multiple of 16; a workgroup finds its expert from the
// offsets on the device, so that nothing waits for the host.
#include <cmath>

#include "ssg_gemm_tile.h"
#include "ssg_i8.h"

namespace ssg {

namespace {

struct I8Params {
    const uint8_t *A, *B, *B2;
    const float *sa, *sb, *sb2;
    void *C;
    int64_t M, N, ldc;
    int KB;                      // blocks of 64 along K
    int c_f32;
    const int *offsets;
    int E;
    int tiles_n;
};

typedef int v4i_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4i_t mfma_i8(const v4i_t &w, const v4i_t &x, const v4i_t &c) {
    // the weights' fragment first: a lane then holds row l & 15 of C and, in its four registers, columns 4 (l >> 4) .. + 3
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0);
}

// Which rows and columns a workgroup has.
struct I8Tile { int expert, row, row_end, col; };        // rows [row, row_end) of the expert, at most; column tile

// Tiles of `edge` rows, column tiles of one row tile after the other in groups of four row tiles of one expert, and
// eight contiguous ranges of that order for the eight XCDs (see map_tile).  False: no such tile.
__device__ __forceinline__ bool find_tile(const I8Params &p, int edge, int vblock, I8Tile &tile) {
    const int lane = threadIdx.x & 63;
    int total = 0;                                       // row tiles
    if (p.offsets) {
        for (int e0 = 0; e0 < p.E; e0 += 64) {
            const int e = e0 + lane;
            int n = 0;
            if (e < p.E) n = (p.offsets[e + 1] - p.offsets[e] + edge - 1) / edge;
#pragma unroll
            for (int d = 32; d > 0; d /= 2) n += __shfl_xor(n, d, 64);
            total += n;
        }
    } else {
        total = (int)((p.M + edge - 1) / edge);
    }
    const int all = total * p.tiles_n;
    if (vblock >= all) return false;
    const int full = all & ~7;
    const int t = vblock < full ? (vblock & 7) * (full >> 3) + (vblock >> 3) : vblock;
    int first = 0, tiles = total, lo = 0, hi = (int)((p.M + 15) & ~(int64_t)15), expert = 0;
    if (p.offsets) {
        const int want = t / p.tiles_n;                  // row tile in the order of experts
        int before = 0;
        for (int e0 = 0; e0 < p.E; e0 += 64) {
            const int e = e0 + lane;
            int a = 0, b = 0;
            if (e < p.E) { a = p.offsets[e]; b = p.offsets[e + 1]; }
            const int n = (b - a + edge - 1) / edge;
            int inc = n;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int o = __shfl_up(inc, d, 64);
                if (lane >= d) inc += o;
            }
            const uint64_t hit = __ballot(want >= before + inc - n && want < before + inc);
            if (hit) {
                const int at = __ffsll((unsigned long long)hit) - 1;
                first = before + __shfl(inc - n, at, 64);
                tiles = __shfl(n, at, 64);
                lo = __shfl(a, at, 64);
                hi = __shfl(b, at, 64);
                expert = e0 + at;
                break;
            }
            before += __shfl(inc, 63, 64);
        }
    }
    const int local = t - first * p.tiles_n;
    constexpr int kGroup = 4;
    const int group = local / (kGroup * p.tiles_n), in_group = local - group * (kGroup * p.tiles_n);
    const int height = tiles - group * kGroup < kGroup ? tiles - group * kGroup : kGroup;
    tile.expert = __builtin_amdgcn_readfirstlane(expert);
    tile.col = __builtin_amdgcn_readfirstlane(in_group / height);
    tile.row = __builtin_amdgcn_readfirstlane(lo + (group * kGroup + in_group % height) * edge);
    tile.row_end = __builtin_amdgcn_readfirstlane(hi);
    return true;
}

// Four neighbouring columns of a row.
__device__ __forceinline__ void store4(const I8Params &p, int64_t row, int64_t col, const float (&v)[4]) {
    if (row >= p.M) return;
    if (p.c_f32) *reinterpret_cast<float4 *>(static_cast<float *>(p.C) + row * p.ldc + col) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.C) + row * p.ldc + col) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}
__device__ __forceinline__ void scaled4(const v4i_t &acc, float sa, const float4 &sb, float (&v)[4]) {
    v[0] = __fmul_rn(__fmul_rn((float)acc[0], sa), sb.x);
    v[1] = __fmul_rn(__fmul_rn((float)acc[1], sa), sb.y);
    v[2] = __fmul_rn(__fmul_rn((float)acc[2], sa), sb.z);
    v[3] = __fmul_rn(__fmul_rn((float)acc[3], sa), sb.w);
}

// ---- tiles through LDS -----------------------------------------------------------------------------------
// 4 waves as 2 x 2, RB x RB blocks of 16 x 16 each (RB = 8: 256 x 256, one workgroup to a compute unit; RB = 4: 128 x 128, two).
// K advances in steps of 64 through a ring of five stages.  The fragments of a step are read while the step before it is
// multiplied, so when all waves have passed the barrier at the start of step k the stage of step k is free, and k + 5 is loaded into it.
constexpr int kI8Stages = 5;
template <int WB> constexpr int i8_stage_bytes() { return 8 * WB * 1024; }
template <int WB, bool DUAL> __global__ __launch_bounds__(256, WB == 4 ? 1 : 2) void i8_tile_kernel(I8Params p) {
    constexpr int RB = 2 * WB, kEdge = 64 * WB, kCols = DUAL ? kEdge / 2 : kEdge;
    constexpr int kStage = i8_stage_bytes<WB>();
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kI8Stages * kStage];
    I8Tile tile;
    if (!find_tile(p, kEdge, blockIdx.x, tile)) return;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 1, wn = w & 1;
    int l = tid & 63;
    const int KB = p.KB, col_blocks = (int)(p.N / 16);
    const int first_rb = tile.row / 16, last_rb = tile.row_end / 16 - 1;
    const int first_cb = tile.col * (kCols / 16);
    // the blocks this wave loads; beyond the matrix: its last one again (not stored)
    uint32_t a_lane[WB], b_lane[WB];
#pragma unroll
    for (int j = 0; j < WB; ++j) {
        const int rb = first_rb + w * WB + j;
        a_lane[j] = (uint32_t)((rb < last_rb ? rb : last_rb) - first_rb) * (uint32_t)KB * 1024u + l * 16;
        const int cb = first_cb + (DUAL ? (w & 1) * WB + j : w * WB + j);
        b_lane[j] = (uint32_t)((cb < col_blocks ? cb : col_blocks - 1) - first_cb) * (uint32_t)KB * 1024u + l * 16;
    }
    const uint8_t *a_src = p.A + (int64_t)first_rb * KB * 1024;
    const uint8_t *b_src = (DUAL && w >= 2 ? p.B2 : p.B) + ((int64_t)tile.expert * col_blocks + first_cb) * KB * 1024;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const uint32_t a_dst = smem_base + w * WB * 1024u, b_dst = a_dst + 4 * WB * 1024u;
    auto issue_one = [&](int j, uint32_t slot) {
        if (j < WB) dma16_s(a_src, a_lane[j], a_dst + slot + j * 1024u);
        else dma16_s(b_src, b_lane[j - WB], b_dst + slot + (j - WB) * 1024u);
    };
    // The sources stop at the last block of K: the loop issues loads in every step, the last ones into stages that nothing reads,
    // so that it is one piece of code with one count of loads to wait for.
    int loaded = 0;
    auto advance = [&]() {
        const int by = ++loaded < KB ? 1024 : 0;
        a_src += by;
        b_src += by;
    };
    constexpr int kLoads = 2 * WB;
    static_assert(kLoads == RB, "a load to every column of blocks");
    // Steps come in pairs; where their number is odd the first of a pair multiplies zeros, in the place of a step -1.
    const int odd_steps = KB & 1;
#pragma unroll
    for (int s = 0; s < kI8Stages; ++s) {
        if (s == kI8Stages - 1 && odd_steps) break;      // (step -1 loads it)
#pragma unroll
        for (int j = 0; j < kLoads; ++j) issue_one(j, s * kStage);
        advance();
    }
    v4i_t acc[RB][RB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < RB; ++c) acc[r][c] = v4i_t{0, 0, 0, 0};
    v4i_t fa[2][RB], fb[2][RB];
    const uint8_t *a_frag = smem + wm * RB * 1024 + l * 16, *b_frag = smem + 4 * WB * 1024 + l * 16;
    // block c of this wave's columns; with two matrices the first half of them are W1's, the others W2's same columns
    auto col_block = [&](int c) { return DUAL ? (c / (RB / 2)) * (2 * WB) + wn * (RB / 2) + c % (RB / 2) : wn * RB + c; };
    auto read_one = [&](int set, int i, uint32_t slot) {
        if (i % 2 == 0) fa[set][i / 2] = *reinterpret_cast<const v4i_t *>(a_frag + slot + i / 2 * 1024);
        else fb[set][i / 2] = *reinterpret_cast<const v4i_t *>(b_frag + slot + col_block(i / 2) * 1024);
    };
    wait_dma<(kI8Stages - 2) * kLoads>();                // (stage 0, and with an even number of steps stage 1)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) read_one(0, i, 0);
    if (odd_steps) {
#pragma unroll
        for (int i = 0; i < RB; ++i) fa[0][i] = v4i_t{0, 0, 0, 0};
    }
    uint32_t slot = odd_steps ? (kI8Stages - 1) * kStage : 0;        // of this step's stage
    auto step = [&](auto parity) {
        constexpr int set = decltype(parity)::value;
        const uint32_t next = slot == (kI8Stages - 1) * kStage ? 0 : slot + kStage;
        wait_dma<(kI8Stages - 2) * kLoads>();            // the next step's stage has landed
        __builtin_amdgcn_s_waitcnt(0xC07F);              // this step's fragments are here
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        constexpr int kEvery = RB / 2;                   // MFMAs to a fragment read
#pragma unroll
        for (int t = 0; t < RB * RB; ++t) {
            const int c = t / RB, r = c & 1 ? RB - 1 - t % RB : t % RB;
            acc[r][c] = mfma_i8(fb[set][c], fa[set][r], acc[r][c]);
            if (t % kEvery == 0) read_one(set ^ 1, t / kEvery, next);        // (after the last step: never used)
            if (t % RB == RB / 4) issue_one(t / RB, slot);
            __builtin_amdgcn_sched_barrier(0);
        }
        advance();
        slot = next;
    };
#pragma nounroll
    for (int k = -odd_steps; k < KB; k += 2) {
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
    }
    wait_dma<0>();                                       // (the workgroup's LDS is another's after it)
    __syncthreads();                                     // the ring is free
    asm volatile("" : "+v"(l));
    // 16 rows at a time go through a patch of LDS of the wave's own, so that rows leave in pieces of 16 bytes side by side (straight from
    // the accumulators, 8 bytes of 16 rows in a store, the epilogue of the large tile took 9 us more).  All scales are read
    // before the first store: behind one the compiler would read them again.
    constexpr int kOut = DUAL ? RB / 2 : RB;
    const float *sb = p.sb + (int64_t)tile.expert * p.N, *sb2 = DUAL ? p.sb2 + (int64_t)tile.expert * p.N : nullptr;
    float sa[RB];
    float4 s1[kOut], s2[kOut];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int rb = first_rb + wm * RB + r;
        sa[r] = p.sa[(int64_t)(rb < last_rb ? rb : last_rb) * 16 + (l & 15)];
    }
#pragma unroll
    for (int c = 0; c < kOut; ++c) {
        const int cb = first_cb + wn * kOut + c;
        const int64_t col = (int64_t)(cb < col_blocks ? cb : col_blocks - 1) * 16 + (l >> 4) * 4;
        s1[c] = *reinterpret_cast<const float4 *>(sb + col);
        if (DUAL) s2[c] = *reinterpret_cast<const float4 *>(sb2 + col);
    }
    auto store = [&](auto f32) {
        constexpr bool F32 = decltype(f32)::value;
        constexpr int kSize = F32 ? 4 : 2, kRowBytes = kOut * 16 * kSize, kPitch = kRowBytes + 16;
        constexpr int kLanes = kRowBytes / 16, kAtOnce = 64 / kLanes;        // lanes to a row, rows to a store
        static_assert(4 * 16 * kPitch <= kI8Stages * kStage, "the patches fit the ring");
        uint8_t *patch = smem + w * 16 * kPitch;
        const int64_t col0 = ((int64_t)first_cb + wn * kOut) * 16 + (l % kLanes) * (16 / kSize);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int rb = first_rb + wm * RB + r;
            if (rb > last_rb) break;
#pragma unroll
            for (int c = 0; c < kOut; ++c) {
                float v[4];
                scaled4(acc[r][c], sa[r], s1[c], v);
                if (DUAL) {
                    float g[4];
                    scaled4(acc[r][c + RB / 2], sa[r], s2[c], g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = swiglu_f32(v[i], g[i]);
                }
                uint8_t *at = patch + (l & 15) * kPitch + (c * 16 + (l >> 4) * 4) * kSize;
                if (F32) *reinterpret_cast<float4 *>(at) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint2 *>(at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            }
#pragma unroll
            for (int i = 0; i < 16 / kAtOnce; ++i) {
                const int at = i * kAtOnce + l / kLanes;
                const uint4 v = *reinterpret_cast<const uint4 *>(patch + at * kPitch + l % kLanes * 16);
                const int64_t row = (int64_t)rb * 16 + at;
                if (row < p.M && col0 < p.N) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.C) + (row * p.ldc + col0) * kSize) = v;
            }
        }
    };
    if (!DUAL && p.c_f32) store(std::true_type{});
    else store(std::false_type{});
}

// ---- few rows ------------------------------------------------------------------------------------------
// RB blocks of 16 rows by CB blocks of 16 columns to a workgroup, whose waves share K out and add their sums, integers, in LDS.
// Weights and rows come straight from memory in the order of the lanes; bound by the weights' bytes.
template <int RB, int CB, int WAVES, bool DUAL> __global__ __launch_bounds__(64 * WAVES) void i8_few_kernel(I8Params p) {
    constexpr int NB = DUAL ? 2 * CB : CB;
    __shared__ v4i_t part[WAVES][RB * NB][64];
    I8Tile tile;
    if (!find_tile(p, 16 * RB, blockIdx.x, tile)) return;
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int KB = p.KB, col_blocks = (int)(p.N / 16);
    const int first_rb = tile.row / 16, last_rb = tile.row_end / 16 - 1, first_cb = tile.col * CB;
    const uint8_t *a_src[RB], *b_src[NB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int rb = first_rb + r < last_rb ? first_rb + r : last_rb;
        a_src[r] = p.A + (int64_t)rb * KB * 1024 + l * 16;
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        const int at = first_cb + c % CB, cb = at < col_blocks ? at : col_blocks - 1;
        b_src[c] = (c < CB ? p.B : p.B2) + ((int64_t)tile.expert * col_blocks + cb) * KB * 1024 + l * 16;
    }
    const int share = (KB + WAVES - 1) / WAVES;
    const int k1 = (w + 1) * share < KB ? (w + 1) * share : KB;
    v4i_t acc[RB][NB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < NB; ++c) acc[r][c] = v4i_t{0, 0, 0, 0};
    auto steps = [&](auto count, int k) {
        constexpr int U = decltype(count)::value;
        v4i_t fa[U][RB], fb[U][NB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int c = 0; c < NB; ++c) fb[u][c] = __builtin_nontemporal_load(reinterpret_cast<const v4i_t *>(b_src[c] + (int64_t)(k + u) * 1024));
#pragma unroll
            for (int r = 0; r < RB; ++r) fa[u][r] = *reinterpret_cast<const v4i_t *>(a_src[r] + (int64_t)(k + u) * 1024);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < NB; ++c)
#pragma unroll
                for (int r = 0; r < RB; ++r) acc[r][c] = mfma_i8(fb[u][c], fa[u][r], acc[r][c]);
    };
    constexpr int U = RB + NB > 4 ? 4 : 8;
    int k = w * share;
    for (; k + U <= k1; k += U) steps(std::integral_constant<int, U>{}, k);
    for (; k + 2 <= k1; k += 2) steps(std::integral_constant<int, 2>{}, k);
    for (; k < k1; ++k) steps(std::integral_constant<int, 1>{}, k);
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < NB; ++c) part[w][r * NB + c][l] = acc[r][c];
    __syncthreads();
    const float *sb = p.sb + (int64_t)tile.expert * p.N, *sb2 = DUAL ? p.sb2 + (int64_t)tile.expert * p.N : nullptr;
    for (int i = w; i < RB * CB; i += WAVES) {
        const int r = i / CB, c = i % CB, rb = first_rb + r, cb = first_cb + c;
        if (rb > last_rb || cb >= col_blocks) continue;
        auto sum = [&](int block) {
            v4i_t v = part[0][block][l];
#pragma unroll
            for (int x = 1; x < WAVES; ++x) v += part[x][block][l];
            return v;
        };
        const int64_t row = (int64_t)rb * 16 + (l & 15), col = (int64_t)cb * 16 + (l >> 4) * 4;
        const float sa = p.sa[row];
        float v[4];
        scaled4(sum(r * NB + c), sa, *reinterpret_cast<const float4 *>(sb + col), v);
        if (DUAL) {
            float g[4];
            scaled4(sum(r * NB + CB + c), sa, *reinterpret_cast<const float4 *>(sb2 + col), g);
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = swiglu_f32(v[x], g[x]);
        }
        store4(p, row, col, v);
    }
}

// Row tiles of `edge` rows that the experts can have between them.
int64_t row_tiles_bound(const I8GemmArgs &a, int edge) {
    if (!a.offsets) return (a.M + edge - 1) / edge;
    const int64_t active = std::min<int64_t>(a.E, a.rows_expected);
    return (a.M + active * (edge - 16)) / edge;
}

// Which kernel, from the extents alone.
// One matrix.  Up to 16 and up to 32 rows the blocks that fit them.  Then 64 x 32 where 128 x 128 tiles would leave three quarters
// of the chip idle (4096 x 11008 by 128 rows 20 us and 49 in 32 tiles; 1040 x 2736 by 333 8 and 12; with 96 tiles, 4096 x 4096 by 333,
// 22 and 17), and up to 64 rows always (11008 x 4096 17.5 and 19.6).
// Experts: blocks of 16 rows while an expert has no more on average than 12, which reads weights at 6.0 TB/s (64 experts, d = 2048,
// f = 1376, 64 tokens of 8: gate/up 60 us, 69 in 128 x 128 tiles; with 16 rows on average 74 and 72, with 32 120 and 77).
// Between the tiles: estimated times, where a step of 64 along K takes a compute unit .52 us with two small tiles on it, .28 with
// one, .70 with a large one, and a tile 4 and 9 us beside its steps; with experts half a tile each beyond their average
// rows.  (4096 x 4096 x 11008 133 us in large and 176 in small tiles, 2048 rows 102 and 92; the 64 experts at 4096 tokens 223 and
// 241, at 2048 161 and 141.  Over 98 products 3 % above the better one on average, at most 14 %.)
enum I8Form { FEW_16, FEW_16_EXPERTS, FEW_32, FEW_64, TILE_128, TILE_256 };
I8Form choose_form(const I8GemmArgs &a, bool dual) {
    const double KB = (double)((a.K + 63) / 64), small_step = .52 * KB + 4, small_alone = .28 * KB + 4, large_step = .70 * KB + 9;
    const int64_t cols = dual ? 2 * a.N : a.N, cols128 = (cols + 127) / 128, cols256 = (cols + 255) / 256;
    if (!a.offsets) {
        const int64_t tiles128 = (a.M + 127) / 128 * cols128, tiles256 = (a.M + 255) / 256 * cols256;
        if (a.M <= 16) return FEW_16;
        if (a.M <= 32) return FEW_32;
        if (a.M <= 64 || tiles128 <= 64) return FEW_64;
        const int64_t rounds = tiles128 / 512, rest = tiles128 % 512;
        const double small = rounds * small_step + (rest == 0 ? 0 : rest <= 256 ? small_alone : small_step);
        return (double)((tiles256 + 255) / 256) * large_step < small ? TILE_256 : TILE_128;
    }
    const double active = (double)std::min<int64_t>(a.E, a.rows_expected), rows = (double)a.rows_expected / active;
    if (rows <= 12) return FEW_16_EXPERTS;
    const double small = active * std::max(1.0, rows / 128 + .5) * cols128 / 512 * small_step;
    const double large = std::ceil(active * std::max(1.0, rows / 256 + .5) * cols256 / 256) * large_step;
    return large < small ? TILE_256 : TILE_128;
}

template <bool DUAL> void launch_form(const I8GemmArgs &a, hipStream_t st) {
    I8Params p;
    p.A = a.A; p.B = a.B; p.B2 = a.B2; p.sa = a.sa; p.sb = a.sb; p.sb2 = a.sb2; p.C = a.C;
    p.M = a.M; p.N = a.N; p.ldc = a.ldc; p.KB = (int)((a.K + 63) / 64); p.c_f32 = a.c_f32; p.offsets = a.offsets; p.E = a.E;
    auto go = [&](auto kernel, int edge, int cols, int threads) {
        p.tiles_n = (int)((a.N + cols - 1) / cols);
        const int64_t blocks = row_tiles_bound(a, edge) * p.tiles_n;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, st, p);
    };
    profile_before(DUAL ? kTagI8Swiglu : kTagI8Gemm, st);
    switch (choose_form(a, DUAL)) {
        case FEW_16: go(i8_few_kernel<1, 1, 8, DUAL>, 16, 16, 512); break;
        case FEW_16_EXPERTS: go(i8_few_kernel<1, 1, 4, DUAL>, 16, 16, 256); break;
        case FEW_32: go(i8_few_kernel<2, 1, 4, DUAL>, 32, 16, 256); break;
        case FEW_64: go(i8_few_kernel<4, 2, 8, DUAL>, 64, 32, 512); break;
        case TILE_128: go(i8_tile_kernel<2, DUAL>, 128, DUAL ? 64 : 128, 256); break;
        case TILE_256: go(i8_tile_kernel<4, DUAL>, 256, DUAL ? 128 : 256, 256); break;
    }
    profile_after(st);
}

}  // namespace

void launch_i8_gemm(const I8GemmArgs &a, hipStream_t st) {
    if (a.M == 0) return;
    if (a.B2) launch_form<true>(a, st);
    else launch_form<false>(a, st);
}

}  // namespace ssg
