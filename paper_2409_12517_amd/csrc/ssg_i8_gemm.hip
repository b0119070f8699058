// Products in 8-bit integers with a scale for each token and channel, for one matrix of weights or for those of E experts:
//
//   C[m,n] = (sum_k a[m,k] b[n,k]) sa[m] sb[n]            the sum exact, in 32-bit integers (K <= 131056)
//   h[m,n] = u g sigma(g),  u and g two such products      the gate/up form, h rounded to bf16
//
// Both operands lie in blocks of 16 rows by 64 codes in the order in which a wave holds them (see I8RowsArgs), so a block
// is one 1 KB load, to LDS or straight to registers, with nothing to permute and no LDS bank conflicts.
// With experts the rows of C are sorted by expert and every expert starts at a multiple of 16; the row tiles of all of them are listed
// on the device (see I8RowsArgs), so that nothing waits for the host, which launches for the most there can be.
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
    const int4 *tiles;           // with experts: {tiles in all, ..}, then {first row, end, expert, first tile} of each row tile
    int tiles_n;
};

typedef int v4i_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4i_t mfma_i8(const v4i_t &w, const v4i_t &x, const v4i_t &c) {
    // the weights' fragment first: a lane then holds row l & 15 of C and, in its four registers, columns 4 (l >> 4) .. + 3
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0);
}

// Which rows and columns a workgroup has.
struct I8Tile { int expert, row, row_end, col; };        // rows [row, row_end) of the expert, at most; column tile

__device__ __forceinline__ int row_tiles(const I8Params &p, int edge) {
    return p.tiles ? __builtin_amdgcn_readfirstlane(p.tiles[0].x) : (int)((p.M + edge - 1) / edge);
}
// Tile number v of row_tiles * tiles_n: the column tiles of one row tile after the other in groups of four row tiles of one
// expert, and eight contiguous ranges of that order for the eight XCDs (see map_tile).
__device__ __forceinline__ I8Tile find_tile(const I8Params &p, int edge, int rows, int v) {
    const int all = rows * p.tiles_n, full = all & ~7;
    const int t = v < full ? (v & 7) * (full >> 3) + (v >> 3) : v;
    int4 e = make_int4(0, (int)((p.M + 15) & ~(int64_t)15), 0, 0);
    if (p.tiles) e = p.tiles[1 + t / p.tiles_n];
    const int local = t - e.w * p.tiles_n, tiles = (e.y - e.x + edge - 1) / edge;
    constexpr int kGroup = 4;
    const int group = local / (kGroup * p.tiles_n), in_group = local - group * (kGroup * p.tiles_n);
    const int height = tiles - group * kGroup < kGroup ? tiles - group * kGroup : kGroup;
    I8Tile tile;
    tile.expert = __builtin_amdgcn_readfirstlane(e.z);
    tile.col = __builtin_amdgcn_readfirstlane(in_group / height);
    tile.row = __builtin_amdgcn_readfirstlane(e.x + (group * kGroup + in_group % height) * edge);
    tile.row_end = __builtin_amdgcn_readfirstlane(e.y);
    return tile;
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

// f(0) to f(N - 1), the numbers as constants
template <int N, int I = 0, class F> __device__ __forceinline__ void each(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

// A load of 16 bytes a lane to LDS in two statements, with an MFMA or two between them, which hide one or two other instructions each and
// no more: where in LDS (M0, which nothing else here uses), then the load, from a wave-uniform base and 32-bit offsets.  `no`: not if it
// is 1 (wave-uniform; the branch is inside the statement, so that the code around it stays one block).
template <int OFF> __device__ __forceinline__ void dma_to(uint32_t lds_addr) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_add_u32 m0, %0, %1" :: "s"(lds_addr), "n"(OFF) : "m0", "scc");
#endif
}
__device__ __forceinline__ void dma_from(const uint8_t *base_uniform, uint32_t lane_off) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("global_load_lds_dwordx4 %0, %1" :: "v"(lane_off), "s"(base_uniform) : "memory");
#endif
}
__device__ __forceinline__ void dma_from_unless(int no, const uint8_t *base_uniform, uint32_t lane_off) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_cmp_lg_u32 %2, 0\n\ts_cbranch_scc1 1f\n\tglobal_load_lds_dwordx4 %0, %1\n1:"
                 :: "v"(lane_off), "s"(base_uniform), "s"(no) : "memory", "scc");
#endif
}

// ---- tiles through LDS -----------------------------------------------------------------------------------
// 4 waves as 2 x 2, RB x RB blocks of 16 x 16 each (RB = 8: 256 x 256, one workgroup to a compute unit; RB = 4: 128 x 128, two).
// K advances in steps of 64 through a ring of four stages.  The fragments of a step are read while the step before it is
// multiplied, so when all waves have passed the barrier at the start of step k the stage of step k is free, and k + 4 is loaded into it.
// A workgroup has several tiles one after the other and the ring runs on from one to the next: while a tile's last steps are
// multiplied and its results stored, the first stages of the next are on their way.  A tile with no more rows than half (an expert's
// last one) loads and multiplies half of them: 4 by 8 blocks to a wave.
// Bound by the matrix cores under the chip's power: 4096 x 4096 x 11008 takes 125 to 143 us, 140 on average, 2.6 POP/s, with MFMAs in 76 % of the
// cycles at 1.75 GHz (32 x 32 x 32 MFMAs 163 where it took 148, a ring of five stages the same).  With the SwiGLU product a large tile also spends 9 us on
// its results, half of them (counted) the sigmoid, which its one wave to a SIMD cannot hide: 32768 rows of 64 experts, d = 2048, f = 1376, 226 us, 1.6 POP/s.
constexpr int kI8Stages = 4;
template <int WB> constexpr int i8_stage_bytes() { return 8 * WB * 1024; }
template <int WB, bool DUAL> __global__ __launch_bounds__(256, WB == 4 ? 1 : 2) void i8_tile_kernel(I8Params p) {
    constexpr int RB = 2 * WB, kEdge = 64 * WB, kCols = DUAL ? kEdge / 2 : kEdge, kOut = DUAL ? RB / 2 : RB;
    constexpr int kStage = i8_stage_bytes<WB>(), kRing = kI8Stages * kStage;
    constexpr int kPatch = 16 * (64 * WB + 16);          // of a wave: 16 rows of 64 WB bytes
    constexpr int kScales = 64 * WB * (DUAL ? 3 : 2) * 4;        // of a wave: its workgroup's rows' and columns'
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kRing + 4 * kPatch + 4 * kScales];
    const int rows = row_tiles(p, kEdge), all = rows * p.tiles_n;
    int v = blockIdx.x;
    if (v >= all) return;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 1, wn = w & 1;
    const int lane_id = tid & 63;
    const int KB = p.KB, col_blocks = (int)(p.N / 16);
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const uint32_t b_dst = smem_base + (4 * WB + w * WB) * 1024u;
    // The blocks of a tile that this wave loads: where its first one begins and how far the others are, wave-uniform; beyond the
    // matrix its last one again (not stored).
    struct Source {
        const uint8_t *a, *b;
        uint32_t a_off[WB], b_off[WB], a_dst;
        int half;
    };
    auto source = [&](const I8Tile &tile) {
        Source s;
        const int first_rb = tile.row / 16, last_rb = tile.row_end / 16 - 1, first_cb = tile.col * (kCols / 16);
        s.half = (int)((uint32_t)(last_rb - first_rb - RB) >> 31);       // 1: no more than RB row blocks (a truth value would leave the scalar registers)
        const int mine = (w * WB) >> s.half;             // the first row block of this wave's
        s.a_dst = smem_base + mine * 1024u;
        s.a = p.A + (int64_t)first_rb * KB * 1024;
        s.b = (DUAL && w >= 2 ? p.B2 : p.B) + ((int64_t)tile.expert * col_blocks + first_cb) * KB * 1024;
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            const int rb = first_rb + mine + j, cb = first_cb + (DUAL ? (w & 1) * WB + j : w * WB + j);
            s.a_off[j] = (uint32_t)((rb < last_rb ? rb : last_rb) - first_rb) * (uint32_t)KB * 1024u;
            s.b_off[j] = (uint32_t)((cb < col_blocks ? cb : col_blocks - 1) - first_cb) * (uint32_t)KB * 1024u;
        }
        return s;
    };
    I8Tile tile = find_tile(p, kEdge, rows, v), next_tile = tile;
    Source src = source(tile), next_src = src;
    auto scalar = [](const Source &s) {
        auto u32 = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
        auto ptr = [&](const uint8_t *x) {
            const uint64_t u = (uint64_t)(uintptr_t)x;
            return reinterpret_cast<const uint8_t *>((uintptr_t)((uint64_t)u32((uint32_t)(u >> 32)) << 32 | u32((uint32_t)u)));
        };
        Source r;
        r.a = ptr(s.a);
        r.b = ptr(s.b);
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            r.a_off[j] = u32(s.a_off[j]);
            r.b_off[j] = u32(s.b_off[j]);
        }
        r.a_dst = u32(s.a_dst);
        r.half = (int)u32((uint32_t)s.half);
        return r;
    };
    const uint32_t lane = lane_id * 16;
    // (opaque: what is computed from it for one tile is not kept for all, in registers that the main loop needs)
    auto lane_now = [&]() {
        int l = lane_id;
        asm volatile("" : "+v"(l));
        return l;
    };
    uint32_t a_lane[WB], b_lane[WB];                     // lane offsets of the blocks of `src`
    auto take_lanes = [&]() {
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            a_lane[j] = lane + src.a_off[j];
            b_lane[j] = lane + src.b_off[j];
        }
    };
    take_lanes();
    // load j of a stage into `slot`: where to, and the load
    auto issue_to = [&](auto which, uint32_t slot) {
        constexpr int j = decltype(which)::value;
        if (j < WB) dma_to<j * 1024>(src.a_dst + slot);
        else dma_to<(j - WB) * 1024>(b_dst + slot);
    };
    auto issue_from = [&](auto which) {
        constexpr int j = decltype(which)::value;
        if constexpr (j < WB / 2) dma_from(src.a, a_lane[j]);
        else if constexpr (j < WB) dma_from_unless(src.half, src.a, a_lane[j]);
        else dma_from(src.b, b_lane[j - WB]);
    };
    constexpr int kLoads = 2 * WB, kFewest = kLoads - WB / 2;            // of a stage; where the tile is half of one
    static_assert(kLoads == RB, "a load to every column of blocks");
    // After the last stage of this tile come those of the next one (of the last tile's: the same again, which nothing reads).
    // Their number is even, so that it is asked for after every second one.
    int loaded = 0;
    auto two_loaded = [&]() {
        if ((loaded += 2) == KB) {
            src = next_src;
            take_lanes();
            loaded = 0;
        }
    };
    // This tile's scales into the wave's own patch: 16 bytes to a lane, 64 WB rows and columns
    uint8_t *patch = smem + kRing + w * kPatch;
    const uint32_t scales = (uint32_t)(kRing + 4 * kPatch + w * kScales);
    auto fetch_scales = [&]() {
        const int l = lane_now();
        if (l >= 16 * WB) return;
        const int first_rb = tile.row / 16, last_rb = tile.row_end / 16 - 1, first_cb = tile.col * (kCols / 16);
        const int rb = first_rb + l / 4, cb = first_cb + l / 4;
        const float *sa = p.sa + (int64_t)(rb < last_rb ? rb : last_rb) * 16 + l % 4 * 4;
        const int64_t col = (int64_t)tile.expert * p.N + (cb < col_blocks ? cb : col_blocks - 1) * 16 + l % 4 * 4;
        dma16(reinterpret_cast<const uint8_t *>(sa), smem_base + scales);
        dma16(reinterpret_cast<const uint8_t *>(p.sb + col), smem_base + scales + 256 * WB);
        if (DUAL) dma16(reinterpret_cast<const uint8_t *>(p.sb2 + col), smem_base + scales + 512 * WB);
    };
    // the next tile, known before the loads come to it
    auto look_ahead = [&]() {
        const int n = v + (int)gridDim.x;
        if (n < all) {
            next_tile = find_tile(p, kEdge, rows, n);
            next_src = source(next_tile);
        } else {
            next_src = source(tile);
        }
    };
    look_ahead();
#pragma unroll
    for (int s = 0; s < kI8Stages; ++s) {
        each<kLoads>([&](auto j) {
            issue_to(j, s * kStage);
            asm volatile("s_nop 0");
            issue_from(j);
        });
        src.a += 1024;
        src.b += 1024;
        if (s % 2 == 1) two_loaded();
    }
    // block c of this wave's columns; with two matrices the first half of them are W1's, the others W2's same columns
    auto col_block = [&](int c) { return DUAL ? (c / (RB / 2)) * (2 * WB) + wn * (RB / 2) + c % (RB / 2) : wn * RB + c; };
    uint32_t slot = 0;                                   // of this step's stage
    wait_dma<(kI8Stages - 1) * kFewest>();               // stage 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // One tile, RA row blocks to a wave.
    auto run_tile = [&](auto row_blocks) {
        constexpr int RA = decltype(row_blocks)::value;
        v4i_t acc[RA][RB];
        v4i_t fa[2][RA], fb[2][RB];
        const uint8_t *a_frag = smem + wm * RA * 1024 + lane, *b_frag = smem + 4 * WB * 1024 + lane;
        // fragment i in the order of use: the first column's and the rows', then the other columns'
        auto read_one = [&](int set, int i, uint32_t slot) {
            if (i >= 1 && i <= RA) fa[set][i - 1] = *reinterpret_cast<const v4i_t *>(a_frag + slot + (i - 1) * 1024);
            else fb[set][i == 0 ? 0 : i - RA] = *reinterpret_cast<const v4i_t *>(b_frag + slot + col_block(i == 0 ? 0 : i - RA) * 1024);
        };
        auto step = [&](auto parity) {
            constexpr int set = decltype(parity)::value;
            const uint32_t next = slot == (kI8Stages - 1) * kStage ? 0 : slot + kStage;
            wait_dma<(kI8Stages - 2) * kFewest>();           // the next step's stage has landed
            __builtin_amdgcn_s_waitcnt(0xC07F);              // this step's fragments are here
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            constexpr int kEvery = RA * RB / (RA + RB);      // MFMAs to a fragment read
            each<RA * RB>([&](auto at) {
                constexpr int t = decltype(at)::value, c = t / RA, r = c & 1 ? RA - 1 - t % RA : t % RA;
                acc[r][c] = mfma_i8(fb[set][c], fa[set][r], acc[r][c]);
                if (t % kEvery == 0 && t / kEvery < RA + RB) read_one(set ^ 1, t / kEvery, next);
                if (t % RA == (RA > 4 ? 1 : 0)) issue_to(std::integral_constant<int, t / RA>{}, slot);
                if (t % RA == (RA > 4 ? 2 : 1)) issue_from(std::integral_constant<int, t / RA>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            src.a += 1024;
            src.b += 1024;
            slot = next;
        };
        // 16 rows at a time go through the patch, so that rows leave in pieces of 16 bytes side by side (straight from the accumulators,
        // 8 bytes of 16 rows in a store, the epilogue of the large tile took 9 us more)
        auto store = [&](auto f32) {
            const int l = lane_now();
            constexpr bool F32 = decltype(f32)::value;
            constexpr int kSize = F32 ? 4 : 2, kRowBytes = kOut * 16 * kSize < 64 * WB ? kOut * 16 * kSize : 64 * WB;
            constexpr int kPitch = kRowBytes + 16, kPart = kRowBytes / (16 * kSize);             // column blocks at a time
            constexpr int kLanes = kRowBytes / 16, kAtOnce = 64 / kLanes;        // lanes to a row, rows to a store
            static_assert(16 * kPitch <= kPatch && kOut % kPart == 0, "a part of the columns fits the patch");
            const int first_rb = tile.row / 16, last_rb = tile.row_end / 16 - 1;
            const float *sc = reinterpret_cast<const float *>(smem + scales);
#pragma unroll
            for (int r = 0; r < RA; ++r) {
                const int rb = first_rb + wm * RA + r;
                if (rb > last_rb) break;
                const float sa = sc[(wm * RA + r) * 16 + (l & 15)];
#pragma unroll
                for (int c0 = 0; c0 < kOut; c0 += kPart) {
                    const int64_t col0 = (int64_t)tile.col * kCols + (wn * kOut + c0) * 16 + (l % kLanes) * (16 / kSize);
#pragma unroll
                    for (int c = c0; c < c0 + kPart; ++c) {
                        const int at_col = (wn * kOut + c) * 16 + (l >> 4) * 4;
                        float x[4];
                        scaled4(acc[r][c], sa, *reinterpret_cast<const float4 *>(sc + 64 * WB + at_col), x);
                        if (DUAL) {
                            float g[4];
                            scaled4(acc[r][c + RB / 2], sa, *reinterpret_cast<const float4 *>(sc + 128 * WB + at_col), g);
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = swiglu_f32(x[i], g[i]);
                        }
                        uint8_t *at = patch + (l & 15) * kPitch + ((c - c0) * 16 + (l >> 4) * 4) * kSize;
                        if (F32) *reinterpret_cast<float4 *>(at) = make_float4(x[0], x[1], x[2], x[3]);
                        else *reinterpret_cast<uint2 *>(at) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
                    }
#pragma unroll
                    for (int i = 0; i < 16 / kAtOnce; ++i) {
                        const int at = i * kAtOnce + l / kLanes;
                        const uint4 x = *reinterpret_cast<const uint4 *>(patch + at * kPitch + l % kLanes * 16);
                        const int64_t row = (int64_t)rb * 16 + at;
                        if (row < p.M && col0 < p.N) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.C) + (row * p.ldc + col0) * kSize) = x;
                    }
                }
            }
        };
#pragma unroll
        for (int r = 0; r < RA; ++r)
#pragma unroll
            for (int c = 0; c < RB; ++c) {
                acc[r][c] = v4i_t{0, 0, 0, 0};
                // (else the compiler knows the zeros, has them in both halves of the register file and moves half of the accumulators
                // about in every step: 500 moves to 128 MFMAs)
                if (WB == 4) asm volatile("" : "+a"(acc[r][c]));
            }
        // (read again, though the last step of the tile before has, so that no fragments are kept across the epilogue)
#pragma unroll
        for (int i = 0; i < RA + RB; ++i) read_one(0, i, slot);
#pragma nounroll
        for (int k = 0; k < KB; k += 2) {
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            two_loaded();
        }
        wait_dma<2 * kFewest>();                             // the scales are older than the loads of the last two steps
        if (!DUAL && p.c_f32) store(std::true_type{});
        else store(std::false_type{});
    };
    for (;;) {
        // (what is the same in all lanes, said again where the two forms of a tile meet: the compiler loses sight of it)
        src = scalar(src);
        next_src = scalar(next_src);
        slot = (uint32_t)__builtin_amdgcn_readfirstlane((int)slot);
        loaded = __builtin_amdgcn_readfirstlane(loaded);
        v = __builtin_amdgcn_readfirstlane(v);
        fetch_scales();
        if (__builtin_amdgcn_readfirstlane(tile.row_end - tile.row) <= kEdge / 2) run_tile(std::integral_constant<int, RB / 2>{});
        else run_tile(std::integral_constant<int, RB>{});
        v += (int)gridDim.x;
        if (v >= all) break;
        tile = next_tile;
        look_ahead();
    }
    wait_dma<0>();                                       // (the workgroup's LDS is another's after it)
}

// ---- few rows ------------------------------------------------------------------------------------------
// RB blocks of 16 rows by CB blocks of 16 columns to a workgroup, whose waves share K out and add their sums, integers, in LDS.
// Weights and rows come straight from memory in the order of the lanes, four or eight steps' loads at a time.  Bound by the weights'
// bytes: 361 MB of 64 experts, d = 2048, f = 1376, 9 rows each, 61 us, 5.9 TB/s; small products by the loads' latency (1040 x 2736 by 333
// rows 7.6 us).  Buffering by hand doubles the registers and leaves two waves to a SIMD of eight: 132 us for those 61 + 37.
template <int RB, int CB, int WAVES, bool DUAL> __global__ __launch_bounds__(64 * WAVES) void i8_few_kernel(I8Params p) {
    constexpr int NB = DUAL ? 2 * CB : CB;
    __shared__ v4i_t part[WAVES][RB * NB][64];
    const int rows = row_tiles(p, 16 * RB);
    if ((int)blockIdx.x >= rows * p.tiles_n) return;
    const I8Tile tile = find_tile(p, 16 * RB, rows, blockIdx.x);
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

// Which kernel, from the extents alone.
// One matrix.  The smallest blocks whose workgroups the chip holds at once, one to a compute unit, since their waves share K out: 16 x 16
// (512 x 11008 by 64 rows 7.8 us, 11.3 in 32 x 16 and 19.1 in 64 x 32; 4096 x 11008 by 17 rows, where there are 512 of them, 15.6 and 13.6)
// and 32 x 16 (512 x 11008 by 256 rows 11.9, 17.4 in 64 x 32; 4096 x 4096 by 33 rows 8.8 and 8.6); up to 16 and up to 32 rows always.
// Then 64 x 32 where 128 x 128 tiles would leave three quarters of the chip idle (4096 x 11008 by 128 rows 20 us and 49 in 32 tiles;
// 1040 x 2736 by 333 7.6 and 11.6; with 96 tiles, 4096 x 4096 by 333, 21.5 and 15.6), and up to 64 rows always (11008 x 4096 17.3 and 18.2).
// Experts: blocks of 16 rows while an expert has no more on average than 12 (64 experts, d = 2048, f = 1376, 64 tokens of 8: gate/up
// 60 us, 67 in 128 x 128 tiles; with 16 rows on average 77 and 69, with 32 110 and 70).
// Between the tiles: estimated times, where a step of 64 along K takes a compute unit .52 us with two small tiles on it, .28 with
// one, .70 with a large one, and a tile 4 and 9 us beside its steps; with experts half a tile each beyond their average
// rows, and a twentieth more for the large ones.  (4096 x 4096 x 11008 131 us in large and 176 in small tiles, 2048 rows 101 and 93; gate/up of
// the 64 experts at 4096 tokens 222 and 233, at 2048 155 and 136.  Of 46 products with experts the choice takes .7 % longer on average than
// the better of the two, at most 14 %.)
enum I8Form { FEW_16, FEW_16_EXPERTS, FEW_32, FEW_64, TILE_128, TILE_256 };
I8Form choose_form(const I8GemmArgs &a, bool dual) {
    const double KB = (double)(i8_width(a.K) / 64), small_step = .52 * KB + 4, small_alone = .28 * KB + 4, large_step = .70 * KB + 9;
    auto small_time = [&](double tiles) {                // rounds of two to a compute unit, the last one perhaps of one
        const double rounds = std::floor(tiles / 512), rest = tiles - 512 * rounds;
        return rounds * small_step + (rest <= 0 ? 0 : rest <= 256 ? small_alone : small_step);
    };
    const int64_t cols = dual ? 2 * a.N : a.N, cols128 = (cols + 127) / 128, cols256 = (cols + 255) / 256;
    if (a.E == 0) {
        const int64_t tiles128 = (a.M + 127) / 128 * cols128, tiles256 = (a.M + 255) / 256 * cols256;
        const int64_t cols16 = (a.N + 15) / 16;
        // (two matrices come with experts only; should they ever come without, there are tiles for them and no other form)
        if (!dual) {
            if (a.M <= 16 || (a.M + 15) / 16 * cols16 <= 256) return FEW_16;
            if (a.M <= 32 || (a.M + 31) / 32 * cols16 <= 256) return FEW_32;
            if (a.M <= 64 || tiles128 <= 64) return FEW_64;
        }
        return (double)((tiles256 + 255) / 256) * large_step < small_time((double)tiles128) ? TILE_256 : TILE_128;
    }
    const double active = (double)std::min<int64_t>(a.E, a.rows_expected), rows = (double)a.rows_expected / active;
    if (rows <= 12) return FEW_16_EXPERTS;
    const double small = small_time(active * std::max(.6, rows / 128 + .5) * cols128);
    const double large = std::ceil(active * std::max(.6, rows / 256 + .5) * cols256 / 256) * 1.05 * large_step;
    return large < small ? TILE_256 : TILE_128;
}

int form_edge(I8Form f) { return f == TILE_256 ? 256 : f == TILE_128 ? 128 : f == FEW_64 ? 64 : f == FEW_32 ? 32 : 16; }

template <bool DUAL> void launch_form(const I8GemmArgs &a, hipStream_t st) {
    const I8Form form = choose_form(a, DUAL);
    const I8RowTiles rows = i8_row_tiles(a);
    I8Params p;
    p.A = a.A; p.B = a.B; p.B2 = a.B2; p.sa = a.sa; p.sb = a.sb; p.sb2 = a.sb2; p.C = a.C;
    p.M = a.M; p.N = a.N; p.ldc = a.ldc; p.KB = (int)(i8_width(a.K) / 64); p.c_f32 = a.c_f32; p.tiles = reinterpret_cast<const int4 *>(a.tiles);
    auto go = [&](auto kernel, int cols, int threads, int64_t most) {
        p.tiles_n = (int)((a.N + cols - 1) / cols);
        const int64_t blocks = std::min(rows.most * p.tiles_n, most);
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, st, p);
    };
    // the tiles' workgroups stay, one or two to a compute unit; a tile of no more steps than the ring has stages is a workgroup's only one
    // (its loads would run two tiles ahead)
    constexpr int64_t kAll = (int64_t)1 << 31;
    const int64_t units = p.KB > kI8Stages ? 256 : kAll;
    profile_before(DUAL ? kTagI8Swiglu : kTagI8Gemm, st);
    if (form == TILE_128) go(i8_tile_kernel<2, DUAL>, DUAL ? 64 : 128, 256, 2 * units);
    else if (form == TILE_256) go(i8_tile_kernel<4, DUAL>, DUAL ? 128 : 256, 256, units);
    else if (form == FEW_16_EXPERTS) go(i8_few_kernel<1, 1, 4, DUAL>, 16, 256, kAll);
    else if constexpr (!DUAL) {                          // (see choose_form)
        if (form == FEW_16) go(i8_few_kernel<1, 1, 8, false>, 16, 512, kAll);
        else if (form == FEW_32) go(i8_few_kernel<2, 1, 4, false>, 16, 256, kAll);
        else go(i8_few_kernel<4, 2, 8, false>, 32, 512, kAll);
    }
    profile_after(st);
}

}  // namespace

I8RowTiles i8_row_tiles(const I8GemmArgs &a) {
    const int edge = form_edge(choose_form(a, a.B2 != nullptr));
    if (a.E == 0) return {edge, (a.M + edge - 1) / edge};
    return {edge, (a.M + std::min<int64_t>(a.E, a.rows_expected) * (edge - 16)) / edge};
}

I8Plan i8_gemm_plan(const I8GemmArgs &a) {
    const I8Form form = choose_form(a, a.B2 != nullptr);
    const int edge = form_edge(form);
    if (form == TILE_256 || form == TILE_128) return {edge, edge, a.B2 ? edge / 2 : edge};
    return {0, edge, form == FEW_64 ? 32 : 16};
}

void launch_i8_gemm(const I8GemmArgs &a, hipStream_t st) {
    if (a.M == 0) return;
    if (a.B2) launch_form<true>(a, st);
    else launch_form<false>(a, st);
}

}  // namespace ssg
