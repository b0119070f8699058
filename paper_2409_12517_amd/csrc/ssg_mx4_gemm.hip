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

// ---- tiles through LDS -----------------------------------------------------------------------------------
// 4 waves as 2 x 2, RB x RB blocks of 16 x 16 each (RB = 8: 256 x 256, one workgroup to a compute unit; RB = 4: 128 x 128, two).
// K advances in steps of 128 through a ring of four stages.  The fragments of a step are read while the step before it is
// multiplied, so when all waves have passed the barrier at the start of step k the stage of step k is free, and k + 4 is loaded into it.
// Two steps are a pair, whose scales go through a ring of their own, of three pairs: loaded before the pair's first stage, read into registers in
// the step before the pair.
// A workgroup has several tiles one after the other and the rings run on from one to the next: while a tile's last steps are
// multiplied and its results stored, the first stages of the next are on their way.  A tile with no more rows than half
// loads and multiplies half of them: 4 by 8 blocks to a wave.
constexpr int kStages = 4, kScaleSlots = 3;
template <int WB> __global__ __launch_bounds__(256, WB == 4 ? 1 : 2) void mx4_tile_kernel(Mx4Params p) {
    constexpr int RB = 2 * WB, kBlocks = 4 * WB;         // blocks of 16 rows, or columns, of a wave and of the tile
    constexpr int kStage = 2 * kBlocks * 1024, kRing = kStages * kStage;
    constexpr int kPatch = 16 * (64 * WB + 16);          // of a wave: 16 rows of 64 WB bytes
    constexpr int kScales = 2 * kBlocks * 128;           // of a pair: the rows', then the columns'
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kRing + 4 * kPatch + kScaleSlots * kScales];
    const int row_blocks = (int)((p.M + 15) / 16), col_blocks = (int)(p.N / 16);
    const int rows = (row_blocks + kBlocks - 1) / kBlocks, all = rows * p.tiles_n;
    int v = blockIdx.x;
    if (v >= all) return;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 1, wn = w & 1;
    const int lane_id = tid & 63;
    const int KB = p.KB;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const uint32_t b_dst = smem_base + (kBlocks + w * WB) * 1024u;
    // The scales that this wave loads, eight blocks' of a pair: rows' (waves 0 and 1) or columns' (2 and 3).  (A small tile has eight blocks of
    // each, which two waves load both, the same bytes to the same place.)
    const bool s_cols = w >= 2;
    const int s_first = WB == 4 ? (w & 1) * 8 : 0;
    const uint32_t s_dst = smem_base + kRing + 4 * kPatch + ((s_cols ? kBlocks : 0) + s_first) * 128u;
    // The blocks of a tile that this wave loads: where its first one begins and how far the others are, wave-uniform; beyond the
    // matrix its last one again (not stored).
    struct Source {
        const uint8_t *a, *b, *s;
        uint32_t a_off[WB], b_off[WB], a_dst, s_last;
        int half;
    };
    auto source = [&](const Mx4Tile &tile) {
        Source s;
        const int last_r = row_blocks - 1 - tile.rb, last_c = col_blocks - 1 - tile.cb;      // the last ones there are, from the tile's first on
        s.half = (int)((uint32_t)(last_r - RB) >> 31);       // 1: no more than RB row blocks
        const int mine = (w * WB) >> s.half;             // the first row block of this wave's
        s.a_dst = smem_base + mine * 1024u;
        s.a = p.A + (int64_t)tile.rb * KB * 1024;
        s.b = p.B + (int64_t)tile.cb * KB * 1024;
        s.s = s_cols ? p.sb + (int64_t)tile.cb * KB * 64 : p.sa + (int64_t)tile.rb * KB * 64;
        s.s_last = (uint32_t)(s_cols ? last_c : last_r);
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            const int r = mine + j, c = w * WB + j;
            s.a_off[j] = (uint32_t)(r < last_r ? r : last_r) * (uint32_t)KB * 1024u;
            s.b_off[j] = (uint32_t)(c < last_c ? c : last_c) * (uint32_t)KB * 1024u;
        }
        return s;
    };
    Mx4Tile tile = find_tile(p, kBlocks, kBlocks, rows, v), next_tile = tile;
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
        r.s = ptr(s.s);
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            r.a_off[j] = u32(s.a_off[j]);
            r.b_off[j] = u32(s.b_off[j]);
        }
        r.a_dst = u32(s.a_dst);
        r.s_last = u32(s.s_last);
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
    uint32_t a_lane[WB], b_lane[WB], s_lane;             // lane offsets of the blocks of `src`
    auto take_lanes = [&]() {
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            a_lane[j] = lane + src.a_off[j];
            b_lane[j] = lane + src.b_off[j];
        }
        const uint32_t block = (uint32_t)(s_first + lane_id / 8);
        s_lane = (block < src.s_last ? block : src.s_last) * (uint32_t)KB * 64u + (lane_id & 7) * 16;
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
    // the scales of the pair whose first stage is loaded next
    auto issue_scales = [&](uint32_t scale_slot) {
        dma_to<0>(s_dst + scale_slot);
        asm volatile("s_nop 0");
        dma_from(src.s, s_lane);
        src.s += 128;
    };
    auto later = [](uint32_t scale_slot, int by) {
        const uint32_t at = scale_slot + by * kScales;
        return at >= kScaleSlots * kScales ? at - kScaleSlots * kScales : at;
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
    uint8_t *patch = smem + kRing + w * kPatch;
    // the next tile, known before the loads come to it
    auto look_ahead = [&]() {
        const int n = v + (int)gridDim.x;
        if (n < all) {
            next_tile = find_tile(p, kBlocks, kBlocks, rows, n);
            next_src = source(next_tile);
        } else {
            next_src = source(tile);
        }
    };
    look_ahead();
#pragma unroll
    for (int s = 0; s < kStages; ++s) {
        if (s % 2 == 0) issue_scales(s / 2 * kScales);
        each<kLoads>([&](auto j) {
            issue_to(j, s * kStage);
            asm volatile("s_nop 0");
            issue_from(j);
        });
        src.a += 1024;
        src.b += 1024;
        if (s % 2 == 1) two_loaded();
    }
    uint32_t slot = 0, scale_slot = 0;                   // of this step's stage; of this pair's scales
    wait_dma<(kStages - 1) * kFewest + 1>();             // stage 0 and the scales before it (those of the second pair came later)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // One tile, RA row blocks to a wave.
    auto run_tile = [&](auto row_blocks_of_wave) {
        constexpr int RA = decltype(row_blocks_of_wave)::value;
        v4f_t acc[RA][RB];
        v4i_t fa[2][RA], fb[2][RB];
        uint32_t xa[RA], xb[RB], next_xa[RA], next_xb[RB];
        const uint8_t *a_frag = smem + wm * RA * 1024 + lane, *b_frag = smem + (kBlocks + wn * RB) * 1024 + lane;
        const uint8_t *a_scale = smem + kRing + 4 * kPatch + wm * RA * 128 + lane_id * 2, *b_scale = smem + kRing + 4 * kPatch + (kBlocks + wn * RB) * 128 + lane_id * 2;
        // fragment i in the order of use: the first column's and the rows', then the other columns'
        auto read_one = [&](int set, int i, uint32_t slot) {
            if (i >= 1 && i <= RA) fa[set][i - 1] = *reinterpret_cast<const v4i_t *>(a_frag + slot + (i - 1) * 1024);
            else fb[set][i == 0 ? 0 : i - RA] = *reinterpret_cast<const v4i_t *>(b_frag + slot + (i == 0 ? 0 : i - RA) * 1024);
        };
        auto read_scale = [&](int i, uint32_t slot) {
            if (i < RA) next_xa[i] = *reinterpret_cast<const uint16_t *>(a_scale + slot + i * 128);
            else next_xb[i - RA] = *reinterpret_cast<const uint16_t *>(b_scale + slot + (i - RA) * 128);
        };
        auto take_scales = [&]() {
#pragma unroll
            for (int i = 0; i < RA; ++i) xa[i] = next_xa[i];
#pragma unroll
            for (int i = 0; i < RB; ++i) xb[i] = next_xb[i];
        };
        auto step = [&](auto parity) {
            constexpr int set = decltype(parity)::value;
            const uint32_t next = slot == (kStages - 1) * kStage ? 0 : slot + kStage;
            wait_dma<(kStages - 2) * kFewest + 1>();         // the next step's stage has landed, and what came before it (of two stages one brings scales)
            __builtin_amdgcn_s_waitcnt(0xC07F);              // this step's fragments are here
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            if (set == 0) issue_scales(later(scale_slot, 2));
            const uint32_t next_scales = later(scale_slot, 1);
            constexpr int kEvery = RA * RB / (RA + RB);      // MFMAs to a fragment read
            each<RA * RB>([&](auto at) {
                constexpr int t = decltype(at)::value, c = t / RA, r = c & 1 ? RA - 1 - t % RA : t % RA;
                acc[r][c] = mfma_mx4<set>(fb[set][c], xb[c], fa[set][r], xa[r], acc[r][c]);
                if (t % kEvery == 0 && t / kEvery < RA + RB) {
                    read_one(set ^ 1, t / kEvery, next);
                    if (set == 1) read_scale(t / kEvery, next_scales);
                }
                if (t % RA == (RA > 4 ? 1 : 0)) issue_to(std::integral_constant<int, t / RA>{}, slot);
                if (t % RA == (RA > 4 ? 2 : 1)) issue_from(std::integral_constant<int, t / RA>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            src.a += 1024;
            src.b += 1024;
            slot = next;
            if (set == 1) {
                take_scales();
                scale_slot = next_scales;
            }
        };
        // 16 rows at a time go through the patch, so that rows leave in pieces of 16 bytes side by side
        auto store = [&](auto f32) {
            const int l = lane_now();
            constexpr bool F32 = decltype(f32)::value;
            constexpr int kSize = F32 ? 4 : 2, kRowBytes = RB * 16 * kSize < 64 * WB ? RB * 16 * kSize : 64 * WB;
            constexpr int kPitch = kRowBytes + 16, kPart = kRowBytes / (16 * kSize);             // column blocks at a time
            constexpr int kLanes = kRowBytes / 16, kAtOnce = 64 / kLanes;        // lanes to a row, rows to a store
            static_assert(16 * kPitch <= kPatch && RB % kPart == 0, "a part of the columns fits the patch");
#pragma unroll
            for (int r = 0; r < RA; ++r) {
                const int rb = tile.rb + wm * RA + r;
                if (rb >= row_blocks) break;
#pragma unroll
                for (int c0 = 0; c0 < RB; c0 += kPart) {
                    const int64_t col0 = (int64_t)(tile.cb + wn * RB + c0) * 16 + (l % kLanes) * (16 / kSize);
#pragma unroll
                    for (int c = c0; c < c0 + kPart; ++c) {
                        const v4f_t x = acc[r][c];
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
                acc[r][c] = v4f_t{0, 0, 0, 0};
                // (else the compiler knows the zeros, has them in both halves of the register file and moves accumulators about in every step)
                if (WB == 4) asm volatile("" : "+a"(acc[r][c]));
            }
        // (read again, though the last step of the tile before has, so that no fragments are kept across the epilogue)
#pragma unroll
        for (int i = 0; i < RA + RB; ++i) {
            read_one(0, i, slot);
            read_scale(i, scale_slot);
        }
        take_scales();
#pragma nounroll
        for (int k = 0; k < KB; k += 2) {
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            two_loaded();
        }
        if (p.c_f32) store(std::true_type{});
        else store(std::false_type{});
    };
    for (;;) {
        // (what is the same in all lanes, said again where the two forms of a tile meet: the compiler loses sight of it)
        src = scalar(src);
        next_src = scalar(next_src);
        slot = (uint32_t)__builtin_amdgcn_readfirstlane((int)slot);
        scale_slot = (uint32_t)__builtin_amdgcn_readfirstlane((int)scale_slot);
        loaded = __builtin_amdgcn_readfirstlane(loaded);
        v = __builtin_amdgcn_readfirstlane(v);
        if (__builtin_amdgcn_readfirstlane(row_blocks - tile.rb) <= RB) run_tile(std::integral_constant<int, RB / 2>{});
        else run_tile(std::integral_constant<int, RB>{});
        v += (int)gridDim.x;
        if (v >= all) break;
        tile = next_tile;
        look_ahead();
    }
    wait_dma<0>();                                       // (the workgroup's LDS is another's after it)
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

enum Mx4Form { FEW_16, FEW_32, FEW_64, TILE_128, TILE_256 };
Mx4Form choose_form(const Mx4GemmArgs &a) {
    const double KB = (double)(mx4_width(a.K) / 128), small_step = .52 * KB + 4, small_alone = .28 * KB + 4, large_step = .70 * KB + 9;
    auto small_time = [&](double tiles) {                // rounds of two to a compute unit, the last one perhaps of one
        const double rounds = std::floor(tiles / 512), rest = tiles - 512 * rounds;
        return rounds * small_step + (rest <= 0 ? 0 : rest <= 256 ? small_alone : small_step);
    };
    const int64_t cols16 = a.N / 16, tiles128 = (a.M + 127) / 128 * ((a.N + 127) / 128), tiles256 = (a.M + 255) / 256 * ((a.N + 255) / 256);
    if (a.K == 0) return FEW_64;                         // zeros: the tiles' rings want something to load
    if (a.M <= 16 || (a.M + 15) / 16 * cols16 <= 256) return FEW_16;
    if (a.M <= 32 || (a.M + 31) / 32 * cols16 <= 256) return FEW_32;
    if (a.M <= 64 || tiles128 <= 64) return FEW_64;
    return (double)((tiles256 + 255) / 256) * large_step < small_time((double)tiles128) ? TILE_256 : TILE_128;
}

}  // namespace

I8Plan mx4_gemm_plan(const Mx4GemmArgs &a) {
    const Mx4Form form = choose_form(a);
    if (form == TILE_256 || form == TILE_128) return {form == TILE_256 ? 256 : 128, 0, 0};
    return {0, form == FEW_64 ? 64 : form == FEW_32 ? 32 : 16, form == FEW_64 ? 32 : 16};
}

void launch_mx4_gemm(const Mx4GemmArgs &a, hipStream_t st) {
    if (a.M == 0) return;
    const Mx4Form form = choose_form(a);
    Mx4Params p;
    p.A = a.A; p.B = a.B; p.sa = a.sa; p.sb = a.sb; p.C = a.C; p.M = a.M; p.N = a.N; p.ldc = a.ldc; p.KB = (int)(mx4_width(a.K) / 128); p.c_f32 = a.c_f32;
    auto go = [&](auto kernel, int rows, int cols, int threads, int64_t most) {
        p.tiles_n = (int)((a.N + cols - 1) / cols);
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min((a.M + rows - 1) / rows * p.tiles_n, most)), dim3(threads), 0, st, p);
    };
    // the tiles' workgroups stay, one or two to a compute unit; a tile of no more steps than the ring has stages is a workgroup's only one
    // (its loads would run two tiles ahead)
    constexpr int64_t kAll = (int64_t)1 << 31;
    const int64_t units = p.KB > kStages ? 256 : kAll;
    profile_before(kTagMx4Gemm, st);
    if (form == TILE_256) go(mx4_tile_kernel<4>, 256, 256, 256, units);
    else if (form == TILE_128) go(mx4_tile_kernel<2>, 128, 128, 256, 2 * units);
    else if (form == FEW_16) go(mx4_few_kernel<1, 1, 8>, 16, 16, 512, kAll);
    else if (form == FEW_32) go(mx4_few_kernel<2, 1, 4>, 32, 16, 256, kAll);
    else go(mx4_few_kernel<4, 2, 8>, 64, 32, 512, kAll);
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
