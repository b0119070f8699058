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

// The same of 32 x 32: a lane holds row l & 31 of C and, in its sixteen registers i, columns 8 (i / 4) + 4 (l >> 5) + i % 4.
template <int STEP> __device__ __forceinline__ v16f mfma_mx4_wide(const v4i_t &w, uint32_t sw, const v4i_t &x, uint32_t sx, const v16f &c) {
    constexpr int kE2M1 = 4;
    const v8i a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, kE2M1, kE2M1, STEP, (int)sw, STEP, (int)sx);
}

// Tile number v of rows * tiles_n: the column tiles of one row tile after the other in groups of four row tiles, and eight contiguous
// ranges of that order for the eight XCDs.  Each group starts TURN columns behind the one before: from the same column on, XCDs whose ranges start
// with a group would write one part of every row at the same time, and with it a part of the memory's channels (fp32 results 4096 x 16384 x 2048 160 us,
// 112 turned; 4096 x 16384 x 512 in small tiles 93 and 70; 4096 x 11008 x 512 65 and 47; bf16 4096 x 16384 x 2048 103 and 88; at worst 8192 x 4096 x 512 39.9 and 41.7).
constexpr int kGroup = 4;
struct Mx4Tile { int rb, cb; };                          // first row block and column block
template <int TURN> __device__ __forceinline__ Mx4Tile find_tile(const Mx4Params &p, int row_blocks, int col_blocks, int rows, int v) {
    const int all = rows * p.tiles_n, full = all & ~7;
    const int t = v < full ? (v & 7) * (full >> 3) + (v >> 3) : v;
    const int group = t / (kGroup * p.tiles_n), in_group = t - group * (kGroup * p.tiles_n);
    const int height = rows - group * kGroup < kGroup ? rows - group * kGroup : kGroup;
    int col = in_group / height;
    if (TURN > 0) col = (col + group * TURN) % p.tiles_n;
    return {__builtin_amdgcn_readfirstlane((group * kGroup + in_group % height) * row_blocks), __builtin_amdgcn_readfirstlane(col * col_blocks)};
}

// Four neighbouring columns of a row.
__device__ __forceinline__ void store4(const Mx4Params &p, int64_t row, int64_t col, const v4f_t &v) {
    if (row >= p.M) return;
    if (p.c_f32) *reinterpret_cast<float4 *>(static_cast<float *>(p.C) + row * p.ldc + col) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.C) + row * p.ldc + col) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// ---- tiles through LDS -----------------------------------------------------------------------------------
// 4 waves as 2 x 2, TA x TB blocks of 32 x 32 each.
// Products of 32 x 32 x 64, whose rate, with one wave to a SIMD, the power bounds where 16 x 16 x 128 wait on their issue (registers alone, random codes, launches of
// .02 to 18 ms: 5.0 to 6.1 PFLOP/s and 3.7 to 5.2): a fragment is the blocks of two neighbouring 16 rows, half of each along K.
// K advances in steps of 128 through a ring of kStages stages, each in two halves of 64.  The fragments of a half are read while the half before it is
// multiplied, so when all waves have passed the barrier in the middle of step k, everything of its stage is in registers, and k + kStages is loaded
// into it.  Two steps are a pair, whose scales go through a ring of their own, of two pairs: loaded before the pair's first stage, read into
// registers, those of either half while the other half is multiplied.
// A workgroup has several tiles one after the other and the rings run on from one to the next: while a tile's last steps are
// multiplied and its results stored, the first stages of the next are on their way.  A tile with no more rows than half
// loads and multiplies half of them.
// Bound by the matrix cores under the chip's power: 4096 x 4096 x 11008 takes 83 to 85 us, 4.4 PFLOP/s, the MFMAs half of the cycles at 2.1 GHz; without its
// loads to LDS 75, without those, the reads and the stores 67; operands of zeros 59.  4096 x 11008 x 4096 99 us:
// 688 tiles are 2.7 rounds of 256, and the stores of a round take half a step's time from the loads behind them.  8192^3 238 us, 4.6 PFLOP/s.  (16 x 16 x 128
// MFMAs 103 us for 85; results through LDS and the wait for their stores before the next tile's first step 113 for 100; tiles of 128 x 256 twice on a
// compute unit, three stages each, 91 for 85 and 110 for 100; non-temporal stores, groups of two or eight row tiles, loads all at once: within 4 %.)
constexpr int kStages = 4, kScaleSlots = 2;
static_assert(kStages % 2 == 0, "a pair's scales come with the first of two stages, and a tile's last stage with the second of a pair of steps");
template <int TA, int TB> struct TileShape {
    static constexpr int kA = 4 * TA, kB = 4 * TB;       // blocks of 16 rows, and of 16 columns, of the tile
    static constexpr int kStage = (kA + kB) * 1024, kRing = kStages * kStage;
    static constexpr int kScales = (kA + kB) * 128;      // of a pair: the rows', then the columns'
    static constexpr int kLds = kRing + kScaleSlots * kScales, kAtOnce = 163840 / kLds;
    static constexpr int kTurn = 32 * kAtOnce / kGroup;  // columns that an XCD's compute units have at once
};
// wait_dma, unless `no` is above zero (wave-uniform)
template <int N> __device__ __forceinline__ void wait_dma_unless(int no) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_cmp_gt_i32 %1, 0\n\ts_cbranch_scc1 1f\n\ts_waitcnt vmcnt(%0)\n1:" :: "n"(N), "s"(no) : "memory", "scc");
#endif
}
// a's lanes 32 to 63 for b's lanes 0 to 31; of each 32, a's lanes 16 to 31 for b's 0 to 15
__device__ __forceinline__ void swap32(uint32_t &a, uint32_t &b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0]; b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t &a, uint32_t &b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0]; b = r[1];
}

// Tiles v, v + stride, ..
template <int TA, int TB> __device__ __forceinline__ void run_tiles(const Mx4Params &p, uint8_t *smem, int v, const int stride) {
    using Shape = TileShape<TA, TB>;
    constexpr int kA = Shape::kA, kB = Shape::kB, kStage = Shape::kStage, kRing = Shape::kRing, kScales = Shape::kScales;
    const int row_blocks = (int)((p.M + 15) / 16), col_blocks = (int)(p.N / 16);
    const int rows = (row_blocks + kA - 1) / kA, all = rows * p.tiles_n;
    if (v >= all) return;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 1, wn = w & 1;
    const int lane_id = tid & 63;
    const int KB = p.KB;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const uint32_t b_dst = smem_base + (kA + w * TB) * 1024u;
    // The scales that this wave loads, those of eight blocks of a pair, rows or columns (where there are fewer than four times eight, the last waves load
    // the same bytes to the same place).
    constexpr int kPieces = (kA + kB) / 8;
    const int piece = w < kPieces ? w : kPieces - 1;
    const bool s_cols = piece >= kA / 8;
    const int s_first = s_cols ? (piece - kA / 8) * 8 : piece * 8;
    const uint32_t s_dst = smem_base + kRing + piece * 1024u;
    // The blocks of a tile that this wave loads: where its first one begins and how far the others are, wave-uniform; beyond the
    // matrix its last one again (not stored).
    struct Source {
        const uint8_t *a, *b, *s;
        uint32_t a_off[TA], b_off[TB], a_dst, s_last;
        int half;
    };
    auto source = [&](const Mx4Tile &tile) {
        Source s;
        const int last_r = row_blocks - 1 - tile.rb, last_c = col_blocks - 1 - tile.cb;      // the last ones there are, from the tile's first on
        s.half = (int)((uint32_t)(last_r - kA / 2) >> 31);   // 1: no more than half of the row blocks
        const int mine = (w * TA) >> s.half;             // the first row block of this wave's
        s.a_dst = smem_base + mine * 1024u;
        s.a = p.A + (int64_t)tile.rb * KB * 1024;
        s.b = p.B + (int64_t)tile.cb * KB * 1024;
        s.s = s_cols ? p.sb + (int64_t)tile.cb * KB * 64 : p.sa + (int64_t)tile.rb * KB * 64;
        s.s_last = (uint32_t)(s_cols ? last_c : last_r);
#pragma unroll
        for (int j = 0; j < TA; ++j) s.a_off[j] = (uint32_t)(mine + j < last_r ? mine + j : last_r) * (uint32_t)KB * 1024u;
#pragma unroll
        for (int j = 0; j < TB; ++j) s.b_off[j] = (uint32_t)(w * TB + j < last_c ? w * TB + j : last_c) * (uint32_t)KB * 1024u;
        return s;
    };
    Mx4Tile tile = find_tile<Shape::kTurn>(p, kA, kB, rows, v), next_tile = tile;
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
        for (int j = 0; j < TA; ++j) r.a_off[j] = u32(s.a_off[j]);
#pragma unroll
        for (int j = 0; j < TB; ++j) r.b_off[j] = u32(s.b_off[j]);
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
    uint32_t a_lane[TA], b_lane[TB], s_lane;             // lane offsets of the blocks of `src`
    auto take_lanes = [&]() {
#pragma unroll
        for (int j = 0; j < TA; ++j) a_lane[j] = lane + src.a_off[j];
#pragma unroll
        for (int j = 0; j < TB; ++j) b_lane[j] = lane + src.b_off[j];
        // in LDS, for every two blocks, what the 64 lanes read for a half lies side by side: half, run of 32, block, 8 rows
        const uint32_t block = (uint32_t)(s_first + (lane_id >> 4) * 2 + (lane_id >> 1 & 1));
        s_lane = (block < src.s_last ? block : src.s_last) * (uint32_t)KB * 64u + (lane_id >> 2 & 3) * 32 + (lane_id & 1) * 16;
    };
    take_lanes();
    // load j of a stage into `slot`: where to, and the load
    auto issue_to = [&](auto which, uint32_t slot) {
        constexpr int j = decltype(which)::value;
        if (j < TA) dma_to<j * 1024>(src.a_dst + slot);
        else dma_to<(j - TA) * 1024>(b_dst + slot);
    };
    auto issue_from = [&](auto which) {
        constexpr int j = decltype(which)::value;
        if constexpr (j < TA / 2) dma_from(src.a, a_lane[j]);
        else if constexpr (j < TA) dma_from_unless(src.half, src.a, a_lane[j]);
        else dma_from(src.b, b_lane[j - TA]);
    };
    // the scales of the pair whose first stage is loaded next
    auto issue_scales = [&](uint32_t scale_slot) {
        dma_to<0>(s_dst + scale_slot);
        asm volatile("s_nop 0");
        dma_from(src.s, s_lane);
        src.s += 128;
    };
    constexpr int kLoads = TA + TB, kFewest = kLoads - TA / 2;           // of a stage; where the tile is half of one
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
    // the next tile, known before the loads come to it
    auto look_ahead = [&]() {
        const int n = v + stride;
        if (n < all) {
            next_tile = find_tile<Shape::kTurn>(p, kA, kB, rows, n);
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
    wait_dma<(kStages - 1) * kFewest + 1>();              // stage 0 and the scales before it (those of the second pair came later)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // Steps of a tile whose wait there is none for: before the last tile's results were stored, all that was loaded had landed.  (A wait for a
    // load waits for the older stores, too, so those get the time of these steps.)
    int waited = 0;
    // One tile, QA blocks of 32 rows to a wave.
    auto run_tile = [&](auto blocks_of_wave) {
        constexpr int QA = decltype(blocks_of_wave)::value, QB = TB;
        v16f acc[QA][QB];
        v4i_t fa[2][QA], fb[2][QB];                      // of the two halves
        uint32_t xa[2][QA], xb[2][QB];
        // lanes 0 to 15 and 32 to 47 have the first block's rows, 16 to 31 and 48 to 63 the second's; the upper half of the lanes the next run of 32
        const int l16 = lane_id & 15, lhi = lane_id >> 4 & 1, run = lane_id >> 5;
        const uint32_t frag_lane = lhi * 1024 + run * 256 + l16 * 16, scale_lane = run * 64 + lhi * 32 + l16 * 2;
        const uint8_t *a_frag = smem + wm * QA * 2048 + frag_lane, *b_frag = smem + (kA + wn * 2 * TB) * 1024 + frag_lane;
        const uint8_t *a_scale = smem + kRing + wm * QA * 256 + scale_lane, *b_scale = smem + kRing + (kA + wn * 2 * TB) * 128 + scale_lane;
        // fragment i of a half in the order of use: the first column's and the rows', then the other columns'
        auto read_one = [&](int half, int i, uint32_t slot) {
            if (i >= 1 && i <= QA) fa[half][i - 1] = *reinterpret_cast<const v4i_t *>(a_frag + slot + half * 512 + (i - 1) * 2048);
            else fb[half][i == 0 ? 0 : i - QA] = *reinterpret_cast<const v4i_t *>(b_frag + slot + half * 512 + (i == 0 ? 0 : i - QA) * 2048);
        };
        auto read_scale = [&](int half, int i, uint32_t slot) {
            if (i < QA) xa[half][i] = *reinterpret_cast<const uint16_t *>(a_scale + slot + half * 128 + i * 256);
            else xb[half][i - QA] = *reinterpret_cast<const uint16_t *>(b_scale + slot + half * 128 + (i - QA) * 256);
        };
        // One half of a step; `other`: what is read and loaded between the MFMAs.
        auto multiply = [&](auto parity, auto half, auto &&other) {
            constexpr int P = decltype(parity)::value, H = decltype(half)::value;
            each<QA * QB>([&](auto at) {
                constexpr int t = decltype(at)::value, c = t / QA, r = c & 1 ? QA - 1 - t % QA : t % QA;
                acc[r][c] = mfma_mx4_wide<P>(fb[H][c], xb[H][c], fa[H][r], xa[H][r], acc[r][c]);
                other(at);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        constexpr int kMfmas = QA * QB, kReads = QA + QB, kReadsEach = (kReads + kMfmas - 1) / kMfmas, kLoadsEach = (kLoads + kMfmas - 1) / kMfmas;
        auto step = [&](auto parity) {
            constexpr int P = decltype(parity)::value;
            const uint32_t next = slot == (kStages - 1) * kStage ? 0 : slot + kStage, next_scales = scale_slot ^ kScales;
            multiply(parity, std::integral_constant<int, 0>{}, [&](auto at) {
                constexpr int t = decltype(at)::value;
#pragma unroll
                for (int i = t * kReadsEach; i < (t + 1) * kReadsEach && i < kReads; ++i) {
                    read_one(1, i, slot);
                    if (P == 0) read_scale(1, i, scale_slot);
                }
            });
            // the next step's stage has landed, and the scales before it: of two stages after it one brings scales
            wait_dma_unless<(kStages - 2) * kFewest + (kStages - 2) / 2>(waited);
            --waited;
            __builtin_amdgcn_s_waitcnt(0xC07F);              // all of this step's fragments are here
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            if (P == 0) issue_scales(scale_slot);
            multiply(parity, std::integral_constant<int, 1>{}, [&](auto at) {
                constexpr int t = decltype(at)::value;
#pragma unroll
                for (int i = t * kReadsEach; i < (t + 1) * kReadsEach && i < kReads; ++i) {
                    read_one(0, i, next);
                    if (P == 1) read_scale(0, i, next_scales);
                }
                if constexpr (kMfmas >= 2 * kLoads) {
                    if constexpr (t % 2 == 0 && t / 2 < kLoads) issue_to(std::integral_constant<int, t / 2>{}, slot);
                    if constexpr (t % 2 == 1 && t / 2 < kLoads) issue_from(std::integral_constant<int, t / 2>{});
                } else {
                    each<kLoadsEach>([&](auto i) {
                        constexpr int j = t * kLoadsEach + decltype(i)::value;
                        if constexpr (j < kLoads) {
                            issue_to(std::integral_constant<int, j>{}, slot);
                            asm volatile("s_nop 0");
                            issue_from(std::integral_constant<int, j>{});
                        }
                    });
                }
            });
            // (else the compiler moves all the MFMAs, whose results nothing else in the block reads, behind the block's reads and loads)
#pragma unroll
            for (int r = 0; r < QA; ++r)
#pragma unroll
                for (int c = 0; c < QB; ++c) {
                    if (TA * TB > 8) asm volatile("" : "+a"(acc[r][c]));
                    else asm volatile("" : "+v"(acc[r][c]));
                }
            src.a += 1024;
            src.b += 1024;
            slot = next;
            if (P == 1) scale_slot = next_scales;
            if (P == 1) two_loaded();
        };
        // A lane has row l % 32 of a block and of each eight columns four, those from 4 (l / 32) on.  Exchanged between lanes until one store takes 64 bytes of
        // each of 16 rows.
        auto store = [&](auto f32) {
            const int l = lane_now();
            constexpr bool F32 = decltype(f32)::value;
            const int piece_of_lane = (l >> 4 & 1) * 2 + (l >> 5);
#pragma unroll
            for (int r = 0; r < QA; ++r) {
                const int64_t row0 = (int64_t)(tile.rb + (wm * QA + r) * 2) * 16;
                if (row0 >= p.M) break;
#pragma unroll
                for (int c = 0; c < QB; ++c) {
                    const int64_t col0 = (int64_t)(tile.cb + (wn * TB + c) * 2) * 16;
                    auto put = [&](int64_t row, int64_t col, const uint32_t (&q)[4]) {
                        if (row < p.M && col < p.N)
                            *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.C) + (row * p.ldc + col) * (F32 ? 4 : 2)) = make_uint4(q[0], q[1], q[2], q[3]);
                    };
                    if constexpr (F32) {
#pragma unroll
                        for (int i = 0; i < 16; i += 8) {        // columns 2 i .. 2 i + 15
                            uint32_t x[4], y[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                x[j] = __float_as_uint(acc[r][c][i + j]);
                                y[j] = __float_as_uint(acc[r][c][i + 4 + j]);
                                swap16(x[j], y[j]);
                            }
                            put(row0 + (l & 15), col0 + 2 * i + piece_of_lane * 4, x);
                            put(row0 + 16 + (l & 15), col0 + 2 * i + piece_of_lane * 4, y);
                        }
                    } else {
                        uint32_t x[4], y[4];                     // of columns 0 to 15 and 16 to 31
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            x[j] = pack_bf16x2(acc[r][c][2 * j], acc[r][c][2 * j + 1]);
                            x[2 + j] = pack_bf16x2(acc[r][c][4 + 2 * j], acc[r][c][4 + 2 * j + 1]);
                            y[j] = pack_bf16x2(acc[r][c][8 + 2 * j], acc[r][c][8 + 2 * j + 1]);
                            y[2 + j] = pack_bf16x2(acc[r][c][12 + 2 * j], acc[r][c][12 + 2 * j + 1]);
                            swap32(x[j], x[2 + j]);
                            swap32(y[j], y[2 + j]);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) swap16(x[j], y[j]);
                        put(row0 + (l & 15), col0 + piece_of_lane * 8, x);
                        put(row0 + 16 + (l & 15), col0 + piece_of_lane * 8, y);
                    }
                }
            }
        };
#pragma unroll
        for (int r = 0; r < QA; ++r)
#pragma unroll
            for (int c = 0; c < QB; ++c) {
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[r][c][i] = 0.0f;
                // (else the compiler knows the zeros, has them in both halves of the register file and moves accumulators about in every step)
                if (TA * TB > 8) asm volatile("" : "+a"(acc[r][c]));
            }
        // (read again, though the last step of the tile before has, so that no fragments are kept across the epilogue)
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            read_one(0, i, slot);
            read_scale(0, i, scale_slot);
        }
#pragma nounroll
        for (int k = 0; k < KB; k += 2) {
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
        }
        wait_dma<0>();
        waited = kStages - 1;
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
        waited = __builtin_amdgcn_readfirstlane(waited);
        v = __builtin_amdgcn_readfirstlane(v);
        if (__builtin_amdgcn_readfirstlane(row_blocks - tile.rb) <= kA / 2) run_tile(std::integral_constant<int, TA / 2>{});
        else run_tile(std::integral_constant<int, TA>{});
        v += stride;
        if (v >= all) break;
        tile = next_tile;
        look_ahead();
    }
    wait_dma<0>();                                       // (the workgroup's LDS is another's after it)
}
template <int TA, int TB> __global__ __launch_bounds__(256, (TileShape<TA, TB>::kAtOnce)) void mx4_tile_kernel(Mx4Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[TileShape<TA, TB>::kLds];
    run_tiles<TA, TB>(p, smem, blockIdx.x, gridDim.x);
}
// Two products' tiles side by side, those of the first below `first`, one to a workgroup.
template <int TA, int TB> __global__ __launch_bounds__(256, (TileShape<TA, TB>::kAtOnce)) void mx4_tile_pair_kernel(Mx4Params a, Mx4Params b, int first) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[TileShape<TA, TB>::kLds];
    const bool in_first = (int)blockIdx.x < first;
    const Mx4Params p = in_first ? a : b;
    run_tiles<TA, TB>(p, smem, (int)blockIdx.x - (in_first ? 0 : first), gridDim.x);
}

// Two products one after the other in the same workgroups.  The second's tiles are counted from the last workgroup, so that those that had one more
// of the first product's have one less of them.  Backward passes of M rows, N -> K, whole, in two launches and in this one: 4096 x 11008 -> 4096 239 233 us;
// 5000 x 2736 -> 8192 185 170; 5608 x 8704 -> 4432 278 251; 3212 x 2416 -> 11136 166 153; of 20 large ones 2 % less time, at worst 1.4 % more.  (Half of
// the workgroups with the products the other way round, so that results of some are stored while others multiply: 1.5 % less, at worst 13 % more.)
template <int TA, int TB> __global__ __launch_bounds__(256, (TileShape<TA, TB>::kAtOnce)) void mx4_tile_both_kernel(Mx4Params a, Mx4Params b) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[TileShape<TA, TB>::kLds];
#pragma nounroll
    for (int i = 0; i < 2; ++i) {
        const Mx4Params p = i ? b : a;
        run_tiles<TA, TB>(p, smem, i ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x, gridDim.x);
        __syncthreads();                                 // (every wave is through with the first one's LDS)
    }
}

// ---- few rows ------------------------------------------------------------------------------------------
// RB blocks of 16 rows by CB blocks of 16 columns to a workgroup, whose waves share K out in pairs of blocks and add their sums in LDS, wave after
// wave.  Both operands come straight from memory in the order of the lanes, U pairs' loads at a time.  Bound by the weights' bytes and by the start
// and end of one round of workgroups: 24 MB of 4096 x 11008 by up to 16 rows 7.0 us, 9 MB of 4096 x 4096 4.2.
template <int RB, int CB, int WAVES> __global__ __launch_bounds__(64 * WAVES) void mx4_few_kernel(Mx4Params p) {
    __shared__ v4f_t part[WAVES][RB * CB][64];
    const int row_blocks = (int)((p.M + 15) / 16), col_blocks = (int)(p.N / 16), pairs = p.KB / 2;
    const Mx4Tile tile = find_tile<0>(p, RB, CB, (row_blocks + RB - 1) / RB, blockIdx.x);
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
    if (U > 2 && at + 2 <= p1) {
        steps(std::integral_constant<int, 2>{}, at);
        at += 2;
    }
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

// ---- few rows, quantized on the way ---------------------------------------------------------------------------
// 16 columns to a workgroup, whose waves share K out.  Its threads quantize the rows, a block each, into LDS while the first weights are on their way.
// (In the registers of the lanes that multiply them, where four of 64 have a row's values, the vector ALU took 3 us: 1 x 4096 -> 11008
// 10.6 us for 7.7.)  Bound by the weights' bytes, 24 MB there, 4.7 us, by the start and end of one round of workgroups, and by loads that nothing needs: U pairs are asked
// for at a time whatever a wave's share is, those beyond it its last one again (32 pairs for 16 at K = 4096, 60 for 43 at 11008).  The rows in LDS lie a multiple of 128
// bytes apart, so that the rows of 16 lanes share banks.
template <bool BF16, int WAVES> __global__ __launch_bounds__(64 * WAVES) void mx4_token_kernel(Mx4TokenArgs a) {
    constexpr int U = 4;                                     // pairs of blocks at a time
    extern __shared__ __attribute__((aligned(16))) uint8_t codes[];          // rows of Kp / 2, then their scales, rows of Kp / 32
    __shared__ v4f_t part[WAVES][64];
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = l >> 4;
    const int pairs = (int)(mx4_width(a.K) / 256), share = (pairs + WAVES - 1) / WAVES;
    const int p0 = w * share < pairs ? w * share : pairs, p1 = p0 + share < pairs ? p0 + share : pairs;
    const uint8_t *b = a.B + (int64_t)blockIdx.x * pairs * 2048 + l * 16, *sb = a.sb + (int64_t)blockIdx.x * pairs * 128 + l * 2;
    v4i_t f[U][2];
    uint32_t sw[U];
    auto load = [&](int at) {                                // beyond the share its last pair again, or the first there is
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = at + u < p1 ? at + u : p1 > p0 ? p1 - 1 : 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) f[u][h] = __builtin_nontemporal_load(reinterpret_cast<const v4i_t *>(b + (int64_t)k * 2048 + h * 1024));
            sw[u] = *reinterpret_cast<const uint16_t *>(sb + (int64_t)k * 128);
        }
    };
    load(p0);
    const int blocks = pairs * 8;                            // of a row
    uint8_t *scales = codes + a.rows * blocks * 16;
    for (int i = tid; i < a.rows * blocks; i += 64 * WAVES) {
        const int r = i / blocks, k = i % blocks;
        Mx4Block<BF16> v;
        v.load(static_cast<const uint8_t *>(a.x) + r * a.ld * (BF16 ? 2 : 4), k * 32, a.K, true);
        const uint32_t byte = mx4_scale_byte(v.top_bits(), a.ceil);
        *reinterpret_cast<uint4 *>(codes + i * 16) = v.codes(byte);
        scales[i] = (uint8_t)byte;
    }
    __syncthreads();
    // rows of C beyond a.rows are computed from the first row and not stored
    const int mine = ((l & 15) < a.rows ? l & 15 : 0) * blocks + g;
    v4f_t acc = {0, 0, 0, 0};
    for (int at = p0; at < p1; at += U) {
        if (at > p0) load(at);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at + u >= p1) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = mine + (at + u) * 8 + h * 4;
                const v4i_t x = *reinterpret_cast<const v4i_t *>(codes + k * 16);
                acc = mfma_mx4<0>(f[u][h], sw[u] >> 8 * h, x, scales[k], acc);
            }
        }
    }
    part[w][l] = acc;
    __syncthreads();
    if (w != 0 || (l & 15) >= a.rows) return;
    v4f_t v = part[0][l];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += part[i][l];
    const int64_t to = (l & 15) * a.ldc + (int64_t)blockIdx.x * 16 + g * 4;
    if (a.c_f32) *reinterpret_cast<float4 *>(static_cast<float *>(a.C) + to) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.C) + to) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// Which kernel, from the extents alone.
// The smallest blocks whose workgroups the chip holds at once, one to a compute unit, since their waves share K out: microseconds in blocks of
//                                  16 x 16   32 x 16   32 x 32   64 x 32   64 x 64   tiles of 128
//     64 x 2736 -> 1040                4.3       3.9       4.5       5.7       8.2       7.0
//    128 x 2736 -> 1040                4.7       5.1       4.6       5.6       8.0       8.3
//    256 x 2736 -> 1040                7.7       6.0       6.1       5.9       8.0       8.3
//     64 x 4096 -> 4096                7.5       6.2       5.6       7.2       9.6       9.0
//    128 x 4096 -> 4096               12.7       8.8       7.4       7.1       9.4      11.0
//    256 x 4096 -> 4096               22.6      15.4      12.2      10.0       9.5      11.0
//    128 x 11008 -> 4096              27.9      19.1      15.8      13.2      18.4      29.4
//    256 x 11008 -> 4096              53.6      35.5      28.4      21.1      18.0      29.3
// Where there are more in any of them: up to 16 and 32 rows blocks of 16 and 32 rows by 16 columns (32 x 4096 -> 11008 10.1 8.7 9.0 9.9 9.8), up to 64 rows
// 32 x 32 (64 x 4096 -> 11008 15.5 12.4 10.5 11.6 10.7 and 11.4 in tiles), then tiles (128 x 4096 -> 11008 27.8 19.0 15.6 14.3 18.0, 13.9 in tiles).
// 64 x 64 where K is long enough that their few steps are not all start and end (512 x 2064 -> 1376 8.6 us and 7.9 in tiles of 128).
// Between the tiles: estimated times.  A round of small tiles, two to a compute unit, takes .51 us a step of 128 along K and 5 beside them; with one to a
// compute unit .33 and 1.5, less where few are left over after whole rounds.  A round of large ones takes .86 us a step with all compute units at work
// and .55 with half of them, where the clock is higher, and 5 to 8.5 beside them.  Measured, small and large: 1024 x 4096 -> 11008 35.1 33.4 us,
// 1536 48.4 59.8, 2048 66.6 63.8, 3000 86.6 92.1, 4096 119 98; 4096 x 4096 -> 4096 45.8 39.2; 2048 x 11008 -> 4096 56.3 61.6, 3000 78.9 74.1;
// 8192 x 2064 -> 1376 20.3 22.8.
enum Mx4Form { FEW_16_16, FEW_32_16, FEW_32_32, FEW_64_32, FEW_64_64, TILE_128, TILE_256 };
struct Mx4Extent { int rows, cols; };
constexpr Mx4Extent kExtents[] = {{16, 16}, {32, 16}, {32, 32}, {64, 32}, {64, 64}, {128, 128}, {256, 256}};
int64_t count_of(const Mx4GemmArgs &a, Mx4Form f) { return (a.M + kExtents[f].rows - 1) / kExtents[f].rows * ((a.N + kExtents[f].cols - 1) / kExtents[f].cols); }
Mx4Form choose_form(const Mx4GemmArgs &a) {
    const double KB = (double)(mx4_width(a.K) / 128);
    for (Mx4Form f : {FEW_16_16, FEW_32_16, FEW_32_32, FEW_64_32, FEW_64_64})
        if (kExtents[f].rows < a.M + 16 && count_of(a, f) <= 256 && (f != FEW_64_64 || KB >= 20)) return f;
    if (a.M <= 64) return a.M <= 16 ? FEW_16_16 : a.M <= 32 ? FEW_32_16 : FEW_32_32;
    const double small_step = .51 * KB + 5, small_alone = .33 * KB + 1.5;
    auto small_time = [&](double tiles) {
        const double rounds = std::floor(tiles / 512), rest = tiles - 512 * rounds;
        const double left = rest > 256 ? small_alone + (rest - 256) / 256 * (small_step - small_alone) : small_alone * (rounds > 0 ? std::max(.3, rest / 256) : 1);
        return rounds * small_step + (rest > 0 ? left : 0);
    };
    auto large_time = [&](double tiles) {
        const double rounds = std::floor(tiles / 256), rest = tiles - 256 * rounds;
        return rounds * (.86 * KB + 5) + (rest > 0 ? KB * (.55 + .31 * std::max(0., rest / 128 - 1)) + 8.5 : 0);
    };
    if (KB <= kStages) return TILE_128;                  // no rings that run on (3000 x 512 -> 11008 28.7 us, 35.0 in large tiles)
    return large_time((double)count_of(a, TILE_256)) < small_time((double)count_of(a, TILE_128)) ? TILE_256 : TILE_128;
}

}  // namespace

I8Plan mx4_gemm_plan(const Mx4GemmArgs &a) {
    const Mx4Form form = choose_form(a);
    return {form >= TILE_128 ? kExtents[form].rows : 0, kExtents[form].rows, kExtents[form].cols};
}

// Sums of nothing: 16 bytes to a thread.
__global__ __launch_bounds__(256) static void mx4_zero_kernel(void *C, int64_t M, int64_t N, int64_t ldc, int size) {
    const int64_t i = block_of_many() * 256 + threadIdx.x, pieces = N * size / 16, row = i / pieces;
    if (row < M) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(C) + row * ldc * size + i % pieces * 16) = make_uint4(0, 0, 0, 0);
}

static Mx4Params params_of(const Mx4GemmArgs &a, Mx4Form form) {
    Mx4Params p;
    p.A = a.A; p.B = a.B; p.sa = a.sa; p.sb = a.sb; p.C = a.C; p.M = a.M; p.N = a.N; p.ldc = a.ldc; p.KB = (int)(mx4_width(a.K) / 128); p.c_f32 = a.c_f32;
    p.tiles_n = (int)((a.N + kExtents[form].cols - 1) / kExtents[form].cols);
    return p;
}

// Two products in tiles of 128 in one launch, a tile to a workgroup and the one with the longer sum first, so that its few long tiles run beside the
// other's.  Backward passes of M rows, N -> K, whole, in two launches and in one: 2383 x 4688 -> 288 34.8 26.0 us; 586 x 3696 -> 2816 34.3 29.0; 256 x 4096 -> 4096
// 28.1 21.9; 777 x 2064 -> 1376 23.9 19.2; 48 x 768 -> 2512 11.2 8.9; over 70 of 1 to 2048 rows and 64 to 12000 columns 11 % less time, at worst 9 % more (1070 x 128 -> 288 9.9 10.8).
// A long sum that blocks of few rows share out takes longer in tiles (.33 us a step; .05 in blocks of 16 x 16, .2 in 64 x 64), which does not pay beside a short launch (105 x 4864 -> 384
// 13.1 17.1, 141 x 7136 -> 112 13.4 20.2).
static bool in_one_launch(const Mx4GemmArgs &longer, const Mx4GemmArgs &other) {
    const Mx4Form form = choose_form(longer);
    if (form > TILE_128 || choose_form(other) > TILE_128) return false;
    const double KB = (double)(mx4_width(longer.K) / 128), other_KB = (double)(mx4_width(other.K) / 128);
    const double few = 3.5 + KB * std::sqrt((double)kExtents[form].rows * kExtents[form].cols) / 320;
    return form == TILE_128 || .33 * KB + 1.5 <= few + std::max(5., (double)count_of(other, TILE_128) / 512 * (.51 * other_KB + 5) + 2);
}
void launch_mx4_gemm_pair(const Mx4GemmArgs &a, const Mx4GemmArgs &b, hipStream_t st) {
    const Mx4GemmArgs &longer = b.K > a.K ? b : a, &other = b.K > a.K ? a : b;
    if (a.M > 0 && b.M > 0 && a.K > 0 && b.K > 0 && in_one_launch(longer, other)) {
        const int first = (int)count_of(longer, TILE_128), all = first + (int)count_of(other, TILE_128);
        profile_before(kTagMx4Gemm, st);
        hipLaunchKernelGGL((mx4_tile_pair_kernel<2, 2>), dim3(all), dim3(256), 0, st, params_of(longer, TILE_128), params_of(other, TILE_128), first);
        profile_after(st);
        return;
    }
    if (a.M > 0 && b.M > 0 && a.K > 0 && b.K > 0 && choose_form(a) == TILE_256 && choose_form(b) == TILE_256) {
        profile_before(kTagMx4Gemm, st);
        const unsigned all = (unsigned)std::min<int64_t>(std::max(count_of(a, TILE_256), count_of(b, TILE_256)), 256);
        hipLaunchKernelGGL((mx4_tile_both_kernel<4, 4>), dim3(all), dim3(256), 0, st, params_of(a, TILE_256), params_of(b, TILE_256));
        profile_after(st);
        return;
    }
    launch_mx4_gemm(a, st);
    launch_mx4_gemm(b, st);
}

void launch_mx4_gemm(const Mx4GemmArgs &a, hipStream_t st) {
    if (a.M == 0) return;
    if (a.K == 0) {
        const int size = a.c_f32 ? 4 : 2;
        hipLaunchKernelGGL(mx4_zero_kernel, grid_of_many((a.M * (a.N * size / 16) + 255) / 256), dim3(256), 0, st, a.C, a.M, a.N, a.ldc, size);
        return;
    }
    const Mx4Form form = choose_form(a);
    const Mx4Params p = params_of(a, form);
    auto go = [&](auto kernel, int threads, int64_t most) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(count_of(a, form), most)), dim3(threads), 0, st, p);
    };
    // the tiles' workgroups stay, one or two to a compute unit; a tile of no more steps than the ring has stages is a workgroup's only one
    // (its loads would run two tiles ahead)
    constexpr int64_t kAll = (int64_t)1 << 31;
    profile_before(kTagMx4Gemm, st);
    switch (form) {
        case FEW_16_16: go(mx4_few_kernel<1, 1, 8>, 512, kAll); break;
        case FEW_32_16: go(mx4_few_kernel<2, 1, 8>, 512, kAll); break;
        case FEW_32_32: go(mx4_few_kernel<2, 2, 8>, 512, kAll); break;
        case FEW_64_32: go(mx4_few_kernel<4, 2, 8>, 512, kAll); break;
        case FEW_64_64: go(mx4_few_kernel<4, 4, 8>, 512, kAll); break;
        case TILE_128: go(mx4_tile_kernel<2, 2>, 256, p.KB > kStages ? 512 : kAll); break;
        case TILE_256: go(mx4_tile_kernel<4, 4>, 256, 256); break;
    }
    profile_after(st);
}

static int64_t token_lds(int64_t M, int64_t K) { return M * (mx4_width(K) / 32 * 17); }
// Every workgroup quantizes all rows, against a launch before the product.  Microseconds of both for rows in bf16, and in fp32 (weights from memory, calls of one graph):
//                             1 row                 2                       4                       8                      16
//   1024 ->  4096                            3.6 5.0   3.8 5.0       3.8 5.1   4.1 5.1       3.9 5.2   4.5 5.0       4.2 5.1   5.6 5.1
//   4096 ->  4096     4.5 6.3   4.9 6.3      4.7 6.3   5.3 6.4       5.1 6.3   6.4 6.4       6.0 6.4   8.4 6.4       7.8 6.4  12.3 6.6
//   1024 -> 11008     5.8 6.1   6.8 5.9      6.0 5.9   6.9 6.1       6.2 6.1   7.3 6.1       6.8 6.1   8.7 6.2       7.9 6.1  11.0 6.3
//   4096 -> 11008     7.8 9.1   8.9 9.1      8.1 9.1  10.0 9.2       9.2 9.1  12.6 9.2      11.6 9.2  18.3 9.3      16.0 9.4  29.5 9.4
//   8192 -> 11008    10.3 13.4 12.2 13.4    11.1 13.4 14.7 13.4     13.7 13.4 20.1 13.6     17.9 13.6 31.1 13.6
//   1024 -> 28672    10.2 9.0  12.3 8.9     10.3 8.9  12.8 9.0      10.9 9.1  14.2 9.0      11.9 9.1  17.7 9.2      14.2 9.1  23.0 9.3
//   8192 -> 28672    21.4 26.0 25.9 25.1    21.6 25.1 30.7 25.0     26.5 25.2 41.4 25.2
//  11008 -> 28672    30.8 34.1 36.0 32.3    31.8 32.0 42.3 32.5     37.7 32.4 58.7 32.4
// So a row costs its share of K in every round of 256 workgroups, 4096 columns, in fp32 2.5 times as much as in bf16; a further round costs its start, which long weights
// hide; and a launch before the product saves less on longer K.  Over 580 pairs of figures, 1 to 16 rows, K 512 to 92160, N 1024 to 60000, the rule's choice takes .3 % more
// than the better one on average, at worst 15 % (one fp32 row 1024 -> 11008).  (One launch for up to four rows of any length, and for more by M K N alone: 8 %, at worst 87.)
bool mx4_token_ok(int64_t M, int64_t N, int64_t K, int bf16) {
    if (M > 16 || token_lds(M, K) > kMx4TokenLds) return false;
    const int64_t cols = std::max<int64_t>(N, 4096);
    return ((bf16 ? 2 : 5) * M - 6) * K * cols + 4 * (cols - 4096) * std::max<int64_t>(8192 - K, 0) <= (int64_t)14 << 24;
}

void launch_mx4_token(const Mx4TokenArgs &a, hipStream_t st) {
    profile_before(kTagMx4Gemm, st);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.N / 16)), dim3(512), (unsigned)token_lds(a.rows, a.K), st, a); };
    if (a.bf16) go(mx4_token_kernel<true, 8>);
    else go(mx4_token_kernel<false, 8>);
    profile_after(st);
}

}  // namespace ssg
