// Matrices in microscaled 4-bit floating point (see ssg_mx4.h), in the layout of the products: from rows, from columns, the way back.
#include "ssg_internal.h"
#include "ssg_lds_load.h"
#include "ssg_mx4.h"

namespace ssg {

namespace {

// A wave has 16 rows by 256 columns, or with HALVES = 1 by 128: lane l row l % 16 and in each half the l / 16-th run of 32, so that the codes of a half leave
// as one piece of 1 KB and the scales as one of 128 bytes (of 64 pieces of one where there is one half).  (A lane's four loads of 16 bytes take the same
// cache lines.)  Bound by memory: 4096 x 11008 bf16, 114 MB, 22 to 24 us, fp32, 204 MB, 43, 4.8 TB/s; little ones by latency, so a wave is a block by itself, on
// any compute unit, and has one half where there are few: 333 x 2736 bf16 2.5 us, two halves 2.6, four waves to a block 2.9, in fp32 3.1, 3.0 and 4.0;
// 64 x 4096 fp32 2.4, 2.7 and 4.0; 1024 x 4096 bf16 4.1, 4.3 and 4.1; 4096 x 4096 8.6, 8.2 and 8.3.
template <bool BF16, int HALVES> __global__ __launch_bounds__(64) void mx4_rows_kernel(Mx4RowsArgs a) {
    const int64_t pairs = mx4_width(a.K) / 256, wave = block_of_many() / (2 / HALVES), rb = wave / pairs, p = wave % pairs;
    if (rb * 16 >= a.rows) return;
    const int l = threadIdx.x, g = l >> 4, first = HALVES == 1 ? (int)(block_of_many() & 1) : 0;
    const int64_t row = rb * 16 + (l & 15);
    const uint8_t *src = static_cast<const uint8_t *>(a.src) + row * a.ld * (BF16 ? 2 : 4);
    Mx4Block<BF16> v[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) v[h].load(src, p * 256 + (first + h) * 128 + g * 32, a.K, row < a.rows);
    uint32_t bytes = 0;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        const uint32_t byte = mx4_scale_byte(v[h].top_bits(), a.ceil);
        bytes |= byte << 8 * h;
        *reinterpret_cast<uint4 *>(a.codes + ((rb * pairs + p) * 2 + first + h) * 1024 + l * 16) = v[h].codes(byte);
    }
    uint8_t *scales = a.scales + (rb * pairs + p) * 128 + l * 2 + first;
    if (HALVES == 2) *reinterpret_cast<uint16_t *>(scales) = (uint16_t)bytes;
    else *scales = (uint8_t)bytes;
}

// The transpose, and with it the rows where both are wanted: a block has 64 of the source's rows (tokens) by 512 bytes of each.  Its threads read pieces of
// 16 bytes, form the rows' codes from them, four neighbouring threads a block of 32, and leave them in LDS, out of which a thread takes 32
// tokens of a column, or of two in bf16, and forms theirs.  The tokens and columns that fill the layouts up are zeros.  Bound by memory: the transpose of
// 4096 x 11008 bf16 24 to 25 us, 4.6 TB/s, fp32 42, 4.9 (bf16 30 beside a kernel that writes 90 MB before it; 38.6 with 32 tokens of eight columns in a thread's registers, too few of them to hide their two rounds of loads); the three
// operands of a backward pass at 4096 x 4096 x 11008, 180 MB, 40 us, 4.5 TB/s (50 with the exchanges among four lanes through LDS).
constexpr int kTileTokens = 64;
struct Mx4Both {
    const void *src;                 // [M, N], `ld` elements apart
    uint8_t *row_codes, *row_scales; // of [M, N], or null
    uint8_t *col_codes, *col_scales; // of its transpose [N, M]
    int64_t M, N, ld;
    int ceil;
    int tiles_n;                     // tiles across, of up(N, 256) columns where rows are wanted, else of N
};
template <bool BF16> struct BothTile { static constexpr int kCols = BF16 ? 256 : 128; };
inline int64_t both_tiles_n(int64_t N, bool rows, bool bf16) { const int cols = bf16 ? 256 : 128; return ((rows ? mx4_width(N) : N) + cols - 1) / cols; }
inline int64_t both_tiles(int64_t M, int64_t N, bool rows, bool bf16) { return mx4_width(M) / kTileTokens * both_tiles_n(N, rows, bf16); }

// a four by four transpose of words among four neighbouring lanes: lane i's word j becomes lane j's word i
template <int D> __device__ __forceinline__ void exchange4(uint32_t (&w)[4]) {
    const bool up = threadIdx.x & D;                         // gives word j and takes word j + D; the others the other way round
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j & D) continue;
        const uint32_t in = quad_xor<D>(up ? w[j] : w[j + D]);
        w[j] = up ? in : w[j];
        w[j + D] = up ? w[j + D] : in;
    }
}
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
    exchange4<1>(w);
    exchange4<2>(w);
}

template <bool BF16> __device__ __forceinline__ void both_tile(const Mx4Both &a, int64_t tile, uint32_t (*lds)[128]) {
    constexpr int kCols = BothTile<BF16>::kCols, kLanes = kCols / 8, kGroups = 256 / kLanes, kEach = kTileTokens / kGroups;      // threads to a row, rows at a time, tokens of a thread
    constexpr int kWords = BF16 ? 4 : 8;                     // of a thread's eight values
    const int tid = threadIdx.x, across = tid % kLanes, group = tid / kLanes;
    const int64_t t0 = tile / a.tiles_n * kTileTokens, c0 = tile % a.tiles_n * kCols, col = c0 + across * 8;
    uint32_t w[kEach][kWords];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int64_t t = t0 + group * kEach + e;
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(a.src) + (t * a.ld + col) * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            uint4 q = make_uint4(0, 0, 0, 0);
            if (t < a.M && col < a.N) q = p[i];
            w[e][4 * i] = q.x; w[e][4 * i + 1] = q.y; w[e][4 * i + 2] = q.z; w[e][4 * i + 3] = q.w;
        }
    }
    // (a word of two bf16, columns 2 i and 2 i + 1, or of one fp32)
#pragma unroll
    for (int e = 0; e < kEach; ++e)
#pragma unroll
        for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4 *>(&lds[group * kEach + e][across * kWords + i]) = make_uint4(w[e][i], w[e][i + 1], w[e][i + 2], w[e][i + 3]);
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    auto larger = [](uint32_t x, uint32_t y) {
        if (BF16) return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
        return x > y ? x : y;
    };
    constexpr uint32_t kAbs = BF16 ? 0x7fff7fffu : 0x7fffffffu;
    if (a.row_codes && t0 < i8_up(a.M, 16)) {
        const int64_t pairs = mx4_width(a.N) / 256;
        uint32_t code[kEach], byte[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kWords; ++i) top = larger(top, w[e][i] & kAbs);
            if (BF16) top = (top & 0xffff0000u) > top << 16 ? top & 0xffff0000u : top << 16;
            byte[e] = mx4_scale_byte(quad_max(top), a.ceil);
            if constexpr (BF16) code[e] = mx4_codes8(w[e], mx4_scale(byte[e]));
            else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[e][i]);
                code[e] = mx4_codes8(f, mx4_scale(byte[e]));
            }
            if (byte[e] == 255u) code[e] = 0;
        }
        const int q = tid & 3;
        const int64_t block_col = col - 8 * q;               // of the block of 32
        auto place = [&](int64_t t) { return t / 16 * pairs + block_col / 256; };
        auto lane_of = [&](int64_t t) { return (int)(block_col % 128 / 32 * 16 + t % 16); };
#pragma unroll
        for (int e = 0; e < kEach; e += 4) {
            uint32_t x[4] = {code[e], code[e + 1], code[e + 2], code[e + 3]};
            transpose4(x);
            const int64_t t = t0 + group * kEach + e + q;
            if (t >= i8_up(a.M, 16) || block_col >= pairs * 256) continue;
            *reinterpret_cast<uint4 *>(a.row_codes + (place(t) * 2 + block_col % 256 / 128) * 1024 + lane_of(t) * 16) = make_uint4(x[0], x[1], x[2], x[3]);
            const uint32_t b = q == 0 ? byte[e] : q == 1 ? byte[e + 1] : q == 2 ? byte[e + 2] : byte[e + 3];
            a.row_scales[place(t) * 128 + lane_of(t) * 2 + block_col % 256 / 128] = (uint8_t)b;
        }
    }
    __syncthreads();
    constexpr int kUnits = BF16 ? 2 : 1, kAcross = 128;      // columns of a thread; words across the tile
    const int word = tid % kAcross, half = tid / kAcross;    // half: which 32 of the tokens
    const int64_t n0 = c0 + word * kUnits, k0 = t0 + half * 32;
    if (n0 >= a.N) return;
    uint32_t v[32], top = 0;
#pragma unroll
    for (int t = 0; t < 32; ++t) {
        v[t] = lds[half * 32 + t][word];
        top = larger(top, v[t] & kAbs);
    }
    const int64_t pairs = mx4_width(a.M) / 256, block = n0 / 16 * pairs + k0 / 256;
    const int parity = (int)(k0 % 256 / 128), lane = (int)(k0 % 128 / 32 * 16 + n0 % 16);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const uint32_t byte = mx4_scale_byte(BF16 ? (u ? top & 0xffff0000u : top << 16) : top, a.ceil);
        const float scale = mx4_scale(byte);
        uint32_t q[4];
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            if constexpr (BF16) {
                uint32_t pair[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) pair[t] = __builtin_amdgcn_perm(v[8 * o + 2 * t + 1], v[8 * o + 2 * t], u ? 0x07060302u : 0x05040100u);
                q[o] = mx4_codes8(pair, scale);
            } else {
                float f[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) f[t] = __uint_as_float(v[8 * o + t]);
                q[o] = mx4_codes8(f, scale);
            }
        }
        *reinterpret_cast<uint4 *>(a.col_codes + (block * 2 + parity) * 1024 + (lane + u) * 16) = byte == 255u ? make_uint4(0, 0, 0, 0) : make_uint4(q[0], q[1], q[2], q[3]);
        a.col_scales[block * 128 + (lane + u) * 2 + parity] = (uint8_t)byte;
    }
}

// one matrix after the other: tiles of the first below `first`
template <bool BF16, bool BF16_2> __global__ __launch_bounds__(256) void mx4_columns_kernel(Mx4Both a, Mx4Both b, int64_t first, int64_t all) {
    __shared__ __attribute__((aligned(16))) uint32_t lds[kTileTokens][128];
    const int64_t tile = block_of_many();
    if (tile < first) both_tile<BF16>(a, tile, lds);
    else if (tile < all) both_tile<BF16_2>(b, tile - first, lds);
}

Mx4Both both_args(const Mx4RowsArgs &t, const Mx4RowsArgs *rows) {
    Mx4Both b;
    b.src = t.src; b.col_codes = t.codes; b.col_scales = t.scales; b.M = t.K; b.N = t.rows; b.ld = t.ld; b.ceil = t.ceil;
    b.row_codes = rows ? rows->codes : nullptr; b.row_scales = rows ? rows->scales : nullptr;
    b.tiles_n = (int)both_tiles_n(b.N, rows != nullptr, t.bf16);
    return b;
}

// The values that the codes stand for.  (Exact in fp32, and in bf16: 0 to 6 times a power of two from 2^-127 up.)  A wave has 16 rows by 256 columns, or one of
// PARTS shares of the rows, and stores 16 bytes to a lane side by side along a row, 256 (512) bytes of four (two) rows at a time; the codes, 4 (2) bytes to a lane, come out of
// the cache lines of a 1 KB block.  Bound by memory: 4096 x 11008 to bf16 25 us, 4.5 TB/s (41 with 64 bytes of a row to a lane), to fp32 55, 3.7;
// little ones by latency: 75 x 2736 in one, two and four parts 2.8 2.4 2.3, to fp32 3.8 2.9 2.5 (four waves to a block 3.0 and 4.2); 333 x 11008 4.3 4.0 4.0
// and 6.7 6.2 6.1; 4096 x 4096 8.7 7.9 9.1 and 16.5 20.8 19.7.
template <bool BF16, int PARTS> __global__ __launch_bounds__(64) void mx4_values_kernel(Mx4ValuesArgs a) {
    constexpr int kEach = BF16 ? 8 : 4, kLanes = 128 / kEach, kRowsAtOnce = 64 / kLanes, kRows = 16 / PARTS, kSteps = kRows / kRowsAtOnce;      // values of a lane, lanes to 128 columns
    const int64_t pairs = mx4_width(a.K) / 256, wave = block_of_many() / PARTS, rb = wave / pairs, p = wave % pairs;
    const int first = (int)(block_of_many() % PARTS) * kRows;
    if (rb * 16 + first >= a.rows) return;
    const int l = threadIdx.x, c = l % kLanes * kEach, g = c / 32;      // column of the 128, its run of 32
    const uint8_t *codes = a.codes + (rb * pairs + p) * 2048 + g * 256 + c % 32 / 2, *scales = a.scales + (rb * pairs + p) * 128 + g * 32;
    uint32_t word[2][kSteps], bytes[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int r = first + i * kRowsAtOnce + l / kLanes;
        bytes[i] = *reinterpret_cast<const uint16_t *>(scales + r * 2);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            word[h][i] = BF16 ? *reinterpret_cast<const uint32_t *>(codes + h * 1024 + r * 16) : *reinterpret_cast<const uint16_t *>(codes + h * 1024 + r * 16);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int64_t row = rb * 16 + first + i * kRowsAtOnce + l / kLanes, k = p * 256 + h * 128 + c;
            const uint32_t byte = bytes[i] >> 8 * h & 255u;
            const float scale = byte == 255u ? __uint_as_float(0x7fc00000u) : mx4_scale(byte);
            float v[kEach];
            each<kEach / 2>([&](auto at) {
                constexpr int j = decltype(at)::value;
                const ssg_f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[h][i], 1.0f, j);
                v[2 * j] = __fmul_rn(x[0], scale);
                v[2 * j + 1] = __fmul_rn(x[1], scale);
            });
            if (row >= a.rows || k >= a.K) continue;
            if constexpr (BF16) {
                uint16_t *out = static_cast<uint16_t *>(a.dst) + row * a.ld + k;
                if (k + kEach <= a.K) {
                    *reinterpret_cast<uint4 *>(out) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                } else {
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (k + j < a.K) out[j] = (uint16_t)f32_to_bf16_bits(v[j]);
                }
            } else {
                float *out = static_cast<float *>(a.dst) + row * a.ld + k;
                if (k + kEach <= a.K) {
                    *reinterpret_cast<float4 *>(out) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (k + j < a.K) out[j] = v[j];
                }
            }
        }
}

// Row-major codes [rows, K / 2] and scales [rows, (K + 31) / 32] into the layout and back; K a multiple of 16.  Bound by memory at sizes that matter, done once for
// a program's weights: 4096 x 11008, 48 MB, 11.4 us and 12.7 back, 4.2 and 3.8 TB/s.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t K, uint8_t *out, uint8_t *out_scales) {
    const int64_t pairs = mx4_width(K) / 256, wave = block_of_many() * 4 + threadIdx.x / 64, rb = wave / pairs, p = wave % pairs;
    if (rb * 16 >= rows) return;
    const int l = threadIdx.x & 63, g = l >> 4;
    const int64_t row = rb * 16 + (l & 15);
    uint32_t bytes = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t k = p * 256 + h * 128 + g * 32;
        uint2 q[2] = {make_uint2(0, 0), make_uint2(0, 0)};
        if (row < rows && k < K) {
            q[0] = *reinterpret_cast<const uint2 *>(codes + row * (K / 2) + k / 2);
            if (k + 16 < K) q[1] = *reinterpret_cast<const uint2 *>(codes + row * (K / 2) + k / 2 + 8);
            bytes |= (uint32_t)scales[row * ((K + 31) / 32) + k / 32] << 8 * h;
        }
        *reinterpret_cast<uint4 *>(out + ((rb * pairs + p) * 2 + h) * 1024 + l * 16) = make_uint4(q[0].x, q[0].y, q[1].x, q[1].y);
    }
    *reinterpret_cast<uint16_t *>(out_scales + (rb * pairs + p) * 128 + l * 2) = (uint16_t)bytes;
}
__global__ __launch_bounds__(256) void mx4_unpack_kernel(const uint8_t *in, const uint8_t *in_scales, int64_t rows, int64_t K, uint8_t *codes, uint8_t *scales) {
    const int64_t pairs = mx4_width(K) / 256, wave = block_of_many() * 4 + threadIdx.x / 64, rb = wave / pairs, p = wave % pairs;
    const int l = threadIdx.x & 63, g = l >> 4;
    const int64_t row = rb * 16 + (l & 15);
    if (row >= rows) return;
    const uint32_t bytes = *reinterpret_cast<const uint16_t *>(in_scales + (rb * pairs + p) * 128 + l * 2);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t k = p * 256 + h * 128 + g * 32;
        if (k >= K) continue;
        const uint4 q = *reinterpret_cast<const uint4 *>(in + ((rb * pairs + p) * 2 + h) * 1024 + l * 16);
        *reinterpret_cast<uint2 *>(codes + row * (K / 2) + k / 2) = make_uint2(q.x, q.y);
        if (k + 16 < K) *reinterpret_cast<uint2 *>(codes + row * (K / 2) + k / 2 + 8) = make_uint2(q.z, q.w);
        scales[row * ((K + 31) / 32) + k / 32] = (uint8_t)(bytes >> 8 * h);
    }
}

// Four waves to a block, one to 16 rows by 256 columns.
dim3 grid_of_pairs(int64_t rows, int64_t K) { return grid_of_many(((rows + 15) / 16 * (mx4_width(K) / 256) + 3) / 4); }

}  // namespace

void launch_mx4_quantize(const Mx4RowsArgs &a, hipStream_t st) {
    if (a.rows == 0) return;
    profile_before(kTagMx4Rows, st, (double)a.rows * a.K * (a.bf16 ? 2 : 4) + (double)(mx4_code_bytes(a.rows, a.K) + mx4_scale_bytes(a.rows, a.K)));
    if (a.transposed) {
        const Mx4Both b = both_args(a, nullptr);
        const int64_t tiles = both_tiles(b.M, b.N, false, a.bf16);
        if (a.bf16) hipLaunchKernelGGL((mx4_columns_kernel<true, true>), grid_of_many(tiles), dim3(256), 0, st, b, b, tiles, tiles);
        else hipLaunchKernelGGL((mx4_columns_kernel<false, false>), grid_of_many(tiles), dim3(256), 0, st, b, b, tiles, tiles);
    } else {
        const int64_t pairs = (a.rows + 15) / 16 * (mx4_width(a.K) / 256);
        auto go = [&](auto kernel, int64_t blocks) { hipLaunchKernelGGL(kernel, grid_of_many(blocks), dim3(64), 0, st, a); };
        if (a.bf16 && pairs <= 1024) go(mx4_rows_kernel<true, 1>, 2 * pairs);
        else if (a.bf16) go(mx4_rows_kernel<true, 2>, pairs);
        else if (pairs <= 1024) go(mx4_rows_kernel<false, 1>, 2 * pairs);
        else go(mx4_rows_kernel<false, 2>, pairs);
    }
    profile_after(st);
}

void launch_mx4_quantize_bwd(const Mx4RowsArgs *rows, const Mx4RowsArgs &dy, const Mx4RowsArgs &x, hipStream_t st) {
    const Mx4Both a = both_args(dy, rows), b = both_args(x, nullptr);
    const int64_t first = both_tiles(a.M, a.N, rows != nullptr, dy.bf16), all = first + both_tiles(b.M, b.N, false, x.bf16);
    profile_before(kTagMx4Rows, st, (double)dy.K * ((double)dy.rows * ((dy.bf16 ? 2 : 4) + (rows ? 2 : 1) * 17 / 32.) + (double)x.rows * ((x.bf16 ? 2 : 4) + 17 / 32.)));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid_of_many(all), dim3(256), 0, st, a, b, first, all); };
    if (dy.bf16 && x.bf16) go(mx4_columns_kernel<true, true>);
    else if (dy.bf16) go(mx4_columns_kernel<true, false>);
    else if (x.bf16) go(mx4_columns_kernel<false, true>);
    else go(mx4_columns_kernel<false, false>);
    profile_after(st);
}

void launch_mx4_dequantize(const Mx4ValuesArgs &a, hipStream_t st) {
    if (a.rows == 0) return;
    profile_before(kTagMx4Rows, st, (double)a.rows * a.K * (a.bf16 ? 2 : 4) + (double)(mx4_code_bytes(a.rows, a.K) + mx4_scale_bytes(a.rows, a.K)));
    const int64_t pairs = (a.rows + 15) / 16 * (mx4_width(a.K) / 256);
    auto go = [&](auto kernel, int64_t blocks) { hipLaunchKernelGGL(kernel, grid_of_many(blocks), dim3(64), 0, st, a); };
    if (a.bf16 && pairs < 1024) go(mx4_values_kernel<true, 4>, 4 * pairs);
    else if (a.bf16) go(mx4_values_kernel<true, 2>, 2 * pairs);
    else if (pairs < 1024) go(mx4_values_kernel<false, 4>, 4 * pairs);
    else go(mx4_values_kernel<false, 1>, pairs);
    profile_after(st);
}

void launch_mx4_pack(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t K, uint8_t *out, uint8_t *out_scales, hipStream_t st) {
    hipLaunchKernelGGL(mx4_pack_kernel, grid_of_pairs(rows, K), dim3(256), 0, st, codes, scales, rows, K, out, out_scales);
}

void launch_mx4_unpack(const uint8_t *in, const uint8_t *in_scales, int64_t rows, int64_t K, uint8_t *codes, uint8_t *scales, hipStream_t st) {
    hipLaunchKernelGGL(mx4_unpack_kernel, grid_of_pairs(rows, K), dim3(256), 0, st, in, in_scales, rows, K, codes, scales);
}

}  // namespace ssg
