// Rows in 8-bit integers with a scale each (tokens of activations, channels of weights), in the layout of the products:
//
//   amax = max_k |x_rk|,  scale_r = fl32(amax / 127),  code = round-to-nearest-even(fl32(x f)),  f = fl32(127 fl32(1 / amax))
//
// (the factor in the two steps that tensor programs form it in, so that their codes are these; codes -127 to 127; scale at
// least 2^-126, 1 / scale the factor there; amax = 0: scale 0, codes 0; a row that holds a NaN or an infinity has a NaN for its
// scale and codes 0, so that everything made from it is NaN).
#include "ssg_device.h"
#include "ssg_i8.h"
#include "ssg_internal.h"

namespace ssg {

namespace {

// The list of row tiles, by one wave.
__device__ __forceinline__ void list_tiles(const int *offsets, int E, int *list, int edge) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int e = e0 + lane;
        int lo = 0, hi = 0;
        if (e < E) { lo = offsets[e]; hi = offsets[e + 1]; }
        const int n = (hi - lo + edge - 1) / edge;
        int inc = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(inc, d, 64);
            if (lane >= d) inc += o;
        }
        const int first = before + inc - n;
        for (int i = 0; i < n; ++i) *reinterpret_cast<int4 *>(list + 4 + 4 * (first + i)) = make_int4(lo, hi, e, first);
        before += __shfl(inc, 63, 64);
    }
    if (lane == 0) *reinterpret_cast<int4 *>(list) = make_int4(before, 0, 0, 0);
}

// Bound by memory: 4096 rows of 11008 bf16 (135 MB) 30 us, 4.5 TB/s; 4096 tokens of 2048 gathered into 32768 rows (17 MB read eight
// times, out of the caches, 67 MB written) 28 us.  A block owns ROWS rows, up to half of a row of
// the layout's blocks: thread t has row t % ROWS and every (threads / ROWS)-th run of 16 codes, so that with eight a wave reads 8 rows x 128
// elements and writes pieces of 128 bytes; at most 128 registers, since one more halves the blocks on a compute unit (a fifth more time for 2304
// rows of 11008).  The first HELD runs of a thread stay in registers between the
// maximum and the codes; what a row has beyond them is read again, out of the L2.
template <bool BF16, int THREADS, int HELD, int ROWS> __global__ __launch_bounds__(THREADS, 4) void i8_rows_kernel(I8RowsArgs a) {
    constexpr int kCols = THREADS / ROWS, kWaves = THREADS / 64;
    __shared__ uint32_t maxima[kWaves][ROWS];
    const int tid = threadIdx.x, r = tid % ROWS, c0 = tid / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    if (a.E > 0 && blockIdx.x == gridDim.x - 1) {       // (the block behind those of the rows)
        if (tid < 128 && a.tiles[tid >> 6].edge) list_tiles(a.offsets, a.E, a.tiles[tid >> 6].list, a.tiles[tid >> 6].edge);
        return;
    }
    if (a.live_rows && (int64_t)blockIdx.x * ROWS >= *a.live_rows) return;
    int64_t from = row < a.rows ? row : -1;
    if (a.source && from >= 0) {
        const int s = a.source[row];
        from = s >= 0 ? s / a.k : -1;
    }
    const int runs = (int)(a.K / 16), padded = (int)(i8_width(a.K) / 16);
    const uint8_t *src = static_cast<const uint8_t *>(a.src) + (from >= 0 ? from : 0) * a.ld * (BF16 ? 2 : 4);
    I8Run<BF16> held[HELD];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        held[i].clear();
        const int c = c0 + i * kCols;
        if (from >= 0 && c < runs) held[i].load(src, c);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) top = held[i].max_bits(top);
    if (from >= 0)
        for (int c = c0 + HELD * kCols; c < runs; c += kCols) {
            I8Run<BF16> run;
            run.load(src, c);
            top = run.max_bits(top);
        }
    top = I8Run<BF16>::as_f32_bits(top);
    auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
#pragma unroll
    for (int d = ROWS; d < 64; d *= 2) top = larger(top, (uint32_t)__shfl_xor((int)top, d, 64));
    if ((tid & 63) < ROWS) maxima[tid >> 6][r] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = larger(top, maxima[i][r]);
    const I8Scale s = i8_scale(top);
    if (tid < ROWS) a.scales[row] = s.scale;
    uint8_t *out = a.codes + (row / 16 * padded * 16 + row % 16) * 16;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int c = c0 + i * kCols;
        held[i].opaque();
        if (c < padded) *reinterpret_cast<uint4 *>(out + (int64_t)c * 256) = held[i].codes(s.factor);
    }
    for (int c = c0 + HELD * kCols; c < padded; c += kCols) {
        I8Run<BF16> run;
        run.clear();
        if (from >= 0 && c < runs) run.load(src, c);
        *reinterpret_cast<uint4 *>(out + (int64_t)c * 256) = run.codes(s.factor);
    }
}

template <bool BF16, int ROWS> void launch_rows_as(const I8RowsArgs &a, hipStream_t st) {
    const unsigned blocks = (unsigned)(i8_up(a.rows, 16) / ROWS) + (a.E > 0);
    const int runs = (int)(i8_width(a.K) / 16);
    // the smallest block whose registers hold the rows: 88 registers of values are 11 runs of bf16, 80 5 of fp32
    auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, st, a); };
    constexpr int kFew = BF16 ? 4 : 2, kMost = BF16 ? 11 : 5, kCols = 256 / ROWS;
    if (runs <= kCols * kFew) go(i8_rows_kernel<BF16, 256, kFew, ROWS>, 256);
    else if (runs <= kCols * kMost) go(i8_rows_kernel<BF16, 256, kMost, ROWS>, 256);
    else if (runs <= 2 * kCols * kMost) go(i8_rows_kernel<BF16, 512, kMost, ROWS>, 512);
    else go(i8_rows_kernel<BF16, 1024, kMost, ROWS>, 1024);
}
// Few rows in smaller blocks, so that they are more compute units' work; many in blocks of eight, whose pieces fill cache lines.  Microseconds in
// blocks of two, four and eight rows, bf16, cold, of 1376, 4096 and 11008:
//    384 rows   3.7  4.0  4.5     4.5  5.2  7.5     7.4  9.2 10.1       2816 rows   6.1  5.3  5.2    13.2 11.6 12.9    31.2 22.6 22.8
//    768        4.0  4.0  4.3     5.2  5.4  7.8    11.3 13.4 14.0       3584        6.6  6.2  5.6    15.2 11.7 13.3    37.5 29.3 25.6
//   1536        4.8  4.6  4.8     6.8  6.1  8.2    15.9 15.7 16.5       8192       13.4 11.4 12.0    29.2 22.1 21.4
//   2304        5.6  5.1  5.1    11.5 10.0 12.0    27.9 20.9 22.5
// Between 2304 and 2816 rows four are faster than eight, or within 4 %, at every width from 688 to 11008 in both types; beyond, that depends on the
// width.
template <bool BF16> void launch_rows(const I8RowsArgs &a, hipStream_t st) {
    if (a.rows <= 512) launch_rows_as<BF16, 2>(a, st);
    else if (a.rows <= 2560) launch_rows_as<BF16, 4>(a, st);
    else launch_rows_as<BF16, 8>(a, st);
}

// Row-major codes and scales into the layout and back, 16 bytes to a thread.
__global__ void i8_pack_kernel(const int8_t *codes, const float *scales, int64_t rows, int64_t K, uint8_t *out, float *out_scales) {
    const int64_t i = block_of_many() * 256 + threadIdx.x;
    const int64_t padded = i8_width(K) / 16, up = i8_up(rows, 16);
    if (i < up) out_scales[i] = i < rows ? scales[i] : 0.0f;
    if (i >= up * padded) return;
    const int64_t r = i / (16 * padded) * 16 + (i & 15), c = i % (16 * padded) / 16;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < rows && c * 16 < K) v = *reinterpret_cast<const uint4 *>(codes + r * K + c * 16);
    *reinterpret_cast<uint4 *>(out + i * 16) = v;
}
__global__ void i8_unpack_kernel(const uint8_t *in, const float *in_scales, int64_t rows, int64_t K, int8_t *codes, float *scales) {
    const int64_t i = block_of_many() * 256 + threadIdx.x;
    const int64_t padded = i8_width(K) / 16, up = i8_up(rows, 16);
    if (i < rows) scales[i] = in_scales[i];
    if (i >= up * padded) return;
    const int64_t r = i / (16 * padded) * 16 + (i & 15), c = i % (16 * padded) / 16;
    if (r < rows && c * 16 < K) *reinterpret_cast<uint4 *>(codes + r * K + c * 16) = *reinterpret_cast<const uint4 *>(in + i * 16);
}

}  // namespace

void launch_i8_quantize(const I8RowsArgs &a, hipStream_t st) {
    if (a.rows == 0) return;
    profile_before(kTagI8Rows, st, (double)a.rows * a.K * (a.bf16 ? 3 : 5));
    if (a.bf16) launch_rows<true>(a, st);
    else launch_rows<false>(a, st);
    profile_after(st);
}

void launch_i8_pack(const int8_t *codes, const float *scales, int64_t rows, int64_t K, uint8_t *out, float *out_scales, hipStream_t st) {
    const int64_t n = i8_code_bytes(rows, K) / 16;
    hipLaunchKernelGGL(i8_pack_kernel, grid_of_many((n + 255) / 256), dim3(256), 0, st, codes, scales, rows, K, out, out_scales);
}

void launch_i8_unpack(const uint8_t *in, const float *in_scales, int64_t rows, int64_t K, int8_t *codes, float *scales, hipStream_t st) {
    const int64_t n = i8_code_bytes(rows, K) / 16;
    hipLaunchKernelGGL(i8_unpack_kernel, grid_of_many((n + 255) / 256), dim3(256), 0, st, in, in_scales, rows, K, codes, scales);
}

}  // namespace ssg
