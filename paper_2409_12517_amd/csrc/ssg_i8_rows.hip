// Rows in 8-bit integers with a scale each (tokens of activations, channels of weights), in the layout of the products:
//
//   amax = max_k |x_rk|,  scale_r = fl32(amax / 127),  code = round-to-nearest-even(fl32(x f)),  f = fl32(127 fl32(1 / amax))
//
// (the factor in the two steps that tensor programs form it in, so that their codes are these; codes -127 to 127; scale at least 2^-126, 1 / scale the factor there; amax = 0: scale 0, codes 0; a row that holds a NaN or an infinity has
// a NaN for its scale and codes 0, so that everything made from it is NaN).
#include "ssg_device.h"
#include "ssg_i8.h"
#include "ssg_internal.h"

namespace ssg {

namespace {

// A block owns 16 rows, as the layout does: thread t has row t % 16 and every (threads / 16)-th run of 16 codes, so that a wave
// reads 16 rows x 64 elements and writes 1 KB of codes in one piece.  The first kHeld runs stay in registers between the maximum and the
// codes; what a row has beyond them is read again, out of the L2.
constexpr int kHeld = 4;
template <bool BF16, int THREADS> __global__ __launch_bounds__(THREADS) void i8_rows_kernel(I8RowsArgs a) {
    constexpr int kCols = THREADS / 16;
    __shared__ uint32_t maxima[THREADS / 64][16];
    const int tid = threadIdx.x, r = tid & 15, c0 = tid >> 4;
    const int64_t row = (int64_t)blockIdx.x * 16 + r;
    if (a.live_rows && (int64_t)blockIdx.x * 16 >= *a.live_rows) return;
    int64_t from = row < a.rows ? row : -1;
    if (a.source && from >= 0) {
        from = a.source[row];
        if (from >= 0) from /= a.k;
    }
    const int runs = (int)(a.K / 16), padded = (int)(i8_up(a.K, 64) / 16);
    const uint8_t *src = static_cast<const uint8_t *>(a.src) + (from >= 0 ? from : 0) * a.ld * (BF16 ? 2 : 4);
    I8Run<BF16> held[kHeld];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        held[i].clear();
        const int c = c0 + i * kCols;
        if (from >= 0 && c < runs) held[i].load(src, c);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) top = held[i].max_bits(top);
    if (from >= 0)
        for (int c = c0 + kHeld * kCols; c < runs; c += kCols) {
            I8Run<BF16> run;
            run.load(src, c);
            top = run.max_bits(top);
        }
    auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    top = larger(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    top = larger(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    if ((tid & 63) < 16) maxima[tid >> 6][r] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) top = larger(top, maxima[i][r]);
    const I8Scale s = i8_scale(top);
    if (tid < 16) a.scales[row] = s.scale;
    uint8_t *out = a.codes + (int64_t)blockIdx.x * padded * 256 + r * 16;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int c = c0 + i * kCols;
        if (c < padded) *reinterpret_cast<uint4 *>(out + (int64_t)c * 256) = held[i].codes(s.factor);
    }
    for (int c = c0 + kHeld * kCols; c < padded; c += kCols) {
        I8Run<BF16> run;
        run.clear();
        if (from >= 0 && c < runs) run.load(src, c);
        *reinterpret_cast<uint4 *>(out + (int64_t)c * 256) = run.codes(s.factor);
    }
}

// Row-major codes and scales into the layout and back, 16 bytes to a thread.
__global__ void i8_pack_kernel(const int8_t *codes, const float *scales, int64_t rows, int64_t K, uint8_t *out, float *out_scales) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t padded = i8_up(K, 64) / 16, up = i8_up(rows, 16);
    if (i < up) out_scales[i] = i < rows ? scales[i] : 0.0f;
    if (i >= up * padded) return;
    const int64_t r = i / (16 * padded) * 16 + (i & 15), c = i % (16 * padded) / 16;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < rows && c * 16 < K) v = *reinterpret_cast<const uint4 *>(codes + r * K + c * 16);
    *reinterpret_cast<uint4 *>(out + i * 16) = v;
}
__global__ void i8_unpack_kernel(const uint8_t *in, const float *in_scales, int64_t rows, int64_t K, int8_t *codes, float *scales) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t padded = i8_up(K, 64) / 16, up = i8_up(rows, 16);
    if (i < rows) scales[i] = in_scales[i];
    if (i >= up * padded) return;
    const int64_t r = i / (16 * padded) * 16 + (i & 15), c = i % (16 * padded) / 16;
    if (r < rows && c * 16 < K) *reinterpret_cast<uint4 *>(codes + r * K + c * 16) = *reinterpret_cast<const uint4 *>(in + i * 16);
}

}  // namespace

void launch_i8_quantize(const I8RowsArgs &a, hipStream_t st) {
    if (a.rows == 0) return;
    const unsigned blocks = (unsigned)((a.rows + 15) / 16);
    profile_before(kTagI8Rows, st, (double)a.rows * a.K * (a.bf16 ? 3 : 5));
    if (a.bf16) hipLaunchKernelGGL((i8_rows_kernel<true, 1024>), dim3(blocks), dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((i8_rows_kernel<false, 1024>), dim3(blocks), dim3(1024), 0, st, a);
    profile_after(st);
}

void launch_i8_pack(const int8_t *codes, const float *scales, int64_t rows, int64_t K, uint8_t *out, float *out_scales, hipStream_t st) {
    const int64_t n = i8_code_bytes(rows, K) / 16;
    hipLaunchKernelGGL(i8_pack_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, codes, scales, rows, K, out, out_scales);
}

void launch_i8_unpack(const uint8_t *in, const float *in_scales, int64_t rows, int64_t K, int8_t *codes, float *scales, hipStream_t st) {
    const int64_t n = i8_code_bytes(rows, K) / 16;
    hipLaunchKernelGGL(i8_unpack_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, in, in_scales, rows, K, codes, scales);
}

}  // namespace ssg
