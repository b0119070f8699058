// Matrices in microscaled 4-bit floating point (see ssg_mx4.h), in the layout of the products: from rows, from columns, the way back.
#include "ssg_internal.h"
#include "ssg_mx4.h"

namespace ssg {

namespace {

// A wave has 16 rows by 256 columns: lane l row l % 16 and in each half the l / 16-th run of 32, so that the codes of a half leave as
// one piece of 1 KB and the scales as one of 128 bytes.
template <bool BF16> __global__ __launch_bounds__(256) void mx4_rows_kernel(Mx4RowsArgs a) {
    const int64_t pairs = mx4_width(a.K) / 256, wave = block_of_many() * 4 + threadIdx.x / 64, rb = wave / pairs, p = wave % pairs;
    if (rb * 16 >= a.rows) return;
    const int l = threadIdx.x & 63, g = l >> 4;
    const int64_t row = rb * 16 + (l & 15);
    const uint8_t *src = static_cast<const uint8_t *>(a.src) + row * a.ld * (BF16 ? 2 : 4);
    Mx4Block<BF16> v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) v[h].load(src, p * 256 + h * 128 + g * 32, a.K, row < a.rows);
    uint32_t bytes = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t byte = mx4_scale_byte(v[h].top_bits(), a.ceil);
        bytes |= byte << 8 * h;
        *reinterpret_cast<uint4 *>(a.codes + ((rb * pairs + p) * 2 + h) * 1024 + l * 16) = v[h].codes(byte);
    }
    *reinterpret_cast<uint16_t *>(a.scales + (rb * pairs + p) * 128 + l * 2) = (uint16_t)bytes;
}

// The transpose: a thread has eight columns (four in fp32) of the source and in each half of 256 tokens a run of 32, so that it forms
// their scales and codes by itself and the codes of its columns, neighbouring rows of the layout, lie side by side.
template <bool BF16> __global__ __launch_bounds__(256) void mx4_columns_kernel(Mx4RowsArgs a) {
    constexpr int COLS = BF16 ? 8 : 4;
    const int64_t pairs = mx4_width(a.K) / 256, across = a.rows / COLS, i = block_of_many() * 256 + threadIdx.x;
    if (i >= across * pairs * 4) return;
    const int64_t c0 = i % across * COLS, p = i / across / 4, rb = c0 / 16;
    const int g = (int)(i / across % 4), r0 = (int)(c0 % 16);
    const uint8_t *src = static_cast<const uint8_t *>(a.src) + c0 * (BF16 ? 2 : 4);
    uint32_t bytes[COLS] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t k0 = p * 256 + h * 128 + g * 32;
        uint4 v[32];
#pragma unroll
        for (int t = 0; t < 32; ++t) {
            v[t] = make_uint4(0, 0, 0, 0);
            if (k0 + t < a.K) v[t] = *reinterpret_cast<const uint4 *>(src + (k0 + t) * a.ld * (BF16 ? 2 : 4));
        }
        uint32_t w[32][4];
#pragma unroll
        for (int t = 0; t < 32; ++t) { w[t][0] = v[t].x; w[t][1] = v[t].y; w[t][2] = v[t].z; w[t][3] = v[t].w; }
        uint8_t *out = a.codes + ((rb * pairs + p) * 2 + h) * 1024 + (g * 16 + r0) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            uint32_t top = 0;
#pragma unroll
            for (int t = 0; t < 32; ++t) {
                if (BF16) top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, w[t][j] & 0x7fff7fffu)));
                else top = top > (w[t][j] & 0x7fffffffu) ? top : w[t][j] & 0x7fffffffu;
            }
#pragma unroll
            for (int half = 0; half < (BF16 ? 2 : 1); ++half) {      // the two columns of a word
                const int c = BF16 ? 2 * j + half : j;
                const uint32_t byte = mx4_scale_byte(BF16 ? (half ? top & 0xffff0000u : top << 16) : top, a.ceil);
                const float scale = mx4_scale(byte);
                bytes[c] |= byte << 8 * h;
                uint32_t q[4];
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    if constexpr (BF16) {
                        uint32_t pair[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) pair[t] = __builtin_amdgcn_perm(w[8 * o + 2 * t + 1][j], w[8 * o + 2 * t][j], half ? 0x07060302u : 0x05040100u);
                        q[o] = mx4_codes8(pair, scale);
                    } else {
                        float f[8];
#pragma unroll
                        for (int t = 0; t < 8; ++t) f[t] = __uint_as_float(w[8 * o + t][j]);
                        q[o] = mx4_codes8(f, scale);
                    }
                }
                *reinterpret_cast<uint4 *>(out + c * 16) = byte == 255u ? make_uint4(0, 0, 0, 0) : make_uint4(q[0], q[1], q[2], q[3]);
            }
        }
    }
    uint8_t *out = a.scales + (rb * pairs + p) * 128 + (g * 16 + r0) * 2;
    if constexpr (BF16)
        *reinterpret_cast<uint4 *>(out) = make_uint4(bytes[0] | bytes[1] << 16, bytes[2] | bytes[3] << 16, bytes[4] | bytes[5] << 16, bytes[6] | bytes[7] << 16);
    else *reinterpret_cast<uint2 *>(out) = make_uint2(bytes[0] | bytes[1] << 16, bytes[2] | bytes[3] << 16);
}

// The values that the codes stand for.  (Exact in fp32, and in bf16: 0 to 6 times a power of two from 2^-127 up.)
template <bool BF16> __global__ __launch_bounds__(256) void mx4_values_kernel(Mx4ValuesArgs a) {
    const int64_t pairs = mx4_width(a.K) / 256, wave = block_of_many() * 4 + threadIdx.x / 64, rb = wave / pairs, p = wave % pairs;
    const int l = threadIdx.x & 63, g = l >> 4;
    const int64_t row = rb * 16 + (l & 15);
    if (row >= a.rows) return;
    const uint32_t bytes = *reinterpret_cast<const uint16_t *>(a.scales + (rb * pairs + p) * 128 + l * 2);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t k0 = p * 256 + h * 128 + g * 32;
        const uint4 q = *reinterpret_cast<const uint4 *>(a.codes + ((rb * pairs + p) * 2 + h) * 1024 + l * 16);
        const uint32_t byte = bytes >> 8 * h & 255u, words[4] = {q.x, q.y, q.z, q.w};
        const float scale = byte == 255u ? __uint_as_float(0x7fc00000u) : mx4_scale(byte);
#pragma unroll
        for (int o = 0; o < 4; ++o) {                        // eight values
            const int64_t k = k0 + 8 * o;
            if (k >= a.K) break;
            float v[8];
            auto two = [&](auto at) {
                constexpr int i = decltype(at)::value;
                const ssg_f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(words[o], 1.0f, i);
                v[2 * i] = __fmul_rn(x[0], scale);
                v[2 * i + 1] = __fmul_rn(x[1], scale);
            };
            two(std::integral_constant<int, 0>{});
            two(std::integral_constant<int, 1>{});
            two(std::integral_constant<int, 2>{});
            two(std::integral_constant<int, 3>{});
            if (BF16) {
                uint16_t *out = static_cast<uint16_t *>(a.dst) + row * a.ld + k;
                if (k + 8 <= a.K) {
                    *reinterpret_cast<uint4 *>(out) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (k + i < a.K) out[i] = (uint16_t)f32_to_bf16_bits(v[i]);
                }
            } else {
                float *out = static_cast<float *>(a.dst) + row * a.ld + k;
                if (k + 8 <= a.K) {
                    *reinterpret_cast<float4 *>(out) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4 *>(out + 4) = make_float4(v[4], v[5], v[6], v[7]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (k + i < a.K) out[i] = v[i];
                }
            }
        }
    }
}

// Row-major codes [rows, K / 2] and scales [rows, (K + 31) / 32] into the layout and back; K a multiple of 16.
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
        const dim3 grid = grid_of_many((a.rows / (a.bf16 ? 8 : 4) * (mx4_width(a.K) / 64) + 255) / 256);
        if (a.bf16) hipLaunchKernelGGL(mx4_columns_kernel<true>, grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL(mx4_columns_kernel<false>, grid, dim3(256), 0, st, a);
    } else {
        if (a.bf16) hipLaunchKernelGGL(mx4_rows_kernel<true>, grid_of_pairs(a.rows, a.K), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(mx4_rows_kernel<false>, grid_of_pairs(a.rows, a.K), dim3(256), 0, st, a);
    }
    profile_after(st);
}

void launch_mx4_dequantize(const Mx4ValuesArgs &a, hipStream_t st) {
    if (a.rows == 0) return;
    profile_before(kTagMx4Rows, st, (double)a.rows * a.K * (a.bf16 ? 2 : 4) + (double)(mx4_code_bytes(a.rows, a.K) + mx4_scale_bytes(a.rows, a.K)));
    if (a.bf16) hipLaunchKernelGGL(mx4_values_kernel<true>, grid_of_pairs(a.rows, a.K), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(mx4_values_kernel<false>, grid_of_pairs(a.rows, a.K), dim3(256), 0, st, a);
    profile_after(st);
}

void launch_mx4_pack(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t K, uint8_t *out, uint8_t *out_scales, hipStream_t st) {
    hipLaunchKernelGGL(mx4_pack_kernel, grid_of_pairs(rows, K), dim3(256), 0, st, codes, scales, rows, K, out, out_scales);
}

void launch_mx4_unpack(const uint8_t *in, const uint8_t *in_scales, int64_t rows, int64_t K, uint8_t *codes, uint8_t *scales, hipStream_t st) {
    hipLaunchKernelGGL(mx4_unpack_kernel, grid_of_pairs(rows, K), dim3(256), 0, st, in, in_scales, rows, K, codes, scales);
}

}  // namespace ssg
