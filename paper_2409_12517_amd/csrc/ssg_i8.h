// Device helpers of the products in 8-bit integers: a run of 16 values of a row, its scale and its codes.
#pragma once
#include "ssg_device.h"
#include "ssg_internal.h"

namespace ssg {

struct I8Scale { float scale, factor; };
// From the largest absolute value's bits (those of a NaN or an infinity stand above every number's).
__device__ __forceinline__ I8Scale i8_scale(uint32_t top_bits) {
    if (top_bits >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.0f};
    const float amax = __uint_as_float(top_bits);
    const float scale = __fdiv_rn(amax, 127.0f);
    if (scale >= 0x1p-126f) return {scale, __fmul_rn(127.0f, __fdiv_rn(1.0f, amax))};
    return amax > 0.0f ? I8Scale{0x1p-126f, 0x1p126f} : I8Scale{0.0f, 0.0f};
}

// Four values to four codes.  |v * factor| is at most 127 and a little, where adding 1.5 * 2^23 rounds to a whole number, to even
// between two, and leaves its two's complement in the low bits.
__device__ __forceinline__ uint32_t i8_codes4(float a, float b, float c, float d, float factor) {
    constexpr float kMagic = 12582912.0f;
    const uint32_t x = __float_as_uint(__fadd_rn(__fmul_rn(a, factor), kMagic)), y = __float_as_uint(__fadd_rn(__fmul_rn(b, factor), kMagic));
    const uint32_t z = __float_as_uint(__fadd_rn(__fmul_rn(c, factor), kMagic)), w = __float_as_uint(__fadd_rn(__fmul_rn(d, factor), kMagic));
    const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x0c0c0400u), hi = __builtin_amdgcn_perm(w, z, 0x0c0c0400u);
    return lo | hi << 16;
}

template <bool BF16> struct I8Run {
    uint4 v[BF16 ? 2 : 4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (auto &q : v) q = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load(const uint8_t *row, int run) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + (int64_t)run * (BF16 ? 32 : 64));
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) v[i] = p[i];
    }
    __device__ __forceinline__ float value(int i) const {
        const uint32_t words[4] = {v[i / (BF16 ? 8 : 4)].x, v[i / (BF16 ? 8 : 4)].y, v[i / (BF16 ? 8 : 4)].z, v[i / (BF16 ? 8 : 4)].w};
        if (!BF16) return __uint_as_float(words[i % 4]);
        const uint32_t w = words[i % 8 / 2];
        return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
    // Largest absolute value so far: bits of fp32, or of two bf16 side by side, which are compared as 16-bit integers.
    __device__ __forceinline__ uint32_t max_bits(uint32_t top) const {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (const auto &q : v) {
            const uint32_t words[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (uint32_t w : words) {
                if (BF16) top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
                else top = top > (w & 0x7fffffffu) ? top : w & 0x7fffffffu;
            }
        }
        return top;
    }
    static __device__ __forceinline__ uint32_t as_f32_bits(uint32_t top) {
        if (!BF16) return top;
        const uint32_t hi = top & 0xffff0000u, lo = top << 16;
        return hi > lo ? hi : lo;
    }
    // From here on the values are what lies in their registers (else the compiler keeps every value that it has unpacked).
    __device__ __forceinline__ void opaque() {
#pragma unroll
        for (auto &q : v) asm volatile("" : "+v"(q.x), "+v"(q.y), "+v"(q.z), "+v"(q.w));
    }
    // A factor of 0 (a row of zeros, or one that is not finite) gives codes 0 whatever the values are.
    __device__ __forceinline__ uint4 codes(float factor) const {
        if (factor == 0.0f) return make_uint4(0, 0, 0, 0);
        return make_uint4(i8_codes4(value(0), value(1), value(2), value(3), factor), i8_codes4(value(4), value(5), value(6), value(7), factor),
                          i8_codes4(value(8), value(9), value(10), value(11), factor), i8_codes4(value(12), value(13), value(14), value(15), factor));
    }
};

}  // namespace ssg
