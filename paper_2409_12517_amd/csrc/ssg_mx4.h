// Device helpers of microscaled 4-bit floating point: a block's scale and its codes.
//
// A block is 32 neighbours along K.  With amax its largest magnitude, 2^e <= amax < 2^(e+1):
//   floor rule   X = 2^(e - 2): amax / X lies from 4 to 8, and magnitudes above 6 saturate
//   ceil rule    X the smallest power of two with amax / X <= 6
// X is kept as the byte log2 X + 127, 0 to 252 (so that 6 X is finite; beyond, and below 2^-127, X is the nearest there is).  The codes are
// E2M1: the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 to |x| / X, between two the one whose code is even, with the sign.  x / X is exact.
// A block with a NaN or an infinity has the byte 255, the format's NaN, and codes 0: everything made from it is NaN.
#pragma once
#include "ssg_device.h"
#include "ssg_i8.h"

namespace ssg {

// From the bits of the largest magnitude (those of a NaN or an infinity stand above every number's).
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t top_bits, int ceil) {
    if (top_bits >= 0x7f800000u) return 255u;
    const int e = (int)(top_bits >> 23) + (ceil && (top_bits & 0x7fffffu) > 0x400000u) - 2;
    return (uint32_t)(e < 0 ? 0 : e > 252 ? 252 : e);
}
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x400000u); }

// The word of the lane beside (D = 1) or one over (D = 2) among four neighbouring ones.
template <int D> __device__ __forceinline__ uint32_t quad_xor(uint32_t v) {
    static_assert(D == 1 || D == 2, "of four");
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, D == 1 ? 0xb1 : 0x4e, 0xf, 0xf, true);     // quad_perm [1,0,3,2], [2,3,0,1]
}
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = quad_xor<1>(v);
    v = v > o ? v : o;
    o = quad_xor<2>(v);
    return v > o ? v : o;
}

// Eight values to eight codes, by the conversion instruction (nearest, ties to even codes, saturating), which divides by the scale itself.
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
}
// The same from four words of two bf16 each.
__device__ __forceinline__ uint32_t mx4_codes8(const uint32_t (&w)[4], float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(ssg_bf16x2, w[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(ssg_bf16x2, w[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(ssg_bf16x2, w[2]), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(ssg_bf16x2, w[3]), scale, 3);
}

// The 32 values of a block in the registers of one lane.
template <bool BF16> struct Mx4Block {
    I8Run<BF16> half[2];
    // columns from col on of a row of K, a multiple of 16; beyond it zeros
    __device__ __forceinline__ void load(const uint8_t *row, int64_t col, int64_t K, bool live) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            half[h].clear();
            if (live && col + 16 * h < K) half[h].load(row, (int)(col / 16) + h);
        }
    }
    __device__ __forceinline__ uint32_t top_bits() const { return I8Run<BF16>::as_f32_bits(half[1].max_bits(half[0].max_bits(0))); }
    __device__ __forceinline__ uint4 codes(uint32_t byte) const {
        const float scale = mx4_scale(byte);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                const uint4 q = half[i / 2].v[i % 2];
                const uint32_t words[4] = {q.x, q.y, q.z, q.w};
                w[i] = mx4_codes8(words, scale);
            } else {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = half[i / 2].value(i % 2 * 8 + j);
                w[i] = mx4_codes8(f, scale);
            }
        }
        return byte == 255u ? make_uint4(0, 0, 0, 0) : make_uint4(w[0], w[1], w[2], w[3]);
    }
};

}  // namespace ssg
