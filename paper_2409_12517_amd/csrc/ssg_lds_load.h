// Loads straight to LDS in two statements, and loops over constants: what the tiles that stream blocks of 1 KB share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace ssg {

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

}  // namespace ssg
