// Copies from memory into LDS past the registers, and waits for them.
#pragma once
#include "qtip_device.h"

namespace qtip {

// s_waitcnt that waits until at most n memory loads are outstanding, and for nothing else.
constexpr int vmcnt_only(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0F70; }

// A buffer of `bytes` bytes: what is read behind its end is 0.
__device__ __forceinline__ u32x4_t buffer_of(const void *p, size_t bytes) {
    const uint64_t at = reinterpret_cast<uintptr_t>(p);
    return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)),
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(bytes < 0xFFFFFFFFu ? bytes : 0xFFFFFFFFu)),
                   0x00020000u};
}
// 16 bytes per lane from byte `lane_offset` + `offset` of a buffer into LDS at `to`, lane by lane.  (Written
// out, because the compiler makes every later read of LDS wait for the copy, whatever it reads.  The kernel
// waits for its copies itself; the compiler's own waits only become longer by loads it does not count.)
__device__ __forceinline__ void copy_to_lds(u32x4_t buffer, uint32_t lane_offset, uint32_t offset, const char *to) {
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)to;
    asm volatile("s_mov_b32 m0, %3\n\t"
                 "s_nop 0\n\t"
                 "buffer_load_dwordx4 %0, %1, %2 offen lds"
                 :
                 : "v"(lane_offset), "s"(buffer), "s"(offset), "s"(at)
                 : "memory");
}

template <int N, class F, int I = 0>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, F, I + 1>(static_cast<F &&>(f));
    }
}

}  // namespace qtip
