// Device helpers of the attention kernels: packed P fragments, LDS reads as
// inline assembly with their waits, lane-pair reductions.
#pragma once

#include <type_traits>

#include "cf_device.h"

namespace cf {

// Accumulator elements 8s .. 8s+7 of a block, as 8 packed bf16.
__device__ __forceinline__ u32x4_t pack_step(const f32x16_t& v, int s) {
  return u32x4_t{pack_bf16x2(v[8 * s + 0], v[8 * s + 1]), pack_bf16x2(v[8 * s + 2], v[8 * s + 3]),
                 pack_bf16x2(v[8 * s + 4], v[8 * s + 5]), pack_bf16x2(v[8 * s + 6], v[8 * s + 7])};
}

// Transposing 8-byte LDS read (ds_read_b64_tr_b16) at LDS byte address
// addr + OFF, written as inline assembly.  The compiler builtin carries no
// memory operand, so the compiler's wait insertion assumes it may read bytes
// that an outstanding direct-to-LDS load is still writing and puts a wait for
// every such load (vmcnt(0)) in front of it.  The caller knows the stage it
// reads is not the one being loaded; it waits for the result itself
// (lgkm_wait), since the compiler does not know this instruction loads.
template <int OFF>
__device__ __forceinline__ u32x2_t ds_read_tr_b64(uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "ds offset field");
  u32x2_t v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}
// 16-byte LDS read at byte address addr + OFF as inline assembly, for the
// same reason (K rows sit in a stage that direct loads also write); the
// caller waits for the result.
template <int OFF>
__device__ __forceinline__ u32x4_t ds_read_b128_at(uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "ds offset field");
  u32x4_t v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}
// Wait until at most N LDS operations of this wave are outstanding; v is tied
// to the wait so that its uses cannot move above it.  The count is exact only
// while no scalar memory load is in flight (they share the counter and return
// out of order): the kernel's loop issues none, and each step begins with a
// full wait (lds_sync).
template <int N>
__device__ __forceinline__ void lgkm_wait(u32x4_t& v) {
  asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(v) : "i"(N));
}
// Calls f(std::integral_constant<int, I>) for I = B .. E-1 in order.
template <int B, int E, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>{});
    static_for<B + 1, E>(f);
  }
}

__device__ __forceinline__ float lane_pair_sum(float v) { return v + __shfl_xor(v, 32); }
__device__ __forceinline__ float lane_pair_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }

// lane_pair_max without a trip through LDS: v_permlane32_swap exchanges the upper half of its first
// operand with the lower half of its second, so of two copies every lane gets both halves' values.
__device__ __forceinline__ float lane_pair_max_swap(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return v;
#endif
}

// Accesses that are coherent between the XCDs (bytes `off` behind base, below 2^31), for data that
// workgroups of one launch hand to each other.
__device__ __forceinline__ void coherent_store16(float* base, uint32_t off, u32x4_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_raw_buffer_store_b128(v, __builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7FFFFFFF, 0x00020000), off, 0, 16);
#endif
}
__device__ __forceinline__ void coherent_store8(float* base, uint32_t off, u32x2_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_raw_buffer_store_b64(v, __builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7FFFFFFF, 0x00020000), off, 0, 16);
#endif
}
__device__ __forceinline__ u32x4_t coherent_load16(float* base, uint32_t off) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7FFFFFFF, 0x00020000), off, 0, 16);
#else
  return u32x4_t{};
#endif
}
__device__ __forceinline__ u32x2_t coherent_load8(float* base, uint32_t off) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_raw_buffer_load_b64(__builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7FFFFFFF, 0x00020000), off, 0, 16);
#else
  return u32x2_t{};
#endif
}

// dma16 from base + lane_off + wave_off bytes (base and wave_off wave-uniform, offsets below 2^31): the
// address takes no vector arithmetic beyond the lane's own offset.
__device__ __forceinline__ void dma16_at(const char* base, uint32_t lane_off, uint32_t wave_off, char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0x7FFFFFFF, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, lane_off, wave_off, 0,
                                           0);
#endif
}

}  // namespace cf
