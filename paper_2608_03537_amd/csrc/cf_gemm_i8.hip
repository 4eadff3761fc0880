// Matrix product of 8-bit integers with a scale per token and per channel:
//     C[m, n] = act(float(sum_k A[m, k] B[n, k]) sa[m] sb[n] + bias[n]).
// The sum is exact in 32 bits for K <= 131056 (|product| <= 2^14), so the order
// of its terms is free: waves may split K and tiles may differ in shape without
// changing a bit.
#include <algorithm>

#include "cf_device.h"
#include "cf_internal.h"

namespace cf {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4_t;
typedef __attribute__((__vector_size__(16 * sizeof(int)))) int i32x16_t;

// D (32 n x 32 m) += W (32 n x 32 k) X (32 k x 32 m): lane l gives 16 k of row l % 32 of
// either operand, k group l / 32; layout of D as for the bf16 atom (acc_row).
__device__ __forceinline__ void mma_i8(i32x16_t& acc, u32x4_t w, u32x4_t x) {
  acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4_t, w), __builtin_bit_cast(i32x4_t, x), acc, 0, 0,
                                              0);
}

__device__ __forceinline__ float act_i8(float x, int act) {
  if (act == ACT_GELU) return gelu_erf(x);
  if (act == ACT_GELU_TANH) return gelu_tanh(x);
  if (act == ACT_RELU) return x < 0.0f ? 0.0f : x;
  return x;
}

// 64 x 64 tile, four waves of 32 x 32, operands straight from global memory.
__global__ __launch_bounds__(256) void gemm_i8_direct_kernel(GemmI8Params p) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lr = lane & 31, lg = lane >> 5;
  const int m0 = blockIdx.x * 64 + (wave >> 1) * 32, n0 = blockIdx.y * 64 + (wave & 1) * 32;
  const int8_t* a = p.A + (int64_t)min(m0 + lr, p.M - 1) * p.lda;
  const int8_t* b = p.B + (int64_t)min(n0 + lr, p.N - 1) * p.ldb;
  i32x16_t acc = {};
  for (int k = lg * 16; k - lg * 16 < p.K; k += 32) {
    const u32x4_t zero = {};
    const bool in = k < p.K;   // K is a multiple of 16
    mma_i8(acc, in ? gload16(b + k) : zero, in ? gload16(a + k) : zero);
  }
  const int m = m0 + lr;
  if (m >= p.M) return;
  const float sa = p.sa ? p.sa[m] : 1.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = n0 + acc_row(i, lane);
    if (n >= p.N) continue;
    float x = (float)acc[i] * sa * (p.sb ? p.sb[n] : 1.0f);
    if (p.bias) x += p.bias[n];
    x = act_i8(x, p.act);
    const int64_t at = (int64_t)m * p.ldc + n;
    if (p.c_f32) reinterpret_cast<float*>(p.C)[at] = x;
    else reinterpret_cast<bf16_t*>(p.C)[at] = (bf16_t)pack_bf16x2(x, 0.0f);
  }
}

}  // namespace

hipError_t launch_gemm_i8(const GemmI8Params& p, hipStream_t st) {
  const dim3 grid((unsigned)((p.M + 63) / 64), (unsigned)((p.N + 63) / 64));
  hipLaunchKernelGGL(gemm_i8_direct_kernel, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace cf
