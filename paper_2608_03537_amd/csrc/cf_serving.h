// Host <-> kernel interface of the serving operators (not part of the C ABI), apart from
// cf_internal.h, whose text dates the measured traffic of the headline kernel.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cf {

// RMSNorm with the residual's addition and 8-bit codes (cf_rms_quant.hip).
struct RmsQuantParams {
  int M, N, f32;                           // f32: X, R and H are fp32, else bf16
  const void* X; int64_t ldx;
  const void* R; int64_t ldr;              // or NULL
  void* H; int64_t ldh;                    // or NULL
  const float* gamma;                      // or NULL
  int norm; float eps;
  int e4m3;                                // codes: E4M3, else int8
  void* Q; int64_t ldq; float* s;
};
constexpr int64_t kRmsQuantMaxN = 32768;
hipError_t launch_rms_quant(const RmsQuantParams& p, hipStream_t st);

// int8 product (cf_gemm_i8.hip).
struct GemmI8Params {
  int M, N, K;
  const int8_t* A; int64_t lda;
  const int8_t* B; int64_t ldb;
  const float* sa; const float* sb; const float* bias;   // each or NULL
  int act;                                 // ActKind
  void* C; int64_t ldc; int c_f32;
};
hipError_t launch_gemm_i8(const GemmI8Params& p, hipStream_t st);
void gemm_i8_form(const GemmI8Params& p, char* text, size_t bytes);   // from M, N, K, lda, ldb

// Attention over a shared prefix and each sequence's own keys (cf_prefix.hip).
struct PrefixParams {
  int B, H, Hk, Lq, P, S, d;
  const uint16_t* Q;  int64_t q_b, q_h, q_l;
  const uint16_t* Kp; int64_t kp_h, kp_l;
  const uint16_t* Vp; int64_t vp_h, vp_l;
  const uint16_t* Ks; int64_t ks_b, ks_h, ks_l;
  const uint16_t* Vs; int64_t vs_b, vs_h, vs_l;
  const int32_t* lens;                     // or NULL
  int causal; float scale;
  uint16_t* O; int64_t o_b, o_h, o_l;
  float* ws;
};
constexpr int64_t kPrefixMaxKeys = (int64_t)1 << 30;   // of the prefix, and of the own keys
size_t prefix_workspace(const PrefixParams& p);
hipError_t launch_prefix(const PrefixParams& p, hipStream_t st);
void prefix_form(const PrefixParams& p, char* text, size_t bytes);   // from the sizes

}  // namespace cf
