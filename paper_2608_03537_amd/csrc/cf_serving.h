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

// 4-bit weights (cf_w4.hip).  code: CF_I4 or CF_FP4_E2M1.
struct W4QuantParams {
  int N, K, group, f32, e2m1;              // f32: W is fp32, else bf16
  const void* W; int64_t ldw;
  uint8_t* tiles;
  void* s; int64_t lds; int s_f32;
};
hipError_t launch_w4_quant(const W4QuantParams& p, hipStream_t st);
hipError_t launch_w4_pack(int N, int K, const uint8_t* codes, int64_t ldc, uint8_t* tiles, hipStream_t st);
struct GemmW4Params {
  int M, N, K, group;
  const uint16_t* A; int64_t lda;
  int e2m1;
  const uint8_t* W;
  const void* s; int64_t lds; int s_f32;
  const float* bias;                       // or NULL
  int act;                                 // ActKind
  void* C; int64_t ldc; int c_f32;
};
hipError_t launch_gemm_w4(const GemmW4Params& p, hipStream_t st);
void gemm_w4_form(const GemmW4Params& p, char* text, size_t bytes);   // from the sizes

// Pages of keys and values (cf_cache.hip, cf_paged.hip).
enum CacheCode { CACHE_BF16 = 0, CACHE_I8 = 1, CACHE_E4M3 = 2 };
struct CachePages {
  int code, n_pages, shift;                // pages of 2^shift tokens
  char* K; int64_t k_p, k_h, k_l;          // strides in bytes
  char* V; int64_t v_p, v_h, v_l;
  float* Ks; int64_t ks_p, ks_h;           // in elements
  float* Vs; int64_t vs_p, vs_h;
};
struct CacheWriteParams {
  int T, H, Hk, d;
  const uint16_t* Q; int64_t q_t, q_h;
  uint16_t* Qo; int64_t qo_t, qo_h;
  const uint16_t* K; int64_t k_t, k_h;
  const uint16_t* V; int64_t v_t, v_h;
  const int32_t* slots;
  int rot, neighbours;
  const int32_t* pos; int64_t ldpos;
  const float* freq;
  int first[4];                            // first pair of axes 1 .. 3 (those behind the last: rot / 2), and rot / 2
  CachePages c;
};
hipError_t launch_cache_write(const CacheWriteParams& p, hipStream_t st);
struct CacheReadParams {
  int B, Hk, S, d;
  CachePages c;
  const int32_t* table; int64_t ldt; int pages;
  const int32_t* lens;
  uint16_t* K; int64_t k_b, k_h, k_l;
  uint16_t* V; int64_t v_b, v_h, v_l;
};
hipError_t launch_cache_read(const CacheReadParams& p, hipStream_t st);
struct PagedParams {
  int B, H, Hk, Lq, d;
  const uint16_t* Q; int64_t q_b, q_h, q_l;
  CachePages c;
  const int32_t* table; int64_t ldt; int pages;
  const int32_t* lens;
  int causal; float scale, softcap;
  uint16_t* O; int64_t o_b, o_h, o_l;
  float* ws;
};
size_t paged_workspace(const PagedParams& p);
hipError_t launch_paged(const PagedParams& p, hipStream_t st);
void paged_form(const PagedParams& p, char* text, size_t bytes);   // from the sizes

}  // namespace cf
