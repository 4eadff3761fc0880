// Residual addition, RMSNorm and 8-bit codes with a scale per row, one pass:
//     h = x + r,  t = h gamma,  d = max |t| / qmax,  q = code(t / d),
//     s = d / sqrt(mean(h^2) + eps).
// A row's values stay in registers between the pass that reduces and the pass
// that encodes them, so every byte is read and written once; memory bounds it.
//
// The normed row is t / rms, and rms cancels in (t / rms) / (d / rms): the codes
// come from t and its maximum alone.  A maximum does not depend on the order of
// its terms, so the codes are the same bits however a row is spread over lanes,
// and the sum of squares (fp32, order fixed by the width) enters s only.  It is kept scaled by
// 2^-144 as well, for rows whose sum passes fp32's range.
#include <algorithm>

#include "cf_device.h"
#include "cf_serving.h"

namespace cf {

namespace {

constexpr float kUp = 1.8446744073709552e19f, kDown = 5.4210108624275222e-20f;   // 2^64, 2^-64
constexpr float kSmall = 8.6736173798840355e-19f;                                // 2^-60
// Of N <= 2^15 finite h, (2^-72 h)^2 adds up to less than 2^128; a row whose plain sum passes 2^128 has
// |h| of 2^56 and more, whose scaled squares are normal.
constexpr float kLow = 2.1175823681357508e-22f, kLow2 = 4.4841550858394146e-44f, kHalfLow = 1.4551915228366852e-11f;   // 2^-72, 2^-144, 2^-36

// E = 16 / sizeof(T) consecutive elements of a row as fp32; elements at and
// behind `left` are 0 and not read.
template <typename T, int E>
__device__ __forceinline__ void load_chunk(const T* p, int left, float (&v)[E]) {
  if (left >= E) {
    const u32x4_t u = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        v[i] = __uint_as_float(u[i]);
      } else {
        v[2 * i] = bf16_to_f32(u[i] & 0xFFFFu);
        v[2 * i + 1] = bf16_to_f32(u[i] >> 16);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = 0.0f;
    if (left <= 0) return;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) v[i] = p[i];
        else v[i] = bf16_to_f32(p[i]);
      }
  }
}

template <typename T, int E>
__device__ __forceinline__ void store_chunk(T* p, int left, const float (&v)[E]) {
  if (left >= E) {
    u32x4_t u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(v[i]);
      else u[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    }
    __builtin_nontemporal_store(u, reinterpret_cast<u32x4_t*>(p));
  } else if (left > 0) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) p[i] = v[i];
        else p[i] = (bf16_t)pack_bf16x2(v[i], 0.0f);
      }
  }
}

// Four quotients -> four int8 codes, byte e from the e-th: adding 1.5 * 2^23 to
// |z| <= 2^22 leaves round(z) (to nearest, ties to even) in the low mantissa bits.
__device__ __forceinline__ uint32_t i8x4(float a, float b, float c, float d) {
  constexpr float kMagic = 12582912.0f;
  const uint32_t x = __float_as_uint(a + kMagic), y = __float_as_uint(b + kMagic);
  const uint32_t z = __float_as_uint(c + kMagic), w = __float_as_uint(d + kMagic);
  return (x & 0xFFu) | (y & 0xFFu) << 8 | (z & 0xFFu) << 16 | w << 24;
}

// TPR threads a row, C chunks of E elements a thread; NT / TPR rows a workgroup.
template <typename T, int TPR, int C, int NT>
__global__ __launch_bounds__(NT) void rms_quant_kernel(RmsQuantParams p) {
  constexpr int E = 16 / (int)sizeof(T), ROWS = NT / TPR, W = TPR / 64;
  static_assert(W == 1 || ROWS == 1, "a row is one wave's or the workgroup's");
  const int tid = threadIdx.x, lane = tid & 63, t = tid % TPR;
  const int64_t row = (int64_t)blockIdx.x * ROWS + tid / TPR;
  if (W == 1 && row >= p.M) return;   // whole waves; no barrier follows with one wave a row
  const T* X = reinterpret_cast<const T*>(p.X) + row * p.ldx;
  const T* R = reinterpret_cast<const T*>(p.R) + row * p.ldr;
  T* H = reinterpret_cast<T*>(p.H) + row * p.ldh;

  float v[C][E];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int n = (c * TPR + t) * E;
    load_chunk<T, E>(X + n, p.N - n, v[c]);
  }
  if (p.R) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = (c * TPR + t) * E;
      float r[E];
      load_chunk<T, E>(R + n, p.N - n, r);
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] += r[e];
    }
  }
  float ss = 0.0f, far = 0.0f;
  uint32_t mb = 0;   // maximum of |t| by its bits: a NaN is above infinity, so it is kept
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int n = (c * TPR + t) * E;
    if (n >= p.N) break;
    if (p.H) store_chunk<T, E>(H + n, p.N - n, v[c]);
    if (W == 1 || p.norm) {   // narrow rows always: the branch costs them more (65536 x 256 fp32 39 -> 41 us)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float low = v[c][e] * kLow;
        ss = fmaf(v[c][e], v[c][e], ss);
        far = fmaf(low, low, far);
      }
    }
    if (p.gamma) {
      float g[E];
      if (p.N - n >= E) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
          const f32x4_t q = *reinterpret_cast<const f32x4_t*>(p.gamma + n + i);
#pragma unroll
          for (int e = 0; e < 4; ++e) g[i + e] = q[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = n + e < p.N ? p.gamma[n + e] : 0.0f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] *= g[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) mb = max(mb, __float_as_uint(v[c][e]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    ss += __shfl_xor(ss, o);
    mb = max(mb, (uint32_t)__shfl_xor((int)mb, o));
  }
  if constexpr (W > 1) {
    __shared__ float ss_w[W];
    __shared__ uint32_t mb_w[W];
    if (lane == 0) {
      ss_w[tid >> 6] = ss;
      mb_w[tid >> 6] = mb;
    }
    __syncthreads();
    ss = 0.0f;
    mb = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      ss += ss_w[w];
      mb = max(mb, mb_w[w]);
    }
  }

  const float qmax = p.e4m3 ? 448.0f : 127.0f;
  const float m = __uint_as_float(mb);
  const bool ok = mb != 0 && mb < 0x7F800000u;   // some value, and all finite
  const bool over = ok && p.norm && !(ss < INFINITY);   // the same in every thread of the row
  if (over) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) far += __shfl_xor(far, o);
    if constexpr (W > 1) {
      __shared__ float far_w[W];
      if (lane == 0) far_w[tid >> 6] = far;
      __syncthreads();
      far = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) far += far_w[w];
    }
  }
  // Small rows are raised by 2^64 (exact), so that d and 1 / d stay normal.
  const float up = m < kSmall ? kUp : 1.0f;
  const float d = ok ? m * up / qmax : 1.0f, rd = 1.0f / d;
  if (t == 0) {
    float s = m < kSmall ? d * kDown : d;
    if (over)
      s = d * kHalfLow * (1.0f / sqrtf(far / (float)p.N + p.eps * kLow2)) * kHalfLow * (m < kSmall ? kDown : 1.0f);
    else if (p.norm)
      s = m < kSmall ? d * (1.0f / sqrtf(ss / (float)p.N + p.eps)) * kDown : d / sqrtf(ss / (float)p.N + p.eps);
    p.s[row] = mb == 0 ? 0.0f : ok ? s : __uint_as_float(0x7FC00000u);
  }
  uint8_t* Q = reinterpret_cast<uint8_t*>(p.Q) + row * p.ldq;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int n = (c * TPR + t) * E;
    if (n >= p.N) break;
    uint32_t w[E / 4];
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      float z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = div_rn(v[c][i + e] * up, d, rd);
      const uint32_t q = p.e4m3 ? e4m3x4(z[0], z[1], z[2], z[3]) : i8x4(z[0], z[1], z[2], z[3]);
      w[i / 4] = ok ? q : 0u;
    }
    if (p.N - n >= E) {
      if constexpr (E == 8) __builtin_nontemporal_store(u32x2_t{w[0], w[1]}, reinterpret_cast<u32x2_t*>(Q + n));
      else __builtin_nontemporal_store(w[0], reinterpret_cast<uint32_t*>(Q + n));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (n + e < p.N) Q[n + e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
    }
  }
}

template <typename T, int TPR, int C, int NT>
hipError_t launch(RmsQuantParams p, hipStream_t st) {
  constexpr int ROWS = NT / TPR;
  constexpr int64_t kMost = ((int64_t)1 << 31) / NT * ROWS;   // rows a launch: a grid has less than 2^32 threads
  hipError_t e = hipSuccess;
  for (int64_t left = p.M; left > 0 && e == hipSuccess; left -= kMost) {
    p.M = (int)std::min(left, kMost);
    hipLaunchKernelGGL((rms_quant_kernel<T, TPR, C, NT>), dim3((unsigned)((p.M + ROWS - 1) / ROWS)), dim3(NT), 0, st, p);
    e = hipGetLastError();
    p.X = reinterpret_cast<const T*>(p.X) + p.M * p.ldx;
    if (p.R) p.R = reinterpret_cast<const T*>(p.R) + p.M * p.ldr;
    if (p.H) p.H = reinterpret_cast<T*>(p.H) + p.M * p.ldh;
    p.Q = reinterpret_cast<uint8_t*>(p.Q) + p.M * p.ldq;
    p.s += p.M;
  }
  return e;
}

}  // namespace

// The narrowest form that holds a row: chunks behind N cost their checks, and more threads a
// row with fewer chunks keep more rows of loads in flight.  Measured (us; 16 bytes a thread and
// chunk): 16384 x 4096 bf16 with residual 80 on 256 threads x 2 chunks, 86 on 512 x 2, 93 on 256 x 4, 115 on
// 64 x 8; 4096 x 16384 bf16 without 39 on 1024 x 2, 46 on 512 x 4, 69 on 256 x 8; 65536 x 1024 77 on 64 x
// 2, 117 on 256 x 2; 16384 x 2048 45 on 64 x 4; fp32 8192 x 4096 74 on 512 x 2, 777 x 5120 6.7 on 512 x 4 and 8.2
// on 1024 x 2.  16384 x 4096 is 470 MB at 5.9 TB/s, the rate of a large sum of two arrays (5.85;
// a large read reaches 6.4, a large copy 4.9).  One row takes about 4 us, the launch.
hipError_t launch_rms_quant(const RmsQuantParams& p, hipStream_t st) {
  if (p.f32) {
    if (p.N <= 256) return launch<float, 64, 1, 256>(p, st);
    if (p.N <= 512) return launch<float, 64, 2, 256>(p, st);
    if (p.N <= 1024) return launch<float, 64, 4, 256>(p, st);
    if (p.N <= 2048) return launch<float, 256, 2, 256>(p, st);
    if (p.N <= 4096) return launch<float, 512, 2, 512>(p, st);
    if (p.N <= 8192) return launch<float, 512, 4, 512>(p, st);
    if (p.N <= 16384) return launch<float, 1024, 4, 1024>(p, st);
    return launch<float, 1024, 8, 1024>(p, st);
  }
  if (p.N <= 512) return launch<bf16_t, 64, 1, 256>(p, st);
  if (p.N <= 1024) return launch<bf16_t, 64, 2, 256>(p, st);
  if (p.N <= 2048) return launch<bf16_t, 64, 4, 256>(p, st);
  if (p.N <= 4096) return launch<bf16_t, 256, 2, 256>(p, st);
  if (p.N <= 8192) return launch<bf16_t, 512, 2, 512>(p, st);
  if (p.N <= 16384) return launch<bf16_t, 1024, 2, 1024>(p, st);
  return launch<bf16_t, 1024, 4, 1024>(p, st);
}

}  // namespace cf
