// Rows of keys and values into and out of a cache of pages.
//
// Write: rotary positions of queries and keys, then bf16 rows or 8-bit codes with a scale per
// token and head, straight from the projection's output: every byte is read and written
// once, memory bounds it.  A workgroup takes rows of one token, whose cosines
// and sines (64 bits, rounded to fp32) it computes once into LDS.
// A thread has two 8-element chunks of a row, so that both elements of a pair are its own:
// chunks u and u + rot / 16 where pairs are halves, and any two where they are neighbours.
// Rotation and codes are single fp32 operations in a fixed order (no fused steps), so the codes are those of
// the formula in fp32, bit for bit.
#include <algorithm>

#include "cf_device.h"
#include "cf_serving.h"

namespace cf {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostBlocks = 1 << 20;   // of a grid; more tasks are looped over

__device__ __forceinline__ void unpack8(u32x4_t u, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_to_f32(u[i] & 0xFFFFu);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4_t pack8(const float* v) {
  return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// (x, y) -> (x c - y s, y c + x s), each operation rounded by itself
__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
  const float a = x * c, b = y * s, d = y * c, e = x * s;
  x = a - b;
  y = d + e;
}

// Four |z| <= 127 -> int8 codes, nearest, ties to even (the sum's low mantissa bits).
__device__ __forceinline__ uint32_t codes_i8(const float* z) {
  constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) w |= (__float_as_uint(z[e] + kMagic) & 0xFFu) << (8 * e);
  return w;
}

template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheWriteParams p, int64_t tasks, int nrb) {
  constexpr int TPR = D / 16, RPW = kThreads / TPR;   // threads a row, rows of a workgroup
  __shared__ float cs[D / 2], sn[D / 2];
  const int tid = threadIdx.x, u = tid % TPR, half = p.rot / 2;
  // first elements of the thread's chunks
  const int a0 = 8 * u < half ? 8 * u : p.rot + 16 * (u - half / 8), b0 = 8 * u < half ? 8 * u + half : a0 + 8;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int t = (int)(task / nrb), r = (int)(task % nrb) * RPW + tid / TPR;
    const bool is_q = r < p.H, is_k = !is_q && r < p.H + p.Hk, any = r < p.H + 2 * p.Hk;
    const int hk = is_k ? r - p.H : r - p.H - p.Hk;
    u32x4_t xa = {}, xb = {};
    if (any) {
      const bf16_t* src = is_q ? p.Q + t * p.q_t + r * p.q_h : is_k ? p.K + t * p.k_t + hk * p.k_h : p.V + t * p.v_t + hk * p.v_h;
      xa = gload16(src + a0);
      xb = gload16(src + b0);
    }
    const int slot = p.slots[t];
    if (p.rot > 0) {
      if (tid < half) {
        const int axis = (tid >= p.first[0]) + (tid >= p.first[1]) + (tid >= p.first[2]);
        double s, c;
        sincos((double)p.pos[axis * p.ldpos + t] * (double)p.freq[tid], &s, &c);
        cs[tid] = (float)c;
        sn[tid] = (float)s;
      }
      __syncthreads();
    }
    float v[16];
    unpack8(xa, v);
    unpack8(xb, v + 8);
    if (8 * u < half && (is_q || is_k)) {
      if (p.neighbours) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          turn(v[2 * e], v[2 * e + 1], cs[a0 / 2 + e], sn[a0 / 2 + e]);
          turn(v[8 + 2 * e], v[9 + 2 * e], cs[b0 / 2 + e], sn[b0 / 2 + e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(v[e], v[8 + e], cs[a0 + e], sn[a0 + e]);
      }
    }
    if (p.rot > 0) __syncthreads();   // the next task's table
    if (is_q) {
      bf16_t* dst = p.Qo + t * p.qo_t + r * p.qo_h;
      *reinterpret_cast<u32x4_t*>(dst + a0) = pack8(v);
      *reinterpret_cast<u32x4_t*>(dst + b0) = pack8(v + 8);
    }
    const bool in = any && !is_q && slot >= 0 && (slot >> p.c.shift) < p.c.n_pages;
    const int64_t page = in ? slot >> p.c.shift : 0, l = slot & ((1 << p.c.shift) - 1);
    char* row = is_k ? p.c.K + page * p.c.k_p + hk * p.c.k_h + l * p.c.k_l : p.c.V + page * p.c.v_p + hk * p.c.v_h + l * p.c.v_l;
    if constexpr (CODE == CACHE_BF16) {
      if (in) {
        *reinterpret_cast<u32x4_t*>(row + 2 * a0) = pack8(v);
        *reinterpret_cast<u32x4_t*>(row + 2 * b0) = pack8(v + 8);
      }
    } else {
      constexpr float kMax = CODE == CACHE_I8 ? 127.0f : 448.0f;
      uint32_t mb = 0;   // max |x| by its bits: a NaN is above infinity, so it is kept
#pragma unroll
      for (int e = 0; e < 16; ++e) mb = max(mb, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
      for (int s = 1; s < TPR; s *= 2) mb = max(mb, (uint32_t)__shfl_xor((int)mb, s));
      const bool bad = mb >= 0x7F800000u;
      const float d = __uint_as_float(mb) / kMax;
      float z[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = v[e] / d;
        z[e] = !bad && d > 0.0f ? fminf(fmaxf(w, -kMax), kMax) : 0.0f;   // a subnormal d may be far below its quotient
      }
      if (in) {
        u32x2_t ca, cb;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (CODE == CACHE_I8) {
            ca[i] = codes_i8(z + 4 * i);
            cb[i] = codes_i8(z + 8 + 4 * i);
          } else {
            ca[i] = e4m3x4(z[4 * i], z[4 * i + 1], z[4 * i + 2], z[4 * i + 3]);
            cb[i] = e4m3x4(z[8 + 4 * i], z[9 + 4 * i], z[10 + 4 * i], z[11 + 4 * i]);
          }
        }
        *reinterpret_cast<u32x2_t*>(row + a0) = ca;
        *reinterpret_cast<u32x2_t*>(row + b0) = cb;
        if (u == 0) {
          float* sc = is_k ? p.c.Ks + page * p.c.ks_p + hk * p.c.ks_h : p.c.Vs + page * p.c.vs_p + hk * p.c.vs_h;
          sc[l] = bad ? __uint_as_float(0x7FC00000u) : d;
        }
      }
    }
  }
}

// Read: D / 8 threads a row, which write 16 bytes each; a workgroup takes 64 rows of a (sequence, head), keys and values.
constexpr int kReadRows = 64;
template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheReadParams p, int64_t tasks, int nch) {
  constexpr int TPR = D / 8, RPP = kThreads / TPR, E = CODE == CACHE_BF16 ? 2 : 1;
  const int r = threadIdx.x / TPR, c = threadIdx.x % TPR * 8;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int ch = (int)(task % nch), hk = (int)(task / nch % p.Hk), b = (int)(task / nch / p.Hk);
    const int64_t most = min((int64_t)p.S, (int64_t)p.pages << p.c.shift);
    const int len = (int)min((int64_t)max(p.lens[b], 0), most);
#pragma unroll 4
    for (int i = 0; i < kReadRows / RPP; ++i) {
      const int64_t j = (int64_t)ch * kReadRows + i * RPP + r;
      if (j >= len) break;
      const int page = p.table[b * p.ldt + (j >> p.c.shift)];
      if ((uint32_t)page >= (uint32_t)p.c.n_pages) continue;
      const int64_t l = j & ((1 << p.c.shift) - 1);
      auto one = [&](const char* row, const float* scale, bf16_t* out) {
        if constexpr (CODE == CACHE_BF16) {
          *reinterpret_cast<u32x4_t*>(out) = gload16(row + c * E);
        } else {
          const u32x2_t w = *reinterpret_cast<const u32x2_t*>(row + c * E);
          const float s = scale[l];
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if constexpr (CODE == CACHE_I8) v[e] = (float)(int8_t)(w[e / 4] >> (8 * (e % 4)));
          }
          if constexpr (CODE == CACHE_E4M3) {
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
              const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i2], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i2], true);
              v[4 * i2] = lo[0];
              v[4 * i2 + 1] = lo[1];
              v[4 * i2 + 2] = hi[0];
              v[4 * i2 + 3] = hi[1];
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= s;
          *reinterpret_cast<u32x4_t*>(out) = pack8(v);
        }
      };
      one(p.c.K + page * p.c.k_p + hk * p.c.k_h + l * p.c.k_l, CODE ? p.c.Ks + page * p.c.ks_p + hk * p.c.ks_h : nullptr,
          p.K + b * p.k_b + hk * p.k_h + j * p.k_l + c);
      one(p.c.V + page * p.c.v_p + hk * p.c.v_h + l * p.c.v_l, CODE ? p.c.Vs + page * p.c.vs_p + hk * p.c.vs_h : nullptr,
          p.V + b * p.v_b + hk * p.v_h + j * p.v_l + c);
    }
  }
}

template <int D, int CODE>
hipError_t write_d(const CacheWriteParams& p, hipStream_t st) {
  constexpr int RPW = kThreads / (D / 16);
  const int nrb = (p.H + 2 * p.Hk + RPW - 1) / RPW;
  const int64_t tasks = (int64_t)p.T * nrb;
  hipLaunchKernelGGL((cache_write_kernel<D, CODE>), dim3((unsigned)std::min(tasks, kMostBlocks)), dim3(kThreads), 0, st, p, tasks, nrb);
  return hipGetLastError();
}
template <int D, int CODE>
hipError_t read_d(const CacheReadParams& p, hipStream_t st) {
  const int nch = (p.S + kReadRows - 1) / kReadRows;
  const int64_t tasks = (int64_t)p.B * p.Hk * nch;
  hipLaunchKernelGGL((cache_read_kernel<D, CODE>), dim3((unsigned)std::min(tasks, kMostBlocks)), dim3(kThreads), 0, st, p, tasks, nch);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheWriteParams& p, hipStream_t st) {
  if (p.d == 128)
    return p.c.code == CACHE_BF16 ? write_d<128, CACHE_BF16>(p, st) : p.c.code == CACHE_I8 ? write_d<128, CACHE_I8>(p, st)
                                                                                           : write_d<128, CACHE_E4M3>(p, st);
  return p.c.code == CACHE_BF16 ? write_d<64, CACHE_BF16>(p, st) : p.c.code == CACHE_I8 ? write_d<64, CACHE_I8>(p, st)
                                                                                        : write_d<64, CACHE_E4M3>(p, st);
}

hipError_t launch_cache_read(const CacheReadParams& p, hipStream_t st) {
  if (p.d == 128)
    return p.c.code == CACHE_BF16 ? read_d<128, CACHE_BF16>(p, st) : p.c.code == CACHE_I8 ? read_d<128, CACHE_I8>(p, st)
                                                                                          : read_d<128, CACHE_E4M3>(p, st);
  return p.c.code == CACHE_BF16 ? read_d<64, CACHE_BF16>(p, st) : p.c.code == CACHE_I8 ? read_d<64, CACHE_I8>(p, st)
                                                                                       : read_d<64, CACHE_E4M3>(p, st);
}

}  // namespace cf
