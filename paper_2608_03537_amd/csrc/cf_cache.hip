// Rows of keys and values into and out of a cache of pages.
//
// Write: rotary positions of queries and keys, then bf16 rows or 8-bit codes with a scale per
// token and head, straight from the projection's output: every byte is read and written
// once, memory bounds it (16384 tokens of 32 + 2 x 8 heads, d 128, to int8: 65 us, 5.7 TB/s).  A wave takes rows of one
// token and finds its cosines and sines itself, so no wave waits for another (workgroups of 32 rows of a token with a table of
// angles that a barrier completes: 102 us).  A thread has two 8-element chunks of a row, so that both elements of a pair
// are its own: chunks u and u + rot / 16 where pairs are halves, and any two where they are neighbours.
// Rotation and codes are single fp32 operations in a fixed order (no fused steps), so the codes are those of
// the formula in fp32, bit for bit.
//
// Read: the rows of a sequence gathered from its pages; memory bounds it (16 sequences of 4096 to 8192 int8 rows of 8 heads,
// d 128: 109 to 114 us, 5.6 to 5.4 TB/s; with a row's loads and stores one after the other 142).
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

// What is written is read by another launch: past the second-level cache (16 x 2000 E4M3 rows read 20.9 -> 15.1 us).
__device__ __forceinline__ void store16(void* p, u32x4_t v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(p)); }
__device__ __forceinline__ void store8(void* p, u32x2_t v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x2_t*>(p)); }

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

// Cosine and sine of x in 64 bits, |x| < 2^45: x - k pi/2 with pi/2 in three parts (Cody and Waite), each step fused, so
// the first leaves no rounding where x and k pi/2 cancel; then the Taylor series on [-pi/4, pi/4] up to x^15 and x^16, whose
// next terms are below 5e-17.  Larger angles (and NaN) give NaN.
__device__ __forceinline__ void cos_sin(double x, float& c, float& s) {
  const double k = rint(x * 0.6366197723675814);
  double r = fma(-k, 1.5707963267948966, x);
  r = fma(-k, 6.123233995736766e-17, r);
  r = fma(-k, -1.4973849048591698e-33, r);
  const double y = r * r;
  double a = -1.0 / 1307674368000.0, b = 1.0 / 20922789888000.0;   // 1 / 15!, 1 / 16!
  a = fma(a, y, 1.0 / 6227020800.0);
  b = fma(b, y, -1.0 / 87178291200.0);
  a = fma(a, y, -1.0 / 39916800.0);
  b = fma(b, y, 1.0 / 479001600.0);
  a = fma(a, y, 1.0 / 362880.0);
  b = fma(b, y, -1.0 / 3628800.0);
  a = fma(a, y, -1.0 / 5040.0);
  b = fma(b, y, 1.0 / 40320.0);
  a = fma(a, y, 1.0 / 120.0);
  b = fma(b, y, -1.0 / 720.0);
  a = fma(a, y, -1.0 / 6.0);
  b = fma(b, y, 1.0 / 24.0);
  b = fma(b, y, -0.5);
  const float sr = (float)fma(a * y, r, r), cr = (float)fma(b, y, 1.0);
  const int quarter = fabs(x) < 35184372088832.0 ? (int)((int64_t)k & 3) : -1;
  const float nan = __uint_as_float(0x7FC00000u);
  c = quarter < 0 ? nan : quarter == 0 ? cr : quarter == 1 ? -sr : quarter == 2 ? -cr : sr;
  s = quarter < 0 ? nan : quarter == 0 ? sr : quarter == 1 ? cr : quarter == 2 ? -sr : -cr;
}

constexpr float kSmall = 8.6736173798840355e-19f;   // 2^-60
// A wave takes NP passes of 64 / TPR rows of a token, TPR threads a row, whose loads are all under way at once while its
// lanes find the token's cosines and sines, one pair each (at most 64), which they exchange through LDS of the wave's own.
template <int D, int CODE, int NP>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheWriteParams p, int64_t tasks, int chunks) {
  constexpr int TPR = D / 16, RPP = 64 / TPR, WAVES = kThreads / 64;
  __shared__ __attribute__((aligned(16))) float table[WAVES][2][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), u = lane % TPR, half = p.rot / 2;
  float* const cs = table[wave][0];
  float* const sn = table[wave][1];
  // first elements of the thread's chunks; whether they are turned, and the first pairs
  const bool turned = 8 * u < half;
  const int a0 = turned ? 8 * u : p.rot + 16 * (u - half / 8), b0 = turned ? 8 * u + half : a0 + 8;
  const int pa = p.neighbours ? a0 / 2 : a0, pb = p.neighbours ? b0 / 2 : a0 + 4;
  for (int64_t task = (int64_t)blockIdx.x * WAVES + wave; task < tasks; task += (int64_t)gridDim.x * WAVES) {
    const int t = (int)(task / chunks), r0 = (int)(task % chunks) * (NP * RPP) + lane / TPR;
    const int slot = p.slots[t];
    u32x4_t xa[NP], xb[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = r0 + i * RPP;
      const bf16_t* src = r < p.H ? p.Q + t * p.q_t + r * p.q_h
                          : r < p.H + p.Hk ? p.K + t * p.k_t + (r - p.H) * p.k_h : p.V + t * p.v_t + (r - p.H - p.Hk) * p.v_h;
      xa[i] = xb[i] = u32x4_t{};
      if (r < p.H + 2 * p.Hk) {
        xa[i] = gload16(src + a0);
        xb[i] = gload16(src + b0);
      }
    }
    f32x4_t c0 = {}, c1 = {}, s0 = {}, s1 = {};
    if (half > 0) {
      if (lane < half) {
        const int axis = (lane >= p.first[0]) + (lane >= p.first[1]) + (lane >= p.first[2]);
        float c, s;
        cos_sin((double)p.pos[axis * p.ldpos + t] * (double)p.freq[lane], c, s);
        cs[lane] = c;
        sn[lane] = s;
      }
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");   // a wave's LDS operations keep their order
      if (turned) {
        c0 = *reinterpret_cast<const f32x4_t*>(cs + pa);
        c1 = *reinterpret_cast<const f32x4_t*>(cs + pb);
        s0 = *reinterpret_cast<const f32x4_t*>(sn + pa);
        s1 = *reinterpret_cast<const f32x4_t*>(sn + pb);
      }
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");
    }
    const bool held = slot >= 0 && (slot >> p.c.shift) < p.c.n_pages;
    const int64_t page = held ? slot >> p.c.shift : 0, l = held ? slot & ((1 << p.c.shift) - 1) : 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = r0 + i * RPP;
      const bool is_q = r < p.H, is_k = !is_q && r < p.H + p.Hk, is_v = !is_q && !is_k && r < p.H + 2 * p.Hk;
      const int hk = is_k ? r - p.H : r - p.H - p.Hk;
      float v[16];
      unpack8(xa[i], v);
      unpack8(xb[i], v + 8);
      if (turned && (is_q || is_k)) {
        if (p.neighbours) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            turn(v[2 * e], v[2 * e + 1], c0[e], s0[e]);
            turn(v[8 + 2 * e], v[9 + 2 * e], c1[e], s1[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            turn(v[e], v[8 + e], c0[e], s0[e]);
            turn(v[4 + e], v[12 + e], c1[e], s1[e]);
          }
        }
      }
      char* to = is_q ? reinterpret_cast<char*>(p.Qo + t * p.qo_t + r * p.qo_h)
                 : is_k ? p.c.K + page * p.c.k_p + l * p.c.k_l + hk * p.c.k_h : p.c.V + page * p.c.v_p + l * p.c.v_l + hk * p.c.v_h;
      const bool put = held && (is_k || is_v);
      if (is_q || (CODE == CACHE_BF16 && put)) {
        store16(to + 2 * a0, pack8(v));
        store16(to + 2 * b0, pack8(v + 8));
      }
      if constexpr (CODE != CACHE_BF16) {
        if (!__any(put)) continue;
        constexpr float kMax = CODE == CACHE_I8 ? 127.0f : 448.0f;
        uint32_t mb = 0;   // max |x| by its bits: a NaN is above infinity, so it is kept
#pragma unroll
        for (int e = 0; e < 16; ++e) mb = max(mb, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
        for (int s = 1; s < TPR; s *= 2) mb = max(mb, (uint32_t)__shfl_xor((int)mb, s));
        const bool bad = mb >= 0x7F800000u;
        const float d = __uint_as_float(mb) / kMax, inv = 1.0f / d;
        if (__all(!put || (!bad && d >= kSmall))) {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = div_rn(v[e], d, inv);
        } else {   // some d is so small that the steps of div_rn leave fp32's range, or zero; a subnormal d may be far below its quotient
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float w = v[e] / d;
            v[e] = !bad && d > 0.0f ? fminf(fmaxf(w, -kMax), kMax) : 0.0f;
          }
        }
        if (put) {
          u32x2_t ca, cb;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if constexpr (CODE == CACHE_I8) {
              ca[e] = codes_i8(v + 4 * e);
              cb[e] = codes_i8(v + 8 + 4 * e);
            } else {
              ca[e] = e4m3x4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
              cb[e] = e4m3x4(v[8 + 4 * e], v[9 + 4 * e], v[10 + 4 * e], v[11 + 4 * e]);
            }
          }
          store8(to + a0, ca);
          store8(to + b0, cb);
          if (u == 0) {
            float* sc = is_k ? p.c.Ks + page * p.c.ks_p + hk * p.c.ks_h : p.c.Vs + page * p.c.vs_p + hk * p.c.vs_h;
            sc[l] = bad ? __uint_as_float(0x7FC00000u) : d;
          }
        }
      }
    }
  }
}

// Read: D / 8 threads a row, which write 16 bytes each; a workgroup takes kReadRows rows of a (sequence, head), keys and
// values, all loads of a thread under way at once.
constexpr int kReadRows = 32;
template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheReadParams p, int64_t tasks, int nch) {
  constexpr int TPR = D / 8, RPP = kThreads / TPR, N = kReadRows / RPP, E = CODE == CACHE_BF16 ? 2 : 1;
  const int r = threadIdx.x / TPR, c = threadIdx.x % TPR * 8;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int ch = (int)(task % nch), hk = (int)(task / nch % p.Hk), b = (int)(task / nch / p.Hk);
    const int64_t most = min((int64_t)p.S, (int64_t)p.pages << p.c.shift);
    const int len = (int)min((int64_t)max(p.lens[b], 0), most);
    if ((int64_t)ch * kReadRows >= len) continue;
    int page[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = ch * kReadRows + i * RPP + r;
      page[i] = j < len ? p.table[b * p.ldt + (j >> p.c.shift)] : -1;
    }
    u32x4_t w[N][2];
    float s[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if ((uint32_t)page[i] >= (uint32_t)p.c.n_pages) continue;
      const int64_t l = (ch * kReadRows + i * RPP + r) & ((1 << p.c.shift) - 1), pg = page[i];
      const char* const from[2] = {p.c.K + pg * p.c.k_p + hk * p.c.k_h + l * p.c.k_l + c * E,
                                   p.c.V + pg * p.c.v_p + hk * p.c.v_h + l * p.c.v_l + c * E};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if constexpr (CODE == CACHE_BF16) {
          w[i][x] = gload16(from[x]);
        } else {
          const u32x2_t q = *reinterpret_cast<const u32x2_t*>(from[x]);
          w[i][x][0] = q[0];
          w[i][x][1] = q[1];
        }
      }
      if constexpr (CODE != CACHE_BF16) {
        s[i][0] = p.c.Ks[pg * p.c.ks_p + hk * p.c.ks_h + l];
        s[i][1] = p.c.Vs[pg * p.c.vs_p + hk * p.c.vs_h + l];
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if ((uint32_t)page[i] >= (uint32_t)p.c.n_pages) continue;
      const int64_t j = ch * kReadRows + i * RPP + r;
      bf16_t* const to[2] = {p.K + b * p.k_b + hk * p.k_h + j * p.k_l + c, p.V + b * p.v_b + hk * p.v_h + j * p.v_l + c};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if constexpr (CODE == CACHE_BF16) {
          store16(to[x], w[i][x]);
        } else {
          float v[8];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t q = w[i][x][e];
            if constexpr (CODE == CACHE_I8) {
#pragma unroll
              for (int y = 0; y < 4; ++y) v[4 * e + y] = (float)(int8_t)(q >> (8 * y));
            } else {
              const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
              v[4 * e] = lo[0];
              v[4 * e + 1] = lo[1];
              v[4 * e + 2] = hi[0];
              v[4 * e + 3] = hi[1];
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= s[i][x];
          store16(to[x], pack8(v));
        }
      }
    }
  }
}

template <int D, int CODE, int NP>
hipError_t write_np(const CacheWriteParams& p, hipStream_t st) {
  constexpr int RPW = NP * 64 / (D / 16);   // rows of a wave
  const int chunks = (p.H + 2 * p.Hk + RPW - 1) / RPW;
  const int64_t tasks = (int64_t)p.T * chunks, blocks = (tasks + kThreads / 64 - 1) / (kThreads / 64);
  hipLaunchKernelGGL((cache_write_kernel<D, CODE, NP>), dim3((unsigned)std::min(blocks, kMostBlocks)), dim3(kThreads), 0, st, p, tasks, chunks);
  return hipGetLastError();
}
template <int D, int CODE>
hipError_t write_d(const CacheWriteParams& p, hipStream_t st) {
  // Three passes a wave where those of one fill the chip anyway (2048 tokens of 48 rows, E4M3 11.2 -> 9.8 us; 64 tokens 3.8 -> 5.0).
  const int64_t passes = (int64_t)p.T * (p.H + 2 * p.Hk) * (D / 16) / 64;   // waves, of one pass each
  return passes > 4096 ? write_np<D, CODE, 3>(p, st) : write_np<D, CODE, 1>(p, st);
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
