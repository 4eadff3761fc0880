// Matrix product with 4-bit weights and a scale per group of k:
//     C[m, n] = act(sum_g s[g, n] sum_{k in g} A[m, k] w[n, k] + bias[n]).
//
// Weights come as tiles of 32 channels by 64 k in the order of the operand of the 32 x 32 x 16 MFMA: a wave
// loads a tile's 1024 bytes with one contiguous 16-byte load a lane straight into registers, and makes exact
// bf16 values of its codes there.  Tokens go through LDS by direct loads.  A group's products are summed by the
// MFMAs from zero, then added to the tile's sums with the group's scale, one fused step in fp32: a lane holds one
// channel of a block, so the scale is one value a lane.
#include <algorithm>
#include <cstdio>
#include <type_traits>

#include "cf_gemm_big.h"
#include "cf_serving.h"
#include "cf_attn.h"

namespace cf {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;

template <int ACT>
__device__ __forceinline__ float act_w4(float x) {
  if constexpr (ACT == ACT_GELU) return gelu_erf(x);
  if constexpr (ACT == ACT_GELU_TANH) return 0.5f * x * (1.0f + tanh_exp(0.79788456080286536f * (x + 0.044715f * x * x * x)));
  if constexpr (ACT == ACT_RELU) return x < 0.0f ? 0.0f : x;
  return x;
}
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == ACT_GELU) f(std::integral_constant<int, ACT_GELU>{});
  else if (act == ACT_GELU_TANH) f(std::integral_constant<int, ACT_GELU_TANH>{});
  else if (act == ACT_RELU) f(std::integral_constant<int, ACT_RELU>{});
  else f(std::integral_constant<int, ACT_NONE>{});
}

// Eight codes of neighbouring k -> bf16.  Integers come out as w / 16 (the scale takes the 16).
template <bool E2M1>
__device__ __forceinline__ u32x4_t w4_values(uint32_t w) {
  u32x4_t v = {};
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (E2M1) {
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = pack_bf16x2(__builtin_amdgcn_cvt_off_f32_i4(w >> (8 * i)), __builtin_amdgcn_cvt_off_f32_i4(w >> (8 * i + 4)));
  }
#endif
  return v;
}

struct W4Scales {   // s[k / group, n]
  const void* s;
  int64_t lds;
  uint32_t mul;     // ceil(2^32 / (group / 32)); 0: group 32
  int f32;
  __device__ __forceinline__ float at(int k32, int n) const {   // of k = 32 k32 (below 2^15; group / 32 too)
    const int64_t i = (int64_t)(mul ? __umulhi((uint32_t)k32, mul) : (uint32_t)k32) * lds + n;
    return f32 ? reinterpret_cast<const float*>(s)[i] : bf16_to_f32(reinterpret_cast<const bf16_t*>(s)[i]);
  }
};

// A group of WM x WN waves (32 BM tokens x 32 BN channels each) shares a ring of NS stages of 64 k of the
// tokens; KW groups take the stages in turn and their sums meet in LDS.  AR: token rows that are staged (few tokens: less than
// the 32 of an MFMA, whose other rows repeat them and are not stored).
template <int BM_, int BN_, int WM_, int WN_, int KW_, int NS_, int AR_>
struct W4Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KW = KW_, NS = NS_, AR = AR_;
  static constexpr int GW = WM * WN, NW = GW * KW, NT = 64 * NW;
  static constexpr int TM = AR, TN = 32 * BN * WN, STAGE = AR * 128, PITCH = TN * 4 + 16;
  static constexpr int AHEAD = GW == 1 ? NS : NS - 1;   // steps loaded ahead
  static constexpr int RING = NS * STAGE, OUT = KW * TM * PITCH;
  static constexpr int LDS = KW * RING > OUT ? KW * RING : OUT;
  static constexpr int LPW = AR / 8 / GW;               // wave-wide loads of a stage per wave
  static_assert(LPW * 8 * GW == AR && LDS <= 160 * 1024, "stage split, LDS budget");
  static_assert(AR == 32 * BM * WM || (AR < 32 && BM == 1 && GW == 1), "rows");
};

template <class S, bool E2M1, int FOLD>
__global__ __launch_bounds__(S::NT) void gemm_w4_kernel(GemmW4Params p, W4Scales scales) {
  __shared__ __attribute__((aligned(16))) char smem[S::LDS];
  constexpr int H = 64 / FOLD;   // folds of a step
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int grp = wave / S::GW, gw = wave % S::GW, wm = gw / S::WN, wn = gw % S::WN;
  int rb, c;
  big_tile_order((p.M + S::TM - 1) / S::TM, (p.N + S::TN - 1) / S::TN, rb, c);
  const int m0 = rb * S::TM, n0 = c * S::TN;
  const int KB = (p.K + 63) / 64, steps = grp < KB ? (KB - grp - 1) / S::KW + 1 : 0;
  char* const ring = smem + grp * S::RING;

  // Load i of a wave fills rows 8 (i GW + gw) .. + 7 of a stage; rows past M are clamped.  The 16-byte chunk
  // ch of row r sits at position ch ^ ((r >> 1) & 7).
  const char* src[S::LPW];
#pragma unroll
  for (int i = 0; i < S::LPW; ++i) {
    const int row = 8 * (i * S::GW + gw) + (lane >> 3), ch = (lane & 7) ^ ((row >> 1) & 7);
    src[i] = reinterpret_cast<const char*>(p.A + (int64_t)min(m0 + row, p.M - 1) * p.lda) + ch * 16;
  }
  const uint8_t* wsrc[S::BN];
  int col[S::BN];
#pragma unroll
  for (int b = 0; b < S::BN; ++b) {
    const int nb = min(n0 / 32 + wn * S::BN + b, (p.N + 31) / 32 - 1);   // blocks past N repeat the last
    wsrc[b] = p.W + (int64_t)nb * KB * 1024 + lane * 16;
    col[b] = min(nb * 32 + lr, p.N - 1);
  }
  const bool cut = p.K & 32;   // the last step has 32 k (groups of 64 t divide K: FOLD = 32 only)
  u32x4_t wr[S::AHEAD][S::BN];
  float sr[S::AHEAD][S::BN][H];
  auto load = [&](int i, int u) {   // the group's step i, registers u
    const int kb = grp + i * S::KW;
#pragma unroll
    for (int l = 0; l < S::LPW; ++l) {
      const char* from = src[l] + (int64_t)kb * 128;
      if (FOLD == 32 && cut && kb == KB - 1) {   // chunks behind K: any of the row's, not used
        const int ch = ((lane & 7) ^ ((8 * (l * S::GW + gw) + (lane >> 3)) >> 1 & 7));
        if (ch >= 4) from -= 64;
      }
      dma16(from, ring + i % S::NS * S::STAGE + (l * S::GW + gw) * 1024);
    }
    asm volatile("" ::: "memory");   // the weights' loads stay behind: whoever waits for them has waited for these
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < S::BN; ++b) {
      wr[u][b] = gload16(wsrc[b] + (int64_t)kb * 1024);
#pragma unroll
      for (int h = 0; h < H; ++h) sr[u][b][h] = scales.at(min(2 * kb + h, p.K / 32 - 1), col[b]);
    }
  };
  const uint32_t s0 =
      (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem) + grp * S::RING;
  uint32_t xa[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const int row = wm * 32 * S::BM + (S::AR < 32 ? lr % S::AR : lr);
    xa[ks] = s0 + row * 128 + (((2 * ks + lg) ^ ((row >> 1) & 7)) << 4);
  }
  f32x16_t acc[S::BM][S::BN] = {};
  const int all = (KB + S::KW - 1) / S::KW;   // every group passes every barrier
#pragma unroll
  for (int u = 0; u < S::AHEAD; ++u)
    if (u < steps) load(u, u);
  for (int i0 = 0; i0 < all; i0 += S::AHEAD) {
#pragma unroll
    for (int u = 0; u < S::AHEAD; ++u) {
      const int i = i0 + u;
      if (i >= all) break;
      // The weights' registers are waited for, and with them the step's earlier loads into LDS.
#pragma unroll
      for (int b = 0; b < S::BN; ++b) asm volatile("" : "+v"(wr[u][b])::"memory");
      if constexpr (S::GW > 1) lds_barrier();   // every wave's loads of step i are in, and step i - 1 has been read
      if (i >= steps) continue;
      u32x4_t xf[S::BM][4];
      const uint32_t at = i % S::NS * S::STAGE;
      const uint32_t x[4] = {xa[0] + at, xa[1] + at, xa[2] + at, xa[3] + at};
      if constexpr (S::BM == 2) read_x_half<0>(xf, x);
      else read_w_half_nk<0>(xf[0], x);
      u32x4_t w[S::BN];
      float sc[S::BN][H];
#pragma unroll
      for (int b = 0; b < S::BN; ++b) {
        w[b] = wr[u][b];
#pragma unroll
        for (int h = 0; h < H; ++h) sc[b][h] = E2M1 ? sr[u][b][h] : 16.0f * sr[u][b][h];
      }
      const bool half = cut && grp + i * S::KW == KB - 1;
      if (i + S::AHEAD < steps) load(i + S::AHEAD, u);
#pragma unroll
      for (int b = 0; b < S::BN; ++b) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          if (H == 2 && h == 1 && half) break;
          f32x16_t part[S::BM] = {};
#pragma unroll
          for (int ks = h * 4 / H; ks < (h + 1) * 4 / H; ++ks) {
            const u32x4_t v = w4_values<E2M1>(w[b][ks]);
#pragma unroll
            for (int a = 0; a < S::BM; ++a) Mma<bf16_t>::run(part[a], xf[a][ks], v);
          }
#pragma unroll
          for (int a = 0; a < S::BM; ++a)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = fmaf(part[a][e], sc[b][h], acc[a][b][e]);
        }
      }
    }
  }
  __syncthreads();
  // Sums to LDS, KW planes of TM rows; then a thread adds the planes of 8 columns of a row at a time.
  float* const out = reinterpret_cast<float*>(smem + grp * S::TM * S::PITCH);
#pragma unroll
  for (int a = 0; a < S::BM; ++a)
#pragma unroll
    for (int b = 0; b < S::BN; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = (wm * S::BM + a) * 32 + acc_row(e, lane);
        if (S::AR >= 32 || row < S::AR) out[row * (S::PITCH / 4) + (wn * S::BN + b) * 32 + lr] = acc[a][b][e];
      }
  __syncthreads();
  constexpr int CPR = S::TN / 8;
  with_act(p.act, [&](auto act_t) {
    constexpr int ACT = decltype(act_t)::value;
    for (int x = tid; x < min(S::TM, p.M - m0) * CPR; x += S::NT) {
      const int r = x / CPR, c8 = x % CPR * 8, left = p.N - n0 - c8;
      if (left <= 0) continue;
      float y[8] = {};
#pragma unroll
      for (int k = 0; k < S::KW; ++k) {
        const f32x4_t* from = reinterpret_cast<const f32x4_t*>(smem + (k * S::TM + r) * S::PITCH + c8 * 4);
        const f32x4_t lo = from[0], hi = from[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] += lo[e];
          y[4 + e] += hi[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (p.bias) y[e] += p.bias[min(n0 + c8 + e, p.N - 1)];
        y[e] = act_w4<ACT>(y[e]);
      }
      const int64_t at = (int64_t)(m0 + r) * p.ldc + n0 + c8;
      if (p.c_f32) {
        float* to = reinterpret_cast<float*>(p.C) + at;
        if (left >= 8) {
          *reinterpret_cast<f32x4_t*>(to) = f32x4_t{y[0], y[1], y[2], y[3]};
          *reinterpret_cast<f32x4_t*>(to + 4) = f32x4_t{y[4], y[5], y[6], y[7]};
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (e < left) to[e] = y[e];
        }
      } else {
        bf16_t* to = reinterpret_cast<bf16_t*>(p.C) + at;
        if (left >= 8) {
          *reinterpret_cast<u32x4_t*>(to) = u32x4_t{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                                                    pack_bf16x2(y[6], y[7])};
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (e < left) to[e] = (bf16_t)pack_bf16x2(y[e], 0.0f);
        }
      }
    }
  });
}

template <class S, bool E2M1>
hipError_t launch_code(const GemmW4Params& p, hipStream_t st) {
  const int64_t wgs = (int64_t)((p.M + S::TM - 1) / S::TM) * ((p.N + S::TN - 1) / S::TN);
  const uint32_t g32 = p.group / 32;
  const W4Scales sc{p.s, p.lds, g32 == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + g32 - 1) / g32), p.s_f32};
  if (p.group % 64 == 0) hipLaunchKernelGGL((gemm_w4_kernel<S, E2M1, 64>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p, sc);
  else hipLaunchKernelGGL((gemm_w4_kernel<S, E2M1, 32>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p, sc);
  return hipGetLastError();
}
template <class S>
hipError_t launch_tile(const GemmW4Params& p, hipStream_t st) {
  return p.e2m1 ? launch_code<S, true>(p, st) : launch_code<S, false>(p, st);
}

struct Form {
  int tm, tn, threads, per;
  double step, start;
  hipError_t (*launch)(const GemmW4Params&, hipStream_t);
};
constexpr int kCUs = 256;
template <class S>
constexpr Form tile_form(int per, double step, double start) {
  return {S::TM, S::TN, S::NT, per, step, start, launch_tile<S>};
}
const Form kForms[] = {
    tile_form<W4Tile<1, 1, 1, 1, 8, 4, 8>>(kCUs, 0.02, 2.0),
    tile_form<W4Tile<1, 1, 1, 1, 8, 4, 32>>(kCUs, 0.04, 2.2),
    tile_form<W4Tile<2, 2, 1, 1, 4, 3, 64>>(kCUs, 0.09, 2.5),
    tile_form<W4Tile<2, 2, 2, 2, 2, 3, 128>>(kCUs, 0.14, 3),
    tile_form<W4Tile<2, 2, 4, 2, 1, 3, 256>>(kCUs, 0.45, 3),
};

const Form& choose_form(const GemmW4Params& p) {
  const Form* best = nullptr;
  double least = 0;
  const double kt = (double)((p.K + 63) / 64);
  for (const Form& f : kForms) {
    const int64_t wgs = (int64_t)((p.M + f.tm - 1) / f.tm) * ((p.N + f.tn - 1) / f.tn), rounds = (wgs + f.per - 1) / f.per;
    if (wgs * f.threads > UINT32_MAX) continue;   // a grid has less than 2^32 threads; 128 x 128 tiles of M N <= 2^37 fit
    const double t = (double)rounds * (f.step * kt + f.start);
    if (!best || t < least) {
      best = &f;
      least = t;
    }
  }
  return *best;
}

// ---------------------------------------------------------------------------
// Laying out.
// ---------------------------------------------------------------------------
// Word j of lane 32 h + r of tile (nb, kb): k = 64 kb + 16 j + 8 h .. + 7 of channel 32 nb + r.
__device__ __forceinline__ uint32_t* tile_word(uint8_t* tiles, int KB, int n, int k) {
  return reinterpret_cast<uint32_t*>(tiles + ((int64_t)(n / 32) * KB + k / 64) * 1024 + ((k / 8 % 2) * 32 + n % 32) * 16) + k / 16 % 4;
}

__global__ __launch_bounds__(256) void w4_pack_kernel(int N, int K, const uint8_t* codes, int64_t ldc, uint8_t* tiles) {
  const int KB = (K + 63) / 64, words = KB * 8;   // of a channel
  const int64_t all = (int64_t)((N + 31) / 32) * 32 * words;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < all; x += (int64_t)gridDim.x * 256) {
    const int n = (int)(x / words), k = (int)(x % words) * 8;
    uint32_t w = 0;
    if (n < N && k < K) {
      const uint8_t* from = codes + n * ldc + k / 2;
#pragma unroll
      for (int b = 0; b < 4; ++b) w |= (uint32_t)from[b] << (8 * b);
    }
    *tile_word(tiles, KB, n, k) = w;
  }
}

// A thread takes a group of a channel; the one behind the last, what the tiles have behind K.
__global__ __launch_bounds__(256) void w4_quant_kernel(W4QuantParams p) {
  const int KB = (p.K + 63) / 64, ng = p.K / p.group, per = ng + (p.K % 64 != 0);
  const int64_t all = (int64_t)((p.N + 31) / 32) * 32 * per;
  const float most = p.e2m1 ? 6.0f : 7.0f;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < all; x += (int64_t)gridDim.x * 256) {
    const int n = (int)(x / per), g = (int)(x % per);
    const int k0 = g * p.group, k1 = g < ng ? k0 + p.group : KB * 64;
    const int64_t row = n * p.ldw;
    auto get = [&](int k) {
      return p.f32 ? reinterpret_cast<const float*>(p.W)[row + k] : bf16_to_f32(reinterpret_cast<const bf16_t*>(p.W)[row + k]);
    };
    float s = 0.0f;
    bool bad = false;
    if (n < p.N && g < ng) {
      uint32_t mb = 0;
      for (int k = k0; k < k1; ++k) mb = max(mb, __float_as_uint(get(k)) & 0x7FFFFFFFu);
      bad = mb >= 0x7F800000u;
      s = __uint_as_float(mb) / most;
      if (!p.s_f32) s = bf16_to_f32(pack_bf16x2(s, 0.0f) & 0xFFFFu);
      const float put = bad ? __uint_as_float(0x7FC00000u) : s;
      const int64_t at = g * p.lds + n;
      if (p.s_f32) reinterpret_cast<float*>(p.s)[at] = put;
      else reinterpret_cast<bf16_t*>(p.s)[at] = (bf16_t)(__float_as_uint(put) >> 16);
    }
    for (int k = k0; k < k1; k += 8) {
      uint32_t w = 0;
      if (s > 0.0f && !bad)
        for (int e = 0; e < 8; ++e) {
          const float z = get(k + e) / s;
          uint32_t code;
          if (p.e2m1) {
            const float a = fabsf(z);
            code = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
            if (code && z < 0.0f) code |= 8;
          } else {
            code = (uint32_t)(int)fminf(fmaxf(rintf(z), -7.0f), 7.0f) & 15u;
          }
          w |= code << (4 * e);
        }
      *tile_word(p.tiles, KB, n, k) = w;
    }
  }
}

}  // namespace

hipError_t launch_gemm_w4(const GemmW4Params& p, hipStream_t st) { return choose_form(p).launch(p, st); }

void gemm_w4_form(const GemmW4Params& p, char* text, size_t bytes) {
  const Form& f = choose_form(p);
  snprintf(text, bytes, "%d x %d tiles of %d threads, scales every %d", f.tm, f.tn, f.threads, p.group % 64 == 0 ? 64 : 32);
}

hipError_t launch_w4_pack(int N, int K, const uint8_t* codes, int64_t ldc, uint8_t* tiles, hipStream_t st) {
  const int64_t threads = (int64_t)(N + 31) / 32 * 32 * ((K + 63) / 64) * 8;
  hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)std::min<int64_t>((threads + 255) / 256, 1 << 16)), dim3(256), 0, st, N, K, codes, ldc, tiles);
  return hipGetLastError();
}

hipError_t launch_w4_quant(const W4QuantParams& p, hipStream_t st) {
  const int64_t threads = (int64_t)(p.N + 31) / 32 * 32 * (p.K / p.group + 1);
  hipLaunchKernelGGL(w4_quant_kernel, dim3((unsigned)std::min<int64_t>((threads + 255) / 256, 1 << 16)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace cf
