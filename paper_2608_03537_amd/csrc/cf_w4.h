// Matrix product with 4-bit weights and a scale per group of k:
//     C[m, n] = act(sum_g s[g, n] sum_{k in g} A[m, k] w[n, k] + bias[n]).
//
// Weights come as tiles of 32 channels by 64 k in the order of the operand of the 32 x 32 x 16 MFMA: a wave
// loads a tile's 1024 bytes with one contiguous 16-byte load a lane straight into registers, and makes exact
// bf16 values of its codes there.  Tokens go through LDS by direct loads.  A group's products are summed by the
// MFMAs from zero, then added to the tile's sums with the group's scale, one fused step in fp32: a lane holds one
// channel of a block, so the scale is one value a lane.
//
// Bound.  One token: the launch, and 128 workgroups for 256 CUs with eight steps a wave (1 x 4096 x 4096 int4, 8.7 MB: 6.7 us,
// in a loop of calls 7.4).  Tens: the conversion and the folds of the one wave that a SIMD has (48 x 12288 x 4096 E2M1, 28 MB:
// 12.2 us, 2.3 TB/s).  Thousands: the issue of MFMAs and conversions, and power (4096 x 4096 x 4096 int4: 142 to 147 us, 0.97 to
// 0.93 PFLOP/s; more than eight launches in a row lower the clock to 1.7 GHz and less, and take 171 to 192 us each).
#pragma once

#include <algorithm>
#include <type_traits>

#include "cf_attn.h"
#include "cf_gemm_big.h"
#include "cf_serving.h"

namespace cf {

namespace {

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

// Eight codes of neighbouring k -> bf16.  Integers come out as 16 w (the scale takes the 1 / 16): a code in the high
// half of a byte is a signed byte of 16 times its value, which one conversion takes, and the value's fp32 bits end in
// zeros, so its upper half is its bf16: 15 operations for eight codes, 4 for E2M1.
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
    uint32_t lo = (w << 4) & 0xF0F0F0F0u, hi = w & 0xF0F0F0F0u;
    asm("" : "+v"(lo), "+v"(hi));   // or the conversion takes the masks apart again, byte by byte
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(hi >> (8 * i))), __float_as_uint((float)(int8_t)(lo >> (8 * i))),
                                   0x07060302u);
  }
#endif
  return v;
}

// Buffers: a load from one of no bytes reads nothing and returns 0, so the loops ask for steps behind the last one
// without a branch, and the compiler knows how many loads are under way.
#if defined(__HIP_DEVICE_COMPILE__)
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* p, bool any) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, any ? 0x7FFFFFFF : 0, 0x00020000);
}
#endif

// k32 / (group / 32) for k32, group / 32 <= 2^15, by the product with ceil(2^32 / (group / 32)); 0: group 32.
__device__ __forceinline__ uint32_t group_of(uint32_t k32, uint32_t mul) { return mul ? __umulhi(k32, mul) : k32; }

// A group of WM x WN waves (32 BM tokens x 32 BN channels each) shares a ring of NS stages of 64 k of the
// tokens; KW groups take the stages in turn and their sums meet in LDS.  AR: token rows that are staged (few tokens: less than
// the 32 of an MFMA, whose other rows repeat them and are not stored).
template <int BM_, int BN_, int WM_, int WN_, int KW_, int NS_, int AR_>
struct W4Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KW = KW_, NS = NS_, AR = AR_;
  static constexpr int GW = WM * WN, NW = GW * KW, NT = 64 * NW;
  static constexpr int TM = AR, TN = 32 * BN * WN, STAGE = AR * 128, PITCH = TN * 4 + 16;
  static constexpr int AHEAD = NS - 1;                  // steps loaded ahead
  static constexpr int RING = NS * STAGE, OUT = KW * TM * PITCH;
  static constexpr int LDS = KW * RING > OUT ? KW * RING : OUT;
  static constexpr int LPW = AR / 8 / GW;               // wave-wide loads of a stage per wave
  static_assert(LPW * 8 * GW == AR && LDS <= 160 * 1024, "stage split, LDS budget");
  static_assert(AR == 32 * BM * WM || (AR < 32 && BM == 1 && GW == 1), "rows");
};

template <class S, bool E2M1, int FOLD, class T>
__global__ __launch_bounds__(S::NT) void gemm_w4_kernel(GemmW4Params p, uint32_t mul) {
  __shared__ __attribute__((aligned(16))) char smem[S::LDS];
  constexpr int H = FOLD == 32 ? 2 : 1;         // scales of a step
  constexpr bool PAIRS = FOLD == 128;           // two steps a scale
  constexpr int RE = S::AR < 32 ? S::AR / 2 : 16;   // elements of a block that are rows of their own
  static_assert(!PAIRS || S::NS % 2 == 0, "a pair's steps are in one turn of the ring");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int grp = wave / S::GW, gw = wave % S::GW, wm = gw / S::WN, wn = gw % S::WN;
  int rb, c;
  big_tile_order((p.M + S::TM - 1) / S::TM, (p.N + S::TN - 1) / S::TN, rb, c);
  const int m0 = rb * S::TM, n0 = c * S::TN;
  // Steps of 64 k, or pairs of them, go to the groups of waves in turn.
  constexpr int RUN = PAIRS ? 2 : 1;
  const int KB = (p.K + 63) / 64, steps = grp < KB / RUN ? ((KB / RUN - grp - 1) / S::KW + 1) * RUN : 0;
  [[maybe_unused]] char* const ring = smem + grp * S::RING;

  // Load i of a wave fills rows 8 (i GW + gw) .. + 7 of a stage; rows past M are clamped.  The 16-byte chunk
  // ch of row r sits at position ch ^ ((r >> 1) & 7).
  [[maybe_unused]] const bf16_t* const arows = p.A + (int64_t)m0 * p.lda;
  uint32_t aoff[S::LPW];
  const bool cut = FOLD == 32 && (p.K & 32);   // the last step has 32 k (groups of 64 t divide K)
  uint32_t behind[S::LPW];                     // of the cut step: back to a chunk that the row has
#pragma unroll
  for (int i = 0; i < S::LPW; ++i) {
    const int row = 8 * (i * S::GW + gw) + (lane >> 3), ch = (lane & 7) ^ ((row >> 1) & 7);
    aoff[i] = (uint32_t)min(row, p.M - 1 - m0) * (uint32_t)(p.lda * 2) + ch * 16;
    behind[i] = ch >= 4 ? 64 : 0;
  }
  const uint8_t* wtile[S::BN];
  uint32_t col[S::BN];
#pragma unroll
  for (int b = 0; b < S::BN; ++b) {
    const int nb = min(n0 / 32 + wn * S::BN + b, (p.N + 31) / 32 - 1);   // blocks past N repeat the last
    wtile[b] = p.W + (int64_t)nb * KB * 1024;
    col[b] = (uint32_t)min(nb * 32 + lr, p.N - 1);
  }
  // Tiles begin at different k: together they would read columns of rows that lie a power of two apart, which few
  // channels of the memory hold.
  const int turn = steps > 0 ? (rb * 5 + c) * 3 % steps & (PAIRS ? ~1 : ~0) : 0;
  auto block = [&](int i) {
    const int t = i + turn < steps ? i + turn : i + turn - steps;
    return PAIRS ? 2 * (grp + (t >> 1) * S::KW) + (t & 1) : grp + t * S::KW;
  };
  u32x4_t wr[S::NS][S::BN];
  T sr[S::NS][S::BN][H];
  auto load = [&](int i, int u) {   // the group's step i, stage and registers u; nothing behind the last
#if defined(__HIP_DEVICE_COMPILE__)
    const int kb = block(i);
    const Buffer abuf = buffer_of(arows, i < steps);
#pragma unroll
    for (int l = 0; l < S::LPW; ++l)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(abuf, (__attribute__((address_space(3))) void*)(ring + u * S::STAGE + (l * S::GW + gw) * 1024),
                                               16, cut && kb == KB - 1 ? aoff[l] - behind[l] : aoff[l], kb * 128, 0, 0);
    asm volatile("" ::: "memory");   // the weights' loads stay behind: whoever waits for them has waited for these
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < S::BN; ++b) {
      wr[u][b] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer_of(wtile[b], i < steps), lane * 16, kb * 1024, 0));
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const T* row = reinterpret_cast<const T*>(p.s) + (int64_t)group_of(min(2 * kb + h, p.K / 32 - 1), mul) * p.lds;
        sr[u][b][h] = row[col[b]];
      }
    }
#endif
  };
  // The columns of the output that a thread writes are always the same; their biases are on their way meanwhile.
  constexpr int CPR = S::TN / 8;
  static_assert(S::NT % CPR == 0, "a thread keeps its columns");
  const int c8 = tid % CPR * 8, left = p.N - n0 - c8;
  float bias[8] = {};
  if (p.bias)
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = p.bias[min(n0 + c8 + e, p.N - 1)];
  const uint32_t s0 =
      (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem) + grp * S::RING;
  uint32_t xa[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const int row = wm * 32 * S::BM + (S::AR < 32 ? lr % S::AR : lr);
    xa[ks] = s0 + row * 128 + (((2 * ks + lg) ^ ((row >> 1) & 7)) << 4);
  }
  f32x16_t acc[S::BM][S::BN] = {}, part[S::BM][S::BN];
  if constexpr (FOLD != 32 && S::BN > 1 && (S::KW == 1 || S::GW == 1)) {
    // Blocks of two and more: nothing waits for the rest of its own step.  While the MFMAs of 16 k run, the next 16 k are
    // read from LDS and their weights converted; a stage is loaded again as soon as its last part has been read; a
    // group's sums are added to the tile's before the first MFMA of the next group writes them.  (Against the loop below, us:
    // 1024 x 4096 x 4096 int4 51.5 -> 43, 4096 x 4096 x 4096 150 -> 147, 0.94 PFLOP/s, where int4's conversion, 15 vector
    // operations for 8 codes, and the MFMAs share the issue and the power of a CU; E2M1 136 -> 124; 128 and fewer tokens by
    // 4 to 8 %.  Tiles of single blocks are 2 to 4 % faster below.  Four groups of two waves, with barriers of their own,
    // take 0.8 us more to start here and 0.03 less for every 64 k, for all calls together the same.)
    constexpr int PER = 4 / S::BM;            // pairs of weights converted beside an MFMA
    u32x4_t xf[2][S::BM], v[2][S::BN];
    float sc[S::BN] = {};
#pragma unroll
    for (int u = 0; u < S::NS; ++u) load(u, u);
#pragma unroll
    for (int b = 0; b < S::BN; ++b) asm volatile("" : "+v"(wr[0][b])::"memory");
    if constexpr (S::GW > 1) lds_barrier();
    static_for<0, S::BM>([&](auto a_t) {
      constexpr int a = decltype(a_t)::value;
      xf[0][a] = ds_read_b128_at<a * 4096>(xa[0]);
    });
    auto word_of = [](uint32_t w) {
      asm("" : "+v"(w));   // opaque: the compiler would take its bytes apart long before their use
      return w;
    };
#pragma unroll
    for (int b = 0; b < S::BN; ++b) v[0][b] = w4_values<E2M1>(word_of(wr[0][b][0]));
    auto fold = [&](int a, int b) {
#pragma unroll
      for (int e = 0; e < RE; ++e) acc[a][b][e] = fmaf(part[a][b][e], sc[b], acc[a][b][e]);
    };
#pragma unroll
    for (int a = 0; a < S::BM; ++a)
#pragma unroll
      for (int b = 0; b < S::BN; ++b) part[a][b] = f32x16_t{};
    for (int i0 = 0; i0 < steps; i0 += S::NS) {
      static_for<0, S::NS / RUN>([&](auto run_t) {   // (no branch within a pair)
        if (i0 + decltype(run_t)::value * RUN >= steps) return;
        static_for<0, 4 * RUN>([&](auto part_t) {
          constexpr int u = decltype(run_t)::value * RUN + decltype(part_t)::value / 4, ks = decltype(part_t)::value % 4;
          constexpr int next = (u + 1) % S::NS, cur = ks & 1;
          constexpr bool begins = ks == 0 && !(PAIRS && u % 2), ends = ks == 3 && !(PAIRS && u % 2 == 0);   // a group
          if constexpr (ks < 3)
            static_for<0, S::BM>([&](auto a_t) {
              constexpr int a = decltype(a_t)::value;
              xf[!cur][a] = ds_read_b128_at<a * 4096>(xa[ks + 1] + u * S::STAGE);
            });
          static_for<0, S::BM>([&](auto a_t) {
            constexpr int a = decltype(a_t)::value;
            lgkm_wait<(ks < 3 ? S::BM : 0) + S::BM - 1 - a>(xf[cur][a]);
          });
          uint32_t word = 0;
          static_for<0, S::BM * S::BN>([&](auto c_t) {
            constexpr int c = decltype(c_t)::value, b = c / S::BM, a = c % S::BM;
            if constexpr (begins) {
              fold(a, b);
              part[a][b] = f32x16_t{};
            }
            Mma<bf16_t>::run(part[a][b], xf[cur][a], v[cur][b]);
            if constexpr (ks == 3 && c == 0) {
              if constexpr (ends)
#pragma unroll
                for (int x = 0; x < S::BN; ++x) {
                  if constexpr (sizeof(T) == 4) sc[x] = sr[u][x][0];
                  else sc[x] = bf16_to_f32(sr[u][x][0]);
                  if (!E2M1) sc[x] *= 0.0625f;
                }
              // The next step's weights are waited for, and with them the wave's earlier loads into LDS.
#pragma unroll
              for (int x = 0; x < S::BN; ++x) asm volatile("" : "+v"(wr[next][x])::"memory");
              if constexpr (S::GW > 1) lds_barrier();   // every wave's are in, and this step's stage has been read
              static_for<0, S::BM>([&](auto x_t) {
                constexpr int x = decltype(x_t)::value;
                xf[!cur][x] = ds_read_b128_at<x * 4096>(xa[0] + next * S::STAGE);
              });
              __builtin_amdgcn_sched_barrier(0);
              load(i0 + u + S::NS, u);
              __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (a == 0) word = word_of(ks < 3 ? wr[u][b][(ks + 1) % 4] : wr[next][b][0]);
#pragma unroll
            for (int x = a * PER; x < a * PER + PER; ++x) v[!cur][b][x] = w4_values<E2M1>(word)[x];
          });
        });
      });
    }
    static_for<0, S::BM>([&](auto a_t) { lgkm_wait<0>(xf[0][decltype(a_t)::value]); });   // (of a step that there is not)
#pragma unroll
    for (int a = 0; a < S::BM; ++a)
#pragma unroll
      for (int b = 0; b < S::BN; ++b) fold(a, b);
  } else {
    const int all = (KB / RUN + S::KW - 1) / S::KW * RUN;   // every group passes every barrier
#pragma unroll
    for (int u = 0; u < S::AHEAD; ++u) load(u, u);
    for (int i0 = 0; i0 < all; i0 += S::NS) {
#pragma unroll
      for (int u = 0; u < S::NS; ++u) {
        const int i = i0 + u;
        // The weights' registers are waited for, and with them the step's earlier loads into LDS.
#pragma unroll
        for (int b = 0; b < S::BN; ++b) asm volatile("" : "+v"(wr[u][b])::"memory");
        if constexpr (S::GW > 1) lds_barrier();   // every wave's loads of step i are in, and step i - 1 has been read
        // Fragments of k step ks of every block, in the order in which they are used; each is waited for there.
        u32x4_t xf[4][S::BM];
        static_for<0, 4 * S::BM>([&](auto r_t) {
          constexpr int r = decltype(r_t)::value;
          xf[r / S::BM][r % S::BM] = ds_read_b128_at<r % S::BM * 4096>(xa[r / S::BM] + u * S::STAGE);
        });
        u32x4_t w[S::BN];
        float sc[S::BN][H];
#pragma unroll
        for (int b = 0; b < S::BN; ++b) {
          w[b] = wr[u][b];
#pragma unroll
          for (int h = 0; h < H; ++h) {
            if constexpr (sizeof(T) == 4) sc[b][h] = sr[u][b][h];
            else sc[b][h] = bf16_to_f32(sr[u][b][h]);
            if (!E2M1) sc[b][h] *= 0.0625f;
          }
        }
        const bool half = cut && block(i) == KB - 1, in = i < steps;
        static_for<0, 4>([&](auto ks_t) {
          constexpr int ks = decltype(ks_t)::value, h = H == 2 ? ks / 2 : 0;
          constexpr bool first = H == 2 ? ks % 2 == 0 : ks == 0, fold = H == 2 ? ks % 2 == 1 : ks == 3;
          static_for<0, S::BM>([&](auto a_t) {
            constexpr int a = decltype(a_t)::value;
            lgkm_wait<4 * S::BM - 1 - (ks * S::BM + a)>(xf[ks][a]);
          });
          if (in && !(H == 2 && h == 1 && half)) {
#pragma unroll
            for (int b = 0; b < S::BN; ++b) {
              const u32x4_t v = w4_values<E2M1>(w[b][ks]);
#pragma unroll
              for (int a = 0; a < S::BM; ++a) {
                if (first && !(PAIRS && u % 2)) part[a][b] = f32x16_t{};
                Mma<bf16_t>::run(part[a][b], xf[ks][a], v);
              }
            }
            if constexpr (fold) {
              if (!PAIRS || u % 2)
#pragma unroll
                for (int b = 0; b < S::BN; ++b)
#pragma unroll
                  for (int a = 0; a < S::BM; ++a)
#pragma unroll
                    for (int e = 0; e < RE; ++e) acc[a][b][e] = fmaf(part[a][b][e], sc[b][h], acc[a][b][e]);
            }
          }
          if constexpr (ks == 0) {
            __builtin_amdgcn_sched_barrier(0);
            load(i + S::AHEAD, (u + S::AHEAD) % S::NS);
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      }
    }
  }
  wait_vmcnt<0>();   // loads into LDS of steps that there are not, in either loop: none may land when its stage has a new use
  __syncthreads();
  // Sums to LDS, KW planes of TM rows; then a thread adds the planes of 8 columns of a row at a time.
  float* const out = reinterpret_cast<float*>(smem + grp * S::TM * S::PITCH);
#pragma unroll
  for (int a = 0; a < S::BM; ++a)
#pragma unroll
    for (int b = 0; b < S::BN; ++b)
#pragma unroll
      for (int e = 0; e < RE; ++e) {
        const int row = (wm * S::BM + a) * 32 + acc_row(e, lane);
        out[row * (S::PITCH / 4) + (wn * S::BN + b) * 32 + lr] = acc[a][b][e];
      }
  __syncthreads();
  if (left <= 0) return;
  with_act(p.act, [&](auto act_t) {
    constexpr int ACT = decltype(act_t)::value;
    for (int r = tid / CPR; r < min(S::TM, p.M - m0); r += S::NT / CPR) {
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
        y[e] = act_w4<ACT>(p.bias ? y[e] + bias[e] : y[e]);
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

// The k that a tile's sums take a scale for: pairs of steps where more than a block is folded (48 x 12288 x 4096 E2M1
// 13.6 -> 12.3 us) and every group of waves has as many pairs, or nearly.
inline int w4_fold(int blocks, int KW, int K, int group) {
  const int pairs = K / 128;
  if (blocks > 1 && group % 128 == 0 && (pairs % KW == 0 || pairs >= 4 * KW)) return 128;
  return group % 64 == 0 ? 64 : 32;
}

template <class S, bool E2M1, class T>
hipError_t launch_code(const GemmW4Params& p, hipStream_t st) {
  const int64_t wgs = (int64_t)((p.M + S::TM - 1) / S::TM) * ((p.N + S::TN - 1) / S::TN);
  const uint32_t g32 = p.group / 32, mul = g32 == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + g32 - 1) / g32);
  const int fold = w4_fold(S::BM * S::BN, S::KW, p.K, p.group);
  if constexpr (S::BM * S::BN > 1) {
    if (fold == 128) {
      hipLaunchKernelGGL((gemm_w4_kernel<S, E2M1, 128, T>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p, mul);
      return hipGetLastError();
    }
  }
  if (fold == 64) hipLaunchKernelGGL((gemm_w4_kernel<S, E2M1, 64, T>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p, mul);
  else hipLaunchKernelGGL((gemm_w4_kernel<S, E2M1, 32, T>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p, mul);
  return hipGetLastError();
}

// The compiled tiles; cf_w4.hip chooses between them.
template <class... S>
struct W4Tiles {
  template <bool E2M1, class L>
  static hipError_t launch_of(const GemmW4Params& p, hipStream_t st) {
    return p.s_f32 ? launch_code<L, E2M1, float>(p, st) : launch_code<L, E2M1, bf16_t>(p, st);
  }
  template <bool E2M1>
  static hipError_t launch(int tile, const GemmW4Params& p, hipStream_t st) {
    using Launch = hipError_t (*)(const GemmW4Params&, hipStream_t);
    static constexpr Launch all[] = {launch_of<E2M1, S>...};
    return all[tile](p, st);
  }
};
using AllW4Tiles = W4Tiles<W4Tile<1, 1, 1, 1, 8, 4, 8>, W4Tile<1, 2, 1, 1, 8, 4, 16>, W4Tile<1, 1, 1, 1, 8, 4, 32>,
                           W4Tile<1, 2, 1, 1, 8, 4, 32>, W4Tile<2, 1, 1, 1, 8, 2, 64>, W4Tile<2, 2, 1, 1, 4, 4, 64>,
                           W4Tile<2, 2, 1, 2, 4, 2, 64>, W4Tile<2, 2, 2, 2, 1, 4, 128>>;

}  // namespace

hipError_t launch_w4_int4(int tile, const GemmW4Params& p, hipStream_t st);   // cf_w4_int4.hip
hipError_t launch_w4_e2m1(int tile, const GemmW4Params& p, hipStream_t st);   // cf_w4_e2m1.hip

}  // namespace cf
