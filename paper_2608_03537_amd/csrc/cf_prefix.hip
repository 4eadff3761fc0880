// Attention of a batch whose sequences share a prefix:
//     O_b = softmax(scale Q_b [Kp; Ks_b]^T) [Vp; Vs_b].
//
// Rows.  The queries of one (sequence, key head) are G Lq rows, G = H / Hk query
// heads per key head, ordered query-major (row i G + g is query i of head g), so a
// block of rows spans few queries and causal limits stay close.
//
// Products.  As in b2b_attention_kernel: S^T = K Q^T on 32 x 32 blocks, so a lane
// holds one query row and 16 of its keys; P goes from the accumulators to the
// second product O^T = V^T P^T in registers, V^T by transposing LDS reads.  A wave
// owns 32 rows and keeps the running maximum m and sum l of each (fp32, raised
// lazily).
#include <algorithm>

#include "cf_attn.h"
#include "cf_gemm_tile.h"

namespace cf {

namespace {

// QG waves own 32 rows each; KS groups of QG waves share the rows and take the
// key blocks (BK keys) in turn, each with a ring of two stages in LDS.
template <int D, int QG_, int KS_, int BK_>
struct PrefixShape {
  static constexpr int QG = QG_, KS = KS_, NW = QG * KS, NT = 64 * NW, TM = 32 * QG, BK = BK_;
  static constexpr int NH = BK / 32;              // 32-key parts of a block
  static constexpr int ROW = D * 2, CH = ROW / 16;   // bytes and 16-byte chunks of a key or value row
  static constexpr int KB = BK * ROW, STAGE = 2 * KB;
  static constexpr int RING = KS * 2 * STAGE;
  static constexpr int OROW = D * 4 + 16;         // merge of the groups: one row's fp32 O
  static constexpr int OUT = NW * 32 * (OROW + 8);
  static constexpr int LDS = RING > OUT ? RING : OUT;
  static constexpr int DK = D / 16, BD = D / 32;  // MFMA steps over d, 32-wide blocks of d
  static constexpr int NSA = NH * DK, NSB = 2 * NH * BD;
  static_assert(LDS <= 160 * 1024 && 2 * STAGE <= 65536, "LDS budget, ds offset field");
};

// Own keys of sequence b, and how many of them query i sees.
__device__ __forceinline__ int own_len(const PrefixParams& p, int b) {
  return p.lens ? max(0, min(p.lens[b], p.S)) : p.S;
}
__device__ __forceinline__ int own_seen(const PrefixParams& p, int len, int i) {
  return p.causal ? max(0, len - (p.Lq - 1 - i)) : len;
}

template <int D, int QG, int KS, int BK>
__global__ __launch_bounds__(64 * QG * KS, 2) void prefix_kernel(PrefixParams p) {
  using A = PrefixShape<D, QG, KS, BK>;
  __shared__ __attribute__((aligned(16))) char smem[A::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int wq = KS == 1 ? wave : wave % QG, grp = KS == 1 ? 0 : wave / QG;
  const int G = p.H / p.Hk, R = G * p.Lq;
  const int m0 = blockIdx.x * A::TM;
  const int hk = blockIdx.y % p.Hk, b = blockIdx.y / p.Hk;
  const float sl2 = p.scale * 1.4426950408889634f;   // scale * log2(e), > 0
  constexpr float kLazy = 8.0f;                       // rescale threshold (log2 units)

  // Q fragments (B operand of S^T = K Q^T): this lane's row, 8 d per step.
  const int m = min(m0 + wq * 32 + lr, R - 1), qi = m / G, qh = hk * G + m % G;
  u32x4_t qf[A::DK];
  {
    const bf16_t* q = p.Q + b * p.q_b + qh * p.q_h + qi * p.q_l;
#pragma unroll
    for (int ks = 0; ks < A::DK; ++ks) qf[ks] = gload16(q + ks * 16 + lg * 8);
  }
  const int len = own_len(p, b);

  // Swizzles of the 16-byte chunks of a row, for the fragment reads (K) and the
  // transposing reads (V); see b2b_attention_kernel.
  auto kswz = [](int row) { return A::CH == 16 ? (row & 15) : ((row >> 1) & 7); };
  auto vswz = [](int row) { return A::CH == 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); };
  constexpr int LPR = A::CH, RPI = 64 / LPR;      // lanes per row, rows per wave-wide load
  constexpr int NINS = BK / RPI / QG;             // loads per wave for the K or V of a block
  char* const ring = smem + grp * 2 * A::STAGE;
  const uint32_t s0 =
      (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem) + grp * 2 * A::STAGE;
  uint32_t kbase[A::DK], vbase[A::BD];
  const int r16 = lane & 15, vrow = 4 * lg + (r16 >> 2);
#pragma unroll
  for (int ks = 0; ks < A::DK; ++ks) kbase[ks] = s0 + lr * A::ROW + (((2 * ks + lg) ^ kswz(lr)) << 4);
#pragma unroll
  for (int d = 0; d < A::BD; ++d)
    vbase[d] = s0 + vrow * A::ROW + ((((32 * d + (lane & 16) + 4 * (r16 & 3)) >> 3) ^ vswz(vrow)) << 4) + 8 * (r16 & 1);
  auto lds_sync = [] {
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));
    lds_barrier();
  };

  f32x16_t O[A::BD];
#pragma unroll
  for (int d = 0; d < A::BD; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) O[d][e] = 0.0f;
  float m_used = -INFINITY, lsum = 0.0f;

  using S0_ = std::integral_constant<int, 0>;
  using S1_ = std::integral_constant<int, 1>;
  // The prefix, then the sequence's own keys.
#pragma unroll 1
  for (int seg = 0; seg < 2; ++seg) {
    const bf16_t* Kb = seg == 0 ? p.Kp + hk * p.kp_h : p.Ks + b * p.ks_b + hk * p.ks_h;
    const bf16_t* Vb = seg == 0 ? p.Vp + hk * p.vp_h : p.Vs + b * p.vs_b + hk * p.vs_h;
    const int64_t ldk = seg == 0 ? p.kp_l : p.ks_l, ldv = seg == 0 ? p.vp_l : p.vs_l;
    const int nk = seg == 0 ? p.P : len;                       // keys that may be read
    const int lim = seg == 0 ? p.P : own_seen(p, len, qi);     // keys that this lane's row sees
    const int first = seg == 0 ? p.P : own_seen(p, len, m0 / G);   // ... that every row sees
    const int last = seg == 0 ? p.P : own_seen(p, len, (min(m0 + A::TM, R) - 1) / G);   // ... that some row sees
    const int NB = (last + BK - 1) / BK;

    auto issue_kv = [&](int j, auto stage_t) {
      char* dst = ring + decltype(stage_t)::value * A::STAGE;
#pragma unroll
      for (int ins = 0; ins < NINS; ++ins) {
        const int in = wq + QG * ins, row = in * RPI + lane / LPR;
        const int key = min(j * BK + row, nk - 1);   // rows behind nk: clamped here, masked in P, zeroed in V
        dma16(reinterpret_cast<const char*>(Kb + key * ldk) + (((lane % LPR) ^ kswz(row)) << 4), dst + in * 1024);
        dma16(reinterpret_cast<const char*>(Vb + key * ldv) + (((lane % LPR) ^ vswz(row)) << 4),
              dst + A::KB + in * 1024);
      }
    };
    auto step = [&](int j, auto stage_t, auto next_t) {
      constexpr int ST = decltype(stage_t)::value * A::STAGE;
      wait_vmcnt<0>();
      lds_sync();
      if (j >= NB) return;
      if (j + KS < NB) issue_kv(j + KS, next_t);
      // S^T = K Q^T
      f32x16_t S[A::NH];
      {
        constexpr int KLA = 4;
        const f32x16_t zero = {};
        auto kread = [&](auto i_t) {
          constexpr int i = decltype(i_t)::value;
          return ds_read_b128_at<ST + (i % A::NH) * 32 * A::ROW>(kbase[i / A::NH]);
        };
        u32x4_t kf[KLA];
        static_for<0, KLA>([&](auto i_t) { kf[decltype(i_t)::value] = kread(i_t); });
        static_for<0, A::NSA>([&](auto i_t) {
          constexpr int i = decltype(i_t)::value, h = i % A::NH, ks = i / A::NH, rest = A::NSA - 1 - i;
          lgkm_wait<(rest < KLA - 1 ? rest : KLA - 1)>(kf[i % KLA]);
          S[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i % KLA]),
                                                         __builtin_bit_cast(bf16x8_t, qf[ks]), ks == 0 ? zero : S[h], 0,
                                                         0, 0);
          if constexpr (i + KLA < A::NSA) kf[(i + KLA) % KLA] = kread(std::integral_constant<int, i + KLA>{});
          __builtin_amdgcn_sched_barrier(0);
        });
      }
      const bool mask = (j + 1) * BK > first;   // some row of the workgroup does not see the whole block
      if (mask) {
#pragma unroll
        for (int e = 0; e < 16 * A::NH; ++e) {
          const int key = j * BK + (e >> 4) * 32 + acc_row(e & 15, lane);
          if (key >= lim) S[e >> 4][e & 15] = -INFINITY;
        }
      }
      // softmax of the block
      float t = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16 * A::NH; ++e) t = fmaxf(t, S[e >> 4][e & 15]);
      const float mnew = fmaxf(m_used, lane_pair_max(t) * sl2);
      const bool need = mnew > m_used + kLazy;
      const float m_eff = need ? mnew : m_used;
      const float corr = need ? __builtin_amdgcn_exp2f(m_used - m_eff) : 1.0f;
      m_used = m_eff;
      const float nm = m_used == -INFINITY ? 0.0f : -m_used;   // nothing seen yet: P are 0
      u32x4_t P[A::NH][2];
#pragma unroll
      for (int e = 0; e < 16 * A::NH; ++e)
        S[e >> 4][e & 15] = __builtin_amdgcn_exp2f(fmaf(S[e >> 4][e & 15], sl2, nm));
#pragma unroll
      for (int h = 0; h < A::NH; ++h) {
        P[h][0] = pack_step(S[h], 0);
        P[h][1] = pack_step(S[h], 1);
      }
      if (__any(need)) {
#pragma unroll
        for (int d = 0; d < A::BD; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) O[d][e] *= corr;
        lsum *= corr;
      }
      // O^T += V^T P^T; in a block that reaches behind nk the values there are
      // zeroed (0 * NaN would not be 0)
      auto pv = [&](auto mask_t) {
        constexpr int VT = ST + A::KB;
        auto vfrag = [&](auto i_t) {
          constexpr int i = decltype(i_t)::value;
          constexpr int d = i % A::BD, s = (i / A::BD) & 1, h = i / (2 * A::BD);
          constexpr int off = VT + (32 * h + 16 * s) * A::ROW;
          const u32x2_t lo = ds_read_tr_b64<off>(vbase[d]);
          const u32x2_t hi = ds_read_tr_b64<off + 8 * A::ROW>(vbase[d]);
          return u32x4_t{lo[0], lo[1], hi[0], hi[1]};
        };
        u32x4_t vf[3];
        vf[0] = vfrag(std::integral_constant<int, 0>{});
        vf[1] = vfrag(std::integral_constant<int, 1>{});
        static_for<0, A::NSB>([&](auto i_t) {
          constexpr int i = decltype(i_t)::value;
          constexpr int d = i % A::BD, s = (i / A::BD) & 1, h = i / (2 * A::BD);
          lgkm_wait<(i + 1 < A::NSB ? 2 : 0)>(vf[i % 3]);
          u32x4_t v = vf[i % 3];
          if constexpr (decltype(mask_t)::value) {
            const int left = nk - (j * BK + 32 * h + 16 * s + 4 * lg);   // of the 4 keys of v[0..1]; v[2..3]: 8 on
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int l = left - (e < 2 ? 2 * e : 8 + 2 * (e - 2));
              v[e] = l >= 2 ? v[e] : l == 1 ? v[e] & 0xFFFFu : 0u;
            }
          }
          Mma<bf16_t>::run(O[d], v, P[h][s]);
          if constexpr (i + 2 < A::NSB) vf[(i + 2) % 3] = vfrag(std::integral_constant<int, i + 2>{});
          __builtin_amdgcn_sched_barrier(0);
        });
      };
      if ((j + 1) * BK > nk) pv(std::true_type{});
      else pv(std::false_type{});
      // the row sum from the same bf16 P as the numerator
      typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
      const bf16x2_t one2 = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);
#pragma unroll
      for (int q = 0; q < 2 * A::NH; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = P[q >> 1][q & 1][e];
          lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x), one2, lsum, false);
        }
    };
    if (grp < NB) issue_kv(grp, S0_{});
    for (int j = 0; j < NB; j += 2 * KS) {
      step(j + grp, S0_{}, S1_{});
      if (j + KS < NB) step(j + KS + grp, S1_{}, S0_{});
    }
    __syncthreads();   // the rings are free for the next segment, or for the merge
  }

  // Every wave leaves its O and (m, l) in LDS; thread t takes 8 d of a row and adds
  // the groups in order, scaled to the common maximum.
  const float l = lane_pair_sum(lsum);
  char* const orow = smem + (wave * 32 + lr) * A::OROW;
#pragma unroll
  for (int d = 0; d < A::BD; ++d)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      *reinterpret_cast<f32x4_t*>(orow + (32 * d + 8 * g4 + 4 * lg) * 4) =
          f32x4_t{O[d][4 * g4], O[d][4 * g4 + 1], O[d][4 * g4 + 2], O[d][4 * g4 + 3]};
  float* const ml = reinterpret_cast<float*>(smem + A::NW * 32 * A::OROW);
  if (lg == 0) {
    ml[(wave * 32 + lr) * 2] = m_used;
    ml[(wave * 32 + lr) * 2 + 1] = l;
  }
  __syncthreads();
  constexpr int TPR = D / 8;
  const int rows = min(A::TM, R - m0), d0 = tid % TPR * 8;
  for (int r = tid / TPR; r < rows; r += A::NT / TPR) {
    float mg[KS], M = -INFINITY, L = 0.0f, o[8] = {};
#pragma unroll
    for (int q = 0; q < KS; ++q) M = fmaxf(M, mg[q] = ml[((q * QG + r / 32) * 32 + r % 32) * 2]);
#pragma unroll
    for (int q = 0; q < KS; ++q) {
      const int w = (q * QG + r / 32) * 32 + r % 32;
      const float f = mg[q] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mg[q] - M);
      L = fmaf(f, ml[w * 2 + 1], L);
      const float* src = reinterpret_cast<const float*>(smem + w * A::OROW) + d0;
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(src), y = *reinterpret_cast<const f32x4_t*>(src + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e] = fmaf(f, x[e], o[e]);
        o[4 + e] = fmaf(f, y[e], o[4 + e]);
      }
    }
    const int i = (m0 + r) / G, h = hk * G + (m0 + r) % G;
    const float inv = p.P + own_seen(p, len, i) > 0 ? 1.0f / L : 0.0f;   // a row without keys: 0
    const u32x4_t w = {pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                       pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv)};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(p.O + b * p.o_b + h * p.o_h + i * p.o_l + d0));
  }
}

template <int D, int QG, int KS, int BK>
hipError_t launch_direct(const PrefixParams& p, hipStream_t st) {
  using A = PrefixShape<D, QG, KS, BK>;
  const int R = p.H / p.Hk * p.Lq;
  hipLaunchKernelGGL((prefix_kernel<D, QG, KS, BK>), dim3((unsigned)((R + A::TM - 1) / A::TM), (unsigned)(p.B * p.Hk)),
                     dim3(A::NT), 0, st, p);
  return hipGetLastError();
}

}  // namespace

size_t prefix_workspace(const PrefixParams&) { return 0; }

hipError_t launch_prefix(const PrefixParams& p, hipStream_t st) {
  const bool few = p.H / p.Hk * p.Lq <= 32;
  if (p.d == 128) return few ? launch_direct<128, 1, 4, 32>(p, st) : launch_direct<128, 4, 1, 64>(p, st);
  return few ? launch_direct<64, 1, 8, 32>(p, st) : launch_direct<64, 4, 1, 64>(p, st);
}

}  // namespace cf
