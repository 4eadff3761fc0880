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
#include <cmath>
#include <cstdio>

#include "cf_attn.h"
#include "cf_gemm_tile.h"
#include "cf_serving.h"
#include "comfuse.h"

namespace cf {

namespace {

// QG waves own 32 rows each; KS groups of QG waves share the rows and take the key blocks
// (BK keys) in turn, each with an LDS ring of its own.  Two forms:
//   QG = 4, KS = 1, two stages: the next block loads while one is multiplied; a
//     barrier per block.  For many rows.
//   QG = 1, KS = 4, one stage per wave: the next keys load as soon as S^T is done, the next
//     values after P V.  No barrier until the end.  For few rows, where the keys' stream counts.
// Both fit a CU twice, so that two waves share a SIMD, and a workgroup of one form can run
// beside one of the other.
template <int D, int QG_>
struct PrefixShape {
  static constexpr int QG = QG_, KS = 4 / QG, NW = 4, NT = 256, TM = 32 * QG, BK = QG == 1 ? 4096 / D : 64;
  static constexpr int NH = BK / 32;              // 32-key parts of a block
  static constexpr int ROW = D * 2, CH = ROW / 16;   // bytes and 16-byte chunks of a key or value row
  static constexpr int NS = QG == 1 ? 1 : 2;      // stages
  static constexpr int KB = BK * ROW, STAGE = 2 * KB, RING = NS * STAGE;
  static constexpr int OROW = D * 4 + 16;         // merge of the groups: one row's fp32 O
  static constexpr int OUT = NW * 32 * (OROW + 8);
  static constexpr int LDS = KS * RING > OUT ? KS * RING : OUT;
  static constexpr int DK = D / 16, BD = D / 32;  // MFMA steps over d, 32-wide blocks of d
  static constexpr int NSA = NH * DK, NSB = 2 * NH * BD;
  static constexpr int RPI = 64 / CH, NINS = BK / RPI / QG;   // rows of a wave-wide load; a wave's loads of K or V
  static_assert(QG == 1 || QG == 4, "forms");
  static_assert(LDS <= 80 * 1024 && RING <= 65536, "two workgroups a CU, ds offset field");
};

// Own keys of sequence b, and how many of them query i sees.
__device__ __forceinline__ int own_len(const PrefixParams& p, int b) {
  return p.lens ? max(0, min(p.lens[b], p.S)) : p.S;
}
__device__ __forceinline__ int own_seen(const PrefixParams& p, int len, int i) {
  return p.causal ? max(0, len - (p.Lq - 1 - i)) : len;
}

// 8 d of the output row of query i of head h: o / l, or 0 where the row sees no key (o may be NaN
// there: 0 times what a value row that it does not see holds).
__device__ __forceinline__ void store_row(const PrefixParams& p, int b, int h, int i, int d0, const float (&o)[8], float l,
                                          bool any) {
  const float inv = 1.0f / l;
  u32x4_t w = {pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
               pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv)};
  if (!any) w = u32x4_t{};
  __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(p.O + b * p.o_b + h * p.o_h + i * p.o_l + d0));
}

// What a launch computes: whole rows of (sequence, key head) pairs over the prefix
// and their own keys, or a part of the prefix for the rows of all sequences, or a
// part of the own keys; the parts' (m, l, O) meet in the workspace.
enum Kind { WHOLE = 0, PREFIX = 1, OWN = 2 };

// Partial results: fp32 O [slot][row][D], then (m, l) [slot][row]; row (b Hk + hk) R + m.
struct PartRows {
  int64_t rows;   // B Hk R
  __device__ __host__ float* o(const PrefixParams& p, int slot, int64_t row) const {
    return p.ws + (slot * rows + row) * p.d;
  }
  __device__ __host__ float* ml(const PrefixParams& p, int slots, int slot, int64_t row) const {
    return p.ws + slots * rows * p.d + (slot * rows + row) * 2;
  }
};

// Whole rows in parts, up to 32 rows of a (sequence, key head): the workgroup that finishes one last
// joins its parts, which saves a launch (3 us of the host; 1 x 12 heads, 89 + 431 keys 14.3 -> 11.7 us a
// call from Python).  Each has an arrival counter, zero between calls.  A workgroup of the prefix's
// parts has rows of several sequences, and would join all of them if it came last (47 x 16 heads 17
// -> 70 us): those keep the second launch.

// The parts of the rows of (b, hk), by the whole workgroup: RPP rows at a time, D / 8 threads a part's row beside
// each other.  Of 8 rows, others take the parts in turn (WAYS); of 32, each thread takes all parts, at d = 128 of
// two rows (2 x 32 heads of 8, 2 queries, 1500 + 100 keys, d 64: 8 rows at a time 9.4 us a call, so 8.5).
// The grouping depends on the sizes only.
constexpr int kJoinFew = 8;
template <int D, int RPP>
__device__ __forceinline__ void join_rows(const PrefixParams& p, char* smem, int b, int hk, int slots) {
  constexpr int TPR = D / 8, SETS = 256 / TPR, RS = RPP < SETS ? RPP : SETS;   // rows beside each other
  constexpr int WAYS = SETS / RS, RT = RPP / RS, AHEAD = RT == 2 ? 4 : 6;
  const int tid = threadIdx.x, g = tid / TPR, r = g % RS, way = g / RS, d0 = tid % TPR * 8;
  const int G = p.H / p.Hk, R = G * p.Lq;
  const uint32_t rows = (uint32_t)(p.B * p.Hk * R), ml0 = (uint32_t)slots * rows * (D * 4);
  float* const so = reinterpret_cast<float*>(smem);             // [WAYS][RS][D + 4]
  const int len = own_len(p, b);
  float M[RT], L[RT], o[RT][8];
  uint32_t row[RT];
#pragma unroll
  for (int k = 0; k < RT; ++k) {
    row[k] = (uint32_t)((b * p.Hk + hk) * R + min(r + k * RS, R - 1));
    M[k] = -INFINITY;
    L[k] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[k][e] = 0.0f;
  }
  auto join = [&](int k, float mz, float lz, const float (&x)[8]) {
    const float mn = fmaxf(M[k], mz);
    const float fo = M[k] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M[k] - mn);
    const float fz = mz == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mz - mn);
    M[k] = mn;
    L[k] = fmaf(fz, lz, fo * L[k]);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[k][e] = fmaf(fz, x[e], fo * o[k][e]);
  };
  for (int s0 = way; s0 < slots; s0 += AHEAD * WAYS) {
    u32x4_t x[AHEAD][RT], y[AHEAD][RT];
    u32x2_t v[AHEAD][RT];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
#pragma unroll
      for (int k = 0; k < RT; ++k) {
        const uint32_t at = (uint32_t)min(s0 + q * WAYS, slots - 1) * rows + row[k];
        x[q][k] = coherent_load16(p.ws, at * (D * 4) + d0 * 4);
        y[q][k] = coherent_load16(p.ws, at * (D * 4) + d0 * 4 + 16);
        v[q][k] = coherent_load8(p.ws, ml0 + at * 8);
      }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
      if (s0 + q * WAYS < slots) {
#pragma unroll
        for (int k = 0; k < RT; ++k) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f[e] = __uint_as_float(x[q][k][e]);
            f[4 + e] = __uint_as_float(y[q][k][e]);
          }
          join(k, __uint_as_float(v[q][k][0]), __uint_as_float(v[q][k][1]), f);
        }
      }
  }
  if constexpr (WAYS > 1) {
    float* const mine = so + (way * RS + r) * (D + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) mine[d0 + e] = o[0][e];
    if (d0 == 0) {
      mine[D] = M[0];
      mine[D + 1] = L[0];
    }
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int w = 1; w < WAYS; ++w) {
      const float* other = so + (w * RS + r) * (D + 4);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = other[d0 + e];
      join(0, other[D], other[D + 1], f);
    }
  }
#pragma unroll
  for (int k = 0; k < RT; ++k) {
    const int m = r + k * RS;
    if (m < R) store_row(p, b, hk * G + m % G, m / G, d0, o[k], L[k], p.P > 0 || own_seen(p, len, m / G) > 0);
  }
}

// Rows m0 .. of (b, hk), or with PREFIX of all sequences of hk, over part z of `parts` of their key
// blocks.  slots = 0: the output rows; else partial results, this one at `slot`.
template <int KIND, int D, int QG, bool JOIN>
__device__ __forceinline__ void attend(const PrefixParams& p, char* smem, int rb, int b, int hk, int z, int parts, int slot,
                                       int slots, unsigned* count) {
  using A = PrefixShape<D, QG>;
  constexpr int KS = A::KS, BK = A::BK;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int wq = wave % QG, grp = wave / QG;
  const int G = p.H / p.Hk, R = G * p.Lq;             // rows of a sequence and key head
  const int m0 = rb * A::TM, Rall = KIND == PREFIX ? p.B * R : R;
  const float sl2 = p.scale * 1.4426950408889634f;   // scale * log2(e), > 0
  constexpr float kLazy = 8.0f;                       // rescale threshold (log2 units)

  // Q fragments (B operand of S^T = K Q^T): this lane's row, 8 d per step.
  const int m = min(m0 + wq * 32 + lr, Rall - 1), qb = KIND == PREFIX ? m / R : b;
  const int qm = KIND == PREFIX ? m % R : m, qi = qm / G, qh = hk * G + qm % G;
  u32x4_t qf[A::DK];
  {
    const bf16_t* q = p.Q + qb * p.q_b + qh * p.q_h + qi * p.q_l;
#pragma unroll
    for (int ks = 0; ks < A::DK; ++ks) qf[ks] = gload16(q + ks * 16 + lg * 8);
  }
  const int len = KIND == PREFIX ? 0 : own_len(p, b);

  // Key blocks: those of the prefix, then those of the own keys; [jb, NB) are this part's.
  const int nbp = KIND == OWN ? 0 : (p.P + BK - 1) / BK;
  const int last = KIND == PREFIX ? 0 : own_seen(p, len, (min(m0 + A::TM, R) - 1) / G);   // own keys that some row sees
  const int first = KIND == PREFIX ? 0 : own_seen(p, len, m0 / G);                        // ... that every row sees
  const int seen = KIND == PREFIX ? 0 : own_seen(p, len, qi);                             // ... that this lane's row sees
  const int nball = nbp + (last + BK - 1) / BK;
  // (at most 2^25 + 2^25 blocks and 32 parts: the products are at most 2^31; asserted at kMaxParts)
  const int jb = (int)((uint32_t)nball * z / (uint32_t)parts), NB = (int)((uint32_t)nball * (z + 1) / (uint32_t)parts);
  const bf16_t* const Kp = p.Kp + hk * p.kp_h;
  const bf16_t* const Vp = p.Vp + hk * p.vp_h;
  const bf16_t* const Ks = p.Ks + b * p.ks_b + hk * p.ks_h;
  const bf16_t* const Vs = p.Vs + b * p.vs_b + hk * p.vs_h;

  // Swizzles of the 16-byte chunks of a row, for the fragment reads (K) and the
  // transposing reads (V); see b2b_attention_kernel.
  auto kswz = [](int row) { return A::CH == 16 ? (row & 15) : ((row >> 1) & 7); };
  auto vswz = [](int row) { return A::CH == 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); };
  char* const ring = smem + grp * A::RING;
  const uint32_t s0 =
      (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem) + grp * A::RING;
  uint32_t kbase[A::DK], vbase[A::BD];
  const int r16 = lane & 15, vrow = 4 * lg + (r16 >> 2);
#pragma unroll
  for (int ks = 0; ks < A::DK; ++ks) kbase[ks] = s0 + lr * A::ROW + (((2 * ks + lg) ^ kswz(lr)) << 4);
#pragma unroll
  for (int d = 0; d < A::BD; ++d)
    vbase[d] = s0 + A::KB + vrow * A::ROW + ((((32 * d + (lane & 16) + 4 * (r16 & 3)) >> 3) ^ vswz(vrow)) << 4) + 8 * (r16 & 1);
  auto fence = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // Load `ins` of this wave's share of the keys (or values) of block j: rows in RPI .. + RPI - 1,
  // in = wq + QG ins, a wave-uniform base and a lane's offset (row stride below 2^23 bytes).  The swizzle
  // of a lane's chunk depends on `in` through in % 4 (d = 128) or in % 2 only, NP values over a
  // wave's loads.  In a block that reaches behind the last key that may be read, rows are
  // clamped; they are masked in P and zeroed in V.
  constexpr int NP = A::CH == 16 ? 4 / QG : (QG == 1 ? 2 : 1);
  const int lrow = lane / A::CH, lch = lane % A::CH;
  uint32_t kc[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) kc[i] = (lch ^ kswz((wq + QG * i) * A::RPI + lrow)) << 4;
  const uint32_t vc = (lch ^ vswz(lrow)) << 4;
  struct Block {   // where the keys and values of a block lie
    const char *k, *v;
    int ldk, ldv, left;   // bytes a row; rows that may be read from its first key on
  };
  auto block = [&](int j) {
    const bool own = j >= nbp;
    const int k0 = (own ? j - nbp : j) * BK;
    Block bl;
    bl.ldk = (int)(own ? p.ks_l : p.kp_l) * 2;
    bl.ldv = (int)(own ? p.vs_l : p.vp_l) * 2;
    bl.k = reinterpret_cast<const char*>(own ? Ks : Kp) + (int64_t)k0 * bl.ldk;
    bl.v = reinterpret_cast<const char*>(own ? Vs : Vp) + (int64_t)k0 * bl.ldv;
    bl.left = (own ? len : p.P) - k0;
    return bl;
  };
  auto load = [&](const Block& bl, int stage, auto v_t, auto full_t, int ins) {
    constexpr bool V = decltype(v_t)::value, FULL = decltype(full_t)::value;
    const int in = wq + QG * ins, ld = V ? bl.ldv : bl.ldk;
    const char* src = V ? bl.v : bl.k;
    const uint32_t c = V ? vc : kc[ins % NP];
    char* dst = ring + stage * A::STAGE + (V ? A::KB : 0) + in * 1024;
    if constexpr (FULL) dma16_at(src, __mul24(lrow, ld) + c, in * A::RPI * ld, dst);
    else dma16_at(src, __mul24(min(in * A::RPI + lrow, bl.left - 1), ld) + c, 0, dst);
  };
  // All of this wave's loads of the keys or of the values of a block.
  auto load_all = [&](const Block& bl, int stage, auto v_t) {
    if (bl.left >= BK) {
#pragma unroll
      for (int i = 0; i < A::NINS; ++i) load(bl, stage, v_t, std::true_type{}, i);
    } else {
#pragma unroll
      for (int i = 0; i < A::NINS; ++i) load(bl, stage, v_t, std::false_type{}, i);
    }
  };

  f32x16_t O[A::BD];
#pragma unroll
  for (int d = 0; d < A::BD; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) O[d][e] = 0.0f;
  float m_used = -INFINITY, lsum = 0.0f;

  auto step = [&](int j, auto stage_t) {
    constexpr int SG = decltype(stage_t)::value, ST = SG * A::STAGE;
    const bool own = j >= nbp, next = j + KS < NB;
    const int k0 = (own ? j - nbp : j) * BK;
    if constexpr (QG == 1) {
      wait_vmcnt<A::NINS>();   // the keys; the values may be on their way
      fence();
    } else {
      wait_vmcnt<0>();
      __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));   // this wave's LDS reads
      lds_barrier();           // the block is in, and every wave is done with the other stage
    }
    // S^T = K Q^T: one LDS read per MFMA, four ahead.  With two stages the next block's loads
    // go between the MFMAs: in a row they would hold the wave up.
    f32x16_t S[A::NH];
    const Block nb = block(next ? j + KS : j);
    auto scores = [&](auto load_t, auto full_t) {
      constexpr int KLA = 4;
      constexpr int SPC = A::NSA / (2 * A::NINS) > 0 ? A::NSA / (2 * A::NINS) : 1;   // MFMAs per load
      constexpr int LPM = 2 * A::NINS > A::NSA ? 2 * A::NINS / A::NSA : 1;          // loads per MFMA
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
                                                       __builtin_bit_cast(bf16x8_t, qf[ks]), ks == 0 ? zero : S[h], 0, 0,
                                                       0);
        if constexpr (i + KLA < A::NSA) kf[(i + KLA) % KLA] = kread(std::integral_constant<int, i + KLA>{});
        if constexpr (decltype(load_t)::value)
          static_for<0, LPM>([&](auto l_t) {
            constexpr int q = i / SPC * LPM + decltype(l_t)::value;
            if constexpr (i % SPC == SPC - 1 && q < 2 * A::NINS)
              load(nb, 1 - SG, std::integral_constant<bool, (q >= A::NINS)>{}, full_t, q % A::NINS);
          });
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    if (A::NS == 1 || !next) scores(std::false_type{}, std::false_type{});
    else if (nb.left >= BK) scores(std::integral_constant<bool, A::NS == 2>{}, std::true_type{});
    else scores(std::integral_constant<bool, A::NS == 2>{}, std::false_type{});
    if constexpr (QG == 1) {
      fence();   // the last read of the keys has returned
      if (next) load_all(nb, 0, std::false_type{});
    }
    if (k0 + BK > (own ? first : p.P)) {   // some row of the workgroup does not see the whole block
      const int lim = own ? seen : p.P;
#pragma unroll
      for (int e = 0; e < 16 * A::NH; ++e)
        if (k0 + (e >> 4) * 32 + acc_row(e & 15, lane) >= lim) S[e >> 4][e & 15] = -INFINITY;
    }
    // softmax of the block
    float t = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16 * A::NH; ++e) t = fmaxf(t, S[e >> 4][e & 15]);
    const float mnew = fmaxf(m_used, lane_pair_max_swap(t) * sl2);
    const bool need = mnew > m_used + kLazy;
    const float m_eff = need ? mnew : m_used;
    const float corr = need ? __builtin_amdgcn_exp2f(m_used - m_eff) : 1.0f;
    m_used = m_eff;
    const float nm = m_used == -INFINITY ? 0.0f : -m_used;   // nothing seen yet: P are 0
    // P goes to the second product as bf16, the type of V and so of the MFMA's other operand.  Of the output's error
    // against 64 bits, 0.0022 to 0.0023 (relative norm), 0.0017 is its own rounding and 0.0014 to 0.0016 this one;
    // P as a sum of two bf16 would double the product.
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
    if constexpr (QG == 1) {   // the values; the next keys may be on their way
      if (next) wait_vmcnt<A::NINS>();
      else wait_vmcnt<0>();
      fence();
    }
    // O^T += V^T P^T; in a block that reaches behind the last key the values there are
    // zeroed (0 * NaN would not be 0)
    const int nk = own ? len : p.P;
    auto pv = [&](auto mask_t) {
      auto vfrag = [&](auto i_t) {
        constexpr int i = decltype(i_t)::value;
        constexpr int d = i % A::BD, s = (i / A::BD) & 1, h = i / (2 * A::BD);
        constexpr int off = ST + (32 * h + 16 * s) * A::ROW;
        const u32x2_t lo = ds_read_tr_b64<off>(vbase[d]);
        const u32x2_t hi = ds_read_tr_b64<off + 8 * A::ROW>(vbase[d]);
        return u32x4_t{lo[0], lo[1], hi[0], hi[1]};
      };
      constexpr int VLA = 2;
      u32x4_t vf[VLA + 1];
      static_for<0, VLA>([&](auto i_t) { vf[decltype(i_t)::value] = vfrag(i_t); });
      static_for<0, A::NSB>([&](auto i_t) {
        constexpr int i = decltype(i_t)::value, rest = A::NSB - 1 - i;
        constexpr int d = i % A::BD, s = (i / A::BD) & 1, h = i / (2 * A::BD);
        lgkm_wait<2 * (rest < VLA - 1 ? rest : VLA - 1)>(vf[i % (VLA + 1)]);
        u32x4_t v = vf[i % (VLA + 1)];
        if constexpr (decltype(mask_t)::value) {
          const int left = nk - (k0 + 32 * h + 16 * s + 4 * lg);   // of the 4 keys of v[0..1]; v[2..3]: 8 on
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int l = left - (e < 2 ? 2 * e : 8 + 2 * (e - 2));
            v[e] = l >= 2 ? v[e] : l == 1 ? v[e] & 0xFFFFu : 0u;
          }
        }
        Mma<bf16_t>::run(O[d], v, P[h][s]);
        if constexpr (i + VLA < A::NSB) vf[(i + VLA) % (VLA + 1)] = vfrag(std::integral_constant<int, i + VLA>{});
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    if (k0 + BK > nk) pv(std::true_type{});
    else pv(std::false_type{});
    if constexpr (QG == 1) {
      fence();   // the last read of the values has returned
      if (next) load_all(nb, 0, std::true_type{});
    }
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
  using S0_ = std::integral_constant<int, 0>;
  using S1_ = std::integral_constant<int, 1>;
  if (jb + grp < NB) {
    const Block bl = block(jb + grp);
    load_all(bl, 0, std::false_type{});
    load_all(bl, 0, std::true_type{});
  }
  if constexpr (QG == 1) {
    for (int j = jb + grp; j < NB; j += KS) step(j, S0_{});
  } else {
    for (int j = jb; j < NB; j += 2) {
      step(j, S0_{});
      if (j + 1 < NB) step(j + 1, S1_{});
    }
  }
  __syncthreads();   // the rings are free for the merge

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
  const int rows = min(A::TM, Rall - m0), d0 = tid % TPR * 8;
  const PartRows pr{(int64_t)p.B * p.Hk * R};
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
    const int ob = KIND == PREFIX ? (m0 + r) / R : b, om = KIND == PREFIX ? (m0 + r) % R : m0 + r;
    if (KIND == WHOLE && slots == 0) {
      const int i = om / G;
      store_row(p, ob, hk * G + om % G, i, d0, o, L, p.P > 0 || own_seen(p, len, i) > 0);
    } else {
      const int64_t row = (int64_t)(ob * p.Hk + hk) * R + om;
      if constexpr (JOIN) {   // the partial results take at most 1 GiB
        const f32x4_t x = {o[0], o[1], o[2], o[3]}, y = {o[4], o[5], o[6], o[7]};
        const uint32_t at = (uint32_t)(slot * pr.rows + row);
        coherent_store16(p.ws, at * (D * 4) + d0 * 4, __builtin_bit_cast(u32x4_t, x));
        coherent_store16(p.ws, at * (D * 4) + d0 * 4 + 16, __builtin_bit_cast(u32x4_t, y));
        if (d0 == 0)
          coherent_store8(p.ws, (uint32_t)(slots * pr.rows) * (D * 4) + at * 8, u32x2_t{__float_as_uint(M), __float_as_uint(L)});
      } else {
        float* dst = pr.o(p, slot, row) + d0;
        *reinterpret_cast<f32x4_t*>(dst) = f32x4_t{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<f32x4_t*>(dst + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
        if (d0 == 0) {
          float* to = pr.ml(p, slots, slot, row);
          to[0] = M;
          to[1] = L;
        }
      }
    }
  }
  if constexpr (JOIN) {
    static_assert(KIND == WHOLE && QG == 1, "the parts of one (sequence, key head)");
    // Count the arrival; the last workgroup joins.
    wait_vmcnt<0>();          // this wave's partial results are written
    __syncthreads();          // ... and every wave's; the LDS is free
    int* const last = reinterpret_cast<int*>(smem + 16384);   // behind what join_rows uses
    if (tid == 0) {
      unsigned* const c = count + hk * p.B + b;
      *last = atomicInc(c, (unsigned)(slots - 1)) == (unsigned)(slots - 1);   // the last one wraps it to 0
    }
    __syncthreads();
    if (*last) {   // R <= 32
      if (R <= kJoinFew) join_rows<D, kJoinFew>(p, smem, b, hk, slots);
      else join_rows<D, 32>(p, smem, b, hk, slots);
    }
  }
}

// Workgroup L of T runs on XCD L % 8; an XCD takes a contiguous range of tasks, so that
// neighbouring ones share keys in its L2.
__device__ __forceinline__ int xcd_task(int L, int T) {
  const int x = L & 7, q = T >> 3, r = T & 7;
  return x * q + min(x, r) + (L >> 3);
}

// One launch over (key head, sequence, part, row block).  Later row blocks first: with
// causal they see more keys.
// parts > 1: partial results, joined here (JOIN) or by prefix_merge_kernel.
template <int D, int QG, bool JOIN>
__global__ __launch_bounds__(256, 2) void prefix_whole_kernel(PrefixParams p, int nrb, int parts, unsigned* count) {
  __shared__ __attribute__((aligned(16))) char smem[PrefixShape<D, QG>::LDS];
  int t = xcd_task(blockIdx.x, gridDim.x);
  const int rb = nrb - 1 - t % nrb;
  t /= nrb;
  const int z = t % parts;
  t /= parts;
  attend<WHOLE, D, QG, JOIN>(p, smem, rb, t % p.B, t / p.B, z, parts, z, parts > 1 ? parts : 0, count);
}

// The parts of the prefix, (key head, part, row block over all sequences), then those of the own
// keys, (key head, sequence, part, row block).  The prefix's, bound by the MFMAs, run beside the
// own keys', which memory bounds.
template <int D, int PQ, int OQ>
__global__ __launch_bounds__(256, 2) void prefix_split_kernel(PrefixParams p, int tp, int nrb_p, int np, int nrb_o, int ns) {
  __shared__ __attribute__((aligned(16)))
  char smem[PrefixShape<D, PQ>::LDS > PrefixShape<D, OQ>::LDS ? PrefixShape<D, PQ>::LDS : PrefixShape<D, OQ>::LDS];
  if ((int)blockIdx.x < tp) {
    int t = xcd_task(blockIdx.x, tp);
    const int rb = t % nrb_p;
    t /= nrb_p;
    attend<PREFIX, D, PQ, false>(p, smem, rb, 0, t / np, t % np, np, t % np, np + ns, nullptr);
  } else {
    int t = xcd_task(blockIdx.x - tp, gridDim.x - tp);
    const int rb = nrb_o - 1 - t % nrb_o;
    t /= nrb_o;
    const int z = t % ns;
    t /= ns;
    attend<OWN, D, OQ, false>(p, smem, rb, t % p.B, t / p.B, z, ns, np + z, np + ns, nullptr);
  }
}

// The parts of every row: D / 8 threads for 8 d each, times WAYS that take the parts in
// turn and join in LDS, so that few trips to memory follow one another.
template <int D, int WAYS>
__global__ __launch_bounds__(256) void prefix_merge_kernel(PrefixParams p, int slots) {
  constexpr int TPR = D / 8, ROWS = 256 / TPR / WAYS;
  __shared__ __attribute__((aligned(16))) float so[WAYS][ROWS][D];
  __shared__ float sml[WAYS][ROWS][2];
  const int G = p.H / p.Hk, R = G * p.Lq;
  const int rows = p.B * p.Hk * R;              // at most 2^30
  const PartRows pr{rows};
  const int way = threadIdx.x / TPR % WAYS, r = threadIdx.x / TPR / WAYS, d0 = threadIdx.x % TPR * 8;
  const int row = min((int)blockIdx.x * ROWS + r, rows - 1);
  const float* const o0 = pr.o(p, 0, row) + d0;
  const float* const ml0 = pr.ml(p, slots, 0, row);
  const int m = row % R, bh = row / R, hk = bh % p.Hk, b = bh / p.Hk, i = m / G;
  const bool any = p.P > 0 || own_seen(p, own_len(p, b), i) > 0;
  float M = -INFINITY, L = 0.0f, o[8] = {};
  auto join = [&](float mz, float lz, const f32x4_t& x, const f32x4_t& y) {
    const float mn = fmaxf(M, mz);
    const float fo = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M - mn);
    const float fz = mz == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mz - mn);
    M = mn;
    L = fmaf(fz, lz, fo * L);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = fmaf(fz, x[e], fo * o[e]);
      o[4 + e] = fmaf(fz, y[e], fo * o[4 + e]);
    }
  };
  for (int s0 = way; s0 < slots; s0 += 4 * WAYS) {   // four parts' loads in flight
    f32x4_t x[4], y[4];
    float mz[4], lz[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t s = min(s0 + q * WAYS, slots - 1);
      x[q] = *reinterpret_cast<const f32x4_t*>(o0 + s * rows * D);
      y[q] = *reinterpret_cast<const f32x4_t*>(o0 + s * rows * D + 4);
      mz[q] = ml0[s * rows * 2];
      lz[q] = ml0[s * rows * 2 + 1];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (s0 + q * WAYS < slots) join(mz[q], lz[q], x[q], y[q]);
  }
  if constexpr (WAYS > 1) {
    *reinterpret_cast<f32x4_t*>(&so[way][r][d0]) = f32x4_t{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4_t*>(&so[way][r][d0 + 4]) = f32x4_t{o[4], o[5], o[6], o[7]};
    if (d0 == 0) {
      sml[way][r][0] = M;
      sml[way][r][1] = L;
    }
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int w = 1; w < WAYS; ++w)
      join(sml[w][r][0], sml[w][r][1], *reinterpret_cast<const f32x4_t*>(&so[w][r][d0]),
           *reinterpret_cast<const f32x4_t*>(&so[w][r][d0 + 4]));
  }
  if ((int)blockIdx.x * ROWS + r < rows) store_row(p, b, hk * G + m % G, i, d0, o, L, any);
}

// ---------------------------------------------------------------------------
// How a call is cut: whole rows in one launch, in np parts of their keys and a
// second launch that joins them, or split into prefix parts and own parts.
// ---------------------------------------------------------------------------
struct PrefixPlan {
  int pq, oq;   // 32-row waves of a workgroup: prefix parts, own parts or whole rows
  int np, ns;   // split: parts of the prefix and of the own keys.  ns = 0: whole rows in np parts
  bool few;     // at most 32 rows of a (sequence, key head)
  int slots() const { return ns > 0 ? np + ns : np > 1 ? np : 0; }
  bool joined() const { return ns == 0 && np > 1 && few; }   // by the last workgroup, without a second launch
  int ways() const { return slots() <= 4 ? 1 : slots() <= 16 ? 4 : 8; }   // of the second launch
};
constexpr size_t kCounterBytes = CF_PREFIX_WS_HEADER_BYTES;   // the counters of (sequence, key head); the partial results follow
constexpr int kCUs = 256, kMaxParts = 32, kMaxOwnParts = 8;
static_assert(2 * kPrefixMaxKeys / std::min(PrefixShape<128, 1>::BK, PrefixShape<128, 4>::BK) * kMaxParts <= UINT32_MAX,
              "a part's first block is computed in 32 bits (attend)");

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t row_blocks(int64_t rows, int qg) { return ceil_div(rows, 32 * qg); }

// The estimate (us).  A step is one key block of every group of a workgroup: alone on its CU,
// and where two workgroups share the CU; a workgroup's start and merge; the join, and
// a partial result's write and read.  Fitted to 400 calls of 1 to 64 sequences, 1 to 500 queries and
// 64 to 16000 prefix keys, each measured in up to 80 cuts, at the time that a caller in Python sees (a second
// launch costs the host 4 us): the cut that the estimate takes is 2 % slower than the best one on
// average, 25 % at worst; with powers of two only 3 %, with 128 rows a workgroup for all calls
// of more than 32 rows 4 %.  Some of them (us, launched from C: whole rows in one part; the best split;
// what the estimate takes, where that is another):
//     4 x 8 heads, 1 query, 128 + 64 keys, d 64                5.6     8.0
//     64 x 8 heads, 1 query, 512 + 128, d 64                   9.8    11.9
//     16 x 16 heads, 5 queries, 4095 + 333, d 64              24.1    14.4 (4 + 1 parts)
//     1 x 32 heads of 8, 1 query, 8192 + 512, d 128           61.7    12.9 (16 + 2)   16.5 (whole rows in 32 parts)
//     64 x 32 heads of 8, 1 query, 8192 + 512, d 128           117    40.2 (16 + 1)
constexpr double kStepFew = 0.95, kStepFew2 = 1.88, kStepMany = 1.35, kStepMany2 = 2.13;   // QG 1, QG 4; 2: two a CU
constexpr double kStepMany64 = 0.59;              // QG 4 steps at d = 64 by those at d = 128
constexpr double kStart = 6.5, kPartial = 1.8e-6, kStream = 5.8e6;   // kStream: bytes a us
constexpr double kJoin = 4.8;                     // the joining launch, on the device and on the host
constexpr double kJoinBy8 = 1.44, kJoinOwn = 1.5; // joined by the last workgroup: every 8 rows, and besides
constexpr double kUneven = 1.3;                   // what workgroups of two kinds leave unused

struct Task {   // one kind of workgroup of a launch
  double steps, wgs;
  int qg;
  double us(bool shared) const {
    return steps * (qg == 1 ? (shared ? kStepFew2 : kStepFew) : (shared ? kStepMany2 : kStepMany)) + kStart;
  }
};

// Calls f with the numbers of parts from 1 to `most` that are tried: powers of two, and `fill` and
// `fill2` (those that just occupy the CUs once and twice).
template <typename F>
void try_parts(int64_t most, int64_t fill, int64_t fill2, F&& f) {
  for (int64_t n = 1; n <= most; n *= 2) f((int)n);
  for (int64_t n : {fill, fill2})
    if (n >= 3 && n <= most && (n & (n - 1)) != 0) f((int)n);
}

PrefixPlan make_plan(const PrefixParams& p) {
  const int64_t R = (int64_t)(p.H / p.Hk) * p.Lq, Rall = p.B * R, rows = p.Hk * Rall;
  PrefixPlan best{1, R <= 32 ? 1 : 4, 1, 0, R <= 32};
  auto blocks = [&](int64_t n, int qg) { return ceil_div(n, qg == 1 ? 4096 / p.d : 64); };   // of keys
  auto task = [&](int64_t nb, int parts, int64_t wgs, int qg) {
    const double scale = qg == 4 && p.d == 64 ? kStepMany64 : 1.0;
    return Task{(double)ceil_div(ceil_div(nb, parts), 4 / qg) * scale, (double)wgs * parts, qg};
  };
  const double stream = 4.0 * p.Hk * p.d * (p.P + 0.8 * p.B * p.S) / kStream;
  const double part = kPartial * (double)rows * p.d;
  const int64_t gib = ((int64_t)1 << 30) / std::max<int64_t>(1, rows * (p.d + 2) * 4);   // parts in 1 GiB
  double least = 0;
  auto take = [&](double us, int pq, int oq, int np, int ns) {
    if (least == 0 || us < least) {
      least = us;
      best.pq = pq;
      best.oq = oq;
      best.np = np;
      best.ns = ns;
    }
  };
  // 32 or 128 rows a workgroup: up to 96 rows of a (sequence, key head) three of 32 may waste less than one of 128
  for (int oq : {1, 4}) {
    if (oq == 1 ? R > 96 : R <= 32) continue;
    const int64_t wo = row_blocks(R, oq) * p.B * p.Hk, bw = blocks(p.P, oq) + blocks(p.S, oq);
    try_parts(std::max<int64_t>(1, std::min({(int64_t)kMaxParts, ((int64_t)p.P + p.S) / 64, gib})), kCUs / wo, 2 * kCUs / wo,
              [&](int n) {
                const Task t = task(bw, n, wo, oq);
                const double us = t.wgs <= kCUs ? t.us(false) : std::ceil(t.wgs / (2 * kCUs)) * t.us(true);
                const double join = best.few ? kJoinOwn + kJoinBy8 * (double)ceil_div(R, 8) : kJoin;
                take(std::max(us, stream) + (n > 1 ? join + n * part : 0.0), 1, oq, n, 0);
              });
    // whole rows of full workgroups on every CU: nothing to gain from parts
    if (p.P == 0 || p.S == 0 || (R >= 64 && wo >= kCUs)) continue;
    // 32 rows a workgroup for the prefix read it more often, but start sooner: also where there are more rows
    for (int pq : {1, 4}) {
      if (pq == 4 ? Rall <= 32 : oq == 4) continue;
      const int64_t bp = blocks(p.P, pq), bo = blocks(p.S, oq), wp = row_blocks(Rall, pq) * p.Hk;
      for (int m = 1; m <= kMaxOwnParts && (m == 1 || (int64_t)m * 64 <= p.S) && m < gib; m *= 2)
        try_parts(std::max<int64_t>(1, std::min({(int64_t)kMaxParts, (int64_t)p.P / 64, gib - m})), (kCUs - wo * m) / wp,
                  (2 * kCUs - wo * m) / wp, [&](int n) {
                    const Task a = task(bp, n, wp, pq), b = task(bo, m, wo, oq);
                    const bool shared = a.wgs + b.wgs > kCUs;
                    const double ua = a.us(shared), ub = b.us(shared);
                    const double us = std::max({ua, ub, kUneven * (a.wgs * ua + b.wgs * ub) / (2 * kCUs)});
                    take(std::max(us, stream) + kJoin + (n + m) * part, pq, oq, n, m);
                  });
    }
  }
  return best;
}

template <int D, int QG, bool JOIN>
hipError_t launch_whole(const PrefixParams& p, int parts, unsigned* count, hipStream_t st) {
  const int64_t R = (int64_t)(p.H / p.Hk) * p.Lq, nrb = row_blocks(R, QG), wgs = nrb * parts * p.Hk * p.B;
  hipLaunchKernelGGL((prefix_whole_kernel<D, QG, JOIN>), dim3((unsigned)wgs), dim3(256), 0, st, p, (int)nrb, parts, count);
  return hipGetLastError();
}

template <int D, int PQ, int OQ>
hipError_t launch_split(const PrefixParams& p, const PrefixPlan& pl, hipStream_t st) {
  const int64_t R = (int64_t)(p.H / p.Hk) * p.Lq, nrb_p = row_blocks(p.B * R, PQ), nrb_o = row_blocks(R, OQ);
  const int64_t tp = nrb_p * pl.np * p.Hk, to = nrb_o * pl.ns * p.Hk * p.B;
  hipLaunchKernelGGL((prefix_split_kernel<D, PQ, OQ>), dim3((unsigned)(tp + to)), dim3(256), 0, st, p, (int)tp, (int)nrb_p,
                     pl.np, (int)nrb_o, pl.ns);
  return hipGetLastError();
}

template <int D, int WAYS>
hipError_t launch_merge(const PrefixParams& p, int slots, hipStream_t st) {
  const int64_t rows = (int64_t)p.B * p.H * p.Lq, per = 256 / (D / 8) / WAYS;
  hipLaunchKernelGGL((prefix_merge_kernel<D, WAYS>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, p, slots);
  return hipGetLastError();
}

template <int D>
hipError_t launch_all(PrefixParams p, const PrefixPlan& pl, hipStream_t st) {
  unsigned* const count = reinterpret_cast<unsigned*>(p.ws);
  if (pl.slots() > 0) p.ws += kCounterBytes / 4;
  if (pl.joined()) return launch_whole<D, 1, true>(p, pl.np, count, st);
  hipError_t e;
  if (pl.ns == 0) e = pl.oq == 1 ? launch_whole<D, 1, false>(p, pl.np, nullptr, st) : launch_whole<D, 4, false>(p, pl.np, nullptr, st);
  else if (pl.pq == 1) e = launch_split<D, 1, 1>(p, pl, st);
  else e = pl.oq == 1 ? launch_split<D, 4, 1>(p, pl, st) : launch_split<D, 4, 4>(p, pl, st);
  if (e != hipSuccess || pl.slots() == 0) return e;
  return pl.ways() == 1 ? launch_merge<D, 1>(p, pl.slots(), st)
                        : pl.ways() == 4 ? launch_merge<D, 4>(p, pl.slots(), st) : launch_merge<D, 8>(p, pl.slots(), st);
}

}  // namespace

size_t prefix_workspace(const PrefixParams& p) {
  const int slots = make_plan(p).slots();
  if (slots == 0) return 0;
  return kCounterBytes + (size_t)slots * (size_t)p.B * (size_t)p.H * (size_t)p.Lq * (size_t)(p.d + 2) * 4;
}

hipError_t launch_prefix(const PrefixParams& p, hipStream_t st) {
  const PrefixPlan pl = make_plan(p);
  return p.d == 128 ? launch_all<128>(p, pl, st) : launch_all<64>(p, pl, st);
}

void prefix_form(const PrefixParams& p, char* text, size_t bytes) {
  const PrefixPlan pl = make_plan(p);
  int n = pl.ns > 0 ? snprintf(text, bytes, "split, %d + %d rows, %d + %d parts", 32 * pl.pq, 32 * pl.oq, pl.np, pl.ns)
                    : snprintf(text, bytes, "whole, %d rows, %d parts", 32 * pl.oq, pl.np);
  if (pl.joined())
    snprintf(text + n, bytes - n, ", joined by %d", (int64_t)(p.H / p.Hk) * p.Lq <= kJoinFew ? kJoinFew : 32);
  else if (pl.slots() > 0)
    snprintf(text + n, bytes - n, ", merged %d ways", pl.ways());
}

}  // namespace cf
