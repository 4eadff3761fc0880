// Attention of each sequence's last tokens over its pages:
//     O_b = softmax(cap(scale Q_b K_b^T)) V_b.
//
// Rows.  The queries of one (sequence, key head) are G Lq rows, row i G + g being query i of
// head g, in blocks of 16 RT rows.  The keys of a block are cut into parts, a workgroup each; its four
// waves take 32 keys in turn and keep running maxima and sums of their own, which meet in LDS; the
// parts' results meet in the workspace, where the workgroup that finishes a block last joins them.
//
// Products, on 16 x 16 x 32 MFMAs with no LDS: S^T = K Q^T takes a lane's 16-byte pieces of 16 key
// rows as they lie in a page, so a lane holds one query row c = lane % 16 and keys 4 q + i, q = lane / 16, of
// each 16.  That is the layout in which O^T = V^T P^T takes P^T, with k = 8 q + j standing for key
// 4 q + j (j < 4) and 16 + 4 q + j - 4.  V^T of 16 dimensions needs one dimension of those 8 keys: a lane loads
// D / 16 neighbouring ones of each (16 lanes a whole row), and picking the t-th of each, in the step that makes
// bf16 of the codes, gives the operand for dimensions t, t + D / 16, ...: the transposition costs nothing.
//
// P, times the scale of the value, is rounded to bf16, the type in which the MFMA takes it beside V's exact codes: off by 2^-9 of
// a weight, while the output is rounded to bf16 as well.  Against 64 bits the result is off by 0.0021 to 0.0024 in relative norm,
// 0.0017 of which is the output's rounding.  The sum of the weights is taken before it, in fp32, as maxima and O are.
//
// Bound.  bf16: memory, 6.05 TB/s where the cache is larger than the last-level one (a streaming read with no work
// reaches 6.9).  int8: the conversion of the codes, 3 vector operations for two, with the softmax; three waves a SIMD
// keep 5.3 TB/s (64 sequences of up to 8192 keys, 8 key heads of 4, 832 MB: 156 us).  Several queries and capped scores: the
// softmax (16 sequences of 4 key heads of 4, 5 queries, 4095 E4M3 keys of 64: 15.8 us).  One sequence: its start, the
// parts' way through the workspace and the launch (4096 bf16 keys, 8 key heads of 4: 10.0 us).  More than 32 rows a key head:
// every 32 read and convert the keys and values again.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "cf_attn.h"
#include "cf_gemm_tile.h"
#include "cf_serving.h"
#include "comfuse.h"

namespace cf {

namespace {

constexpr int kWaves = 4, kStepKeys = 32;

// Keys that query i of sequence b sees.
__device__ __forceinline__ int paged_len(const PagedParams& p, int b) {
  return (int)min((int64_t)max(p.lens[b], 0), (int64_t)p.pages << p.c.shift);
}
__device__ __forceinline__ int paged_seen(const PagedParams& p, int len, int i) {
  return p.causal ? max(0, len - (p.Lq - 1 - i)) : len;
}

__device__ __forceinline__ float quad_max(float v) {   // over the lanes c, c + 16, c + 32, c + 48
#if defined(__HIP_DEVICE_COMPILE__)
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
#endif
  return v;
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Two neighbouring codes (bytes 2 h, 2 h + 1 of w) as bf16: exact for int8 and for E4M3.
template <int CODE, int H>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w) {
  if constexpr (CODE == CACHE_I8) {
    return pack_bf16x2((float)(int8_t)(w >> (16 * H)), (float)(int8_t)(w >> (16 * H + 8)));
  } else {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, H != 0));
#else
    return 0;
#endif
  }
}

template <int D, int CODE, int RT>
struct PagedShape {
  static constexpr int DT = D / 16, KS = D / 32;            // 16-wide blocks of d, MFMA steps over d
  static constexpr int E = CODE == CACHE_BF16 ? 2 : 1;      // bytes of an element
  static constexpr int KL = D * E / 64, VW = D * E / 64;    // 16-byte loads of a key tile; words of a value row, of a lane
  static constexpr int ROWS = 16 * RT, PITCH = D + 4;       // merge: floats of a row
  static constexpr int LDS = kWaves * ROWS * PITCH * 4;
};

// 8 d of an output row.
__device__ __forceinline__ void paged_store(const PagedParams& p, int b, int h, int i, int d0, const float (&o)[8], float l) {
  const float inv = 1.0f / l;
  u32x4_t w = {pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv), pack_bf16x2(o[4] * inv, o[5] * inv),
               pack_bf16x2(o[6] * inv, o[7] * inv)};
  if (l == 0.0f) w = u32x4_t{};   // no key
  *reinterpret_cast<u32x4_t*>(p.O + b * p.o_b + h * p.o_h + i * p.o_l + d0) = w;
}

struct Joined {   // running join of parts: maximum, sum, 8 d
  float M = kLowestF32, L = 0.0f, o[8] = {};
  __device__ __forceinline__ void add(float m, float l, const float* x) {
    const float mn = fmaxf(M, m), fo = __builtin_amdgcn_exp2f(M - mn), fz = __builtin_amdgcn_exp2f(m - mn);
    M = mn;
    L = fmaf(fz, l, fo * L);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(fz, x[e], fo * o[e]);
  }
};

// The parts that a block of `steps` steps of 32 keys is cut into, of `most` that are launched.  They go by the length: a table,
// above all in a captured call, may be far wider than its sequences.  One part more shortens the way over the keys and lengthens
// the join's, so the best number goes with the root of the keys, and is less where a partial result has more rows.  Of these,
// as few as leave the longest wave its steps; where there are more than give every CU a workgroup (`each_cu`), a multiple of
// that, for 0.8 of the root.  Up to kOneSteps the way through the workspace, 1 to 3 us, costs more than it gives.  Found with
// 110 calls (1 to 16 sequences, 150 to 8000 keys) under tables of 65536 keys, in 1 to 32 parts each: in 0.84 of the time that
// parts of 128 keys and more take, half of it at best; 240 random calls whose tables are at most twice as wide as needed take
// 0.94 of it, 1.11 at worst.  For instance (us; parts 1, 2, 4, 8, 16, 32):
//     4 x 8 key heads of 4 heads, 350 keys, bf16, d 128       7.8  8.0  7.2  8.1  8.1  8.2
//     8 x 8 of 4, 700 keys, int8, d 64                        9.6  9.3  8.9  9.5   12   12
//     1 x 8 of 4, 6 queries, 2500 keys, bf16, d 128            38   25   17   15   17   24
//     1 x 8 of 4, 8000 keys, E4M3, d 64                        54   33   20   13   11   11
template <int D>
constexpr int kOneSteps = D == 128 ? 14 : 18;
template <int D, int RT>
__device__ __forceinline__ int parts_of(int steps, int most, float each_cu) {
  if (steps <= kOneSteps<D>) return 1;
  auto whole = [](float x) { return __builtin_amdgcn_readfirstlane((int)x); };
  const float root = __builtin_amdgcn_sqrtf((float)steps * (2.0f / RT));
  const int n = max(1, min(most, whole(root)));
  if ((float)n > each_cu) {
    const int times = max(1, whole(root * 0.8f * __builtin_amdgcn_rcpf(each_cu)));
    return max(1, min(most, whole((float)times * each_cu + 0.01f)));
  }
  const int each = whole((float)(steps - 1) * __builtin_amdgcn_rcpf((float)(n * kWaves))) + 1;   // steps of the longest wave
  return min(n, whole((float)(steps - 1) * __builtin_amdgcn_rcpf((float)(each * kWaves))) + 1);
}

// Bytes of the keys and values in use from which their lines are not kept: the last-level cache has 256 MB, and a call over
// more finds little of it there next time (215 MB: 48.3 -> 46.3 us so; 98 MB in it: 19.8 -> 20.7).  A table may be far wider
// than its sequences, so a workgroup decides by its own length, as if all were as long.
constexpr int64_t kOnceBytes = 192 << 20;
__host__ __device__ constexpr bool read_past(int64_t keys, int Hk, int d, bool bf16) {
  return keys * Hk > kOnceBytes / (2 * (bf16 ? 2 * d : d + 4));
}

// MIXED: rows of a block may see different keys, and a value may be infinite or NaN (a check and products of their own for
// such a step; kept out of other calls, which the longer code would cost up to 5 %).
// ONCE: the table has room for so many keys that they may be read past the caches.
// FAR: a cap beyond kNearCap.  1 - 2 / (1 + exp 2 z) is tanh z but for an ulp or two of 1, so a capped score is off by as much of
// the cap, which up to kNearCap is below its own error.  Beyond, where |z| is below 1 / 4 the score is z's odd series up to z^7
// (the next term: 2^-21 of it).  In a kernel of its own: its code beside the other cost short calls 4 %.
constexpr float kNearCap = 64.0f;
template <int D, int CODE, int RT, bool ONCE, bool MIXED, bool FAR>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_kernel(PagedParams p, int nrb, int parts, int turn, float each_cu, unsigned* count) {
  using A = PagedShape<D, CODE, RT>;
  __shared__ __attribute__((aligned(16))) char smem[A::LDS];
  __shared__ int last_one;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, q = lane >> 4;
  // Parts go slowest through the grid: a sequence may have fewer than are launched, and those in use then lie beside each other,
  // on all XCDs (parts beside each other: 4 sequences of 1000 int8 keys, 32 heads of 8, under a wide table 9.1 -> 10.3 us).  Each
  // part begins with other sequences (`turn`), or a CU would have the parts of one (8 x 32 heads of 8, 7759 to 14909 int8 keys
  // 46 -> 40 us).
  int task = blockIdx.x;
  const int rb = task % nrb;
  task /= nrb;
  const int hk = task % p.Hk;
  task /= p.Hk;
  const int z = task / p.B;
  int b = task % p.B + z * turn;
  if (b >= p.B) b -= p.B;
  const int G = p.H / p.Hk, R = G * p.Lq, m0 = rb * A::ROWS;

  // Q fragments (on their way while the length is looked up).  16-byte pieces of a row of codes hold two steps' d of a lane.
  u32x4_t qf[RT][A::KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int m = min(m0 + 16 * rt + c, R - 1), i = m / G;
    const bf16_t* src = p.Q + b * p.q_b + (hk * G + m % G) * p.q_h + i * p.q_l;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks)
      qf[rt][ks] = gload16(src + (CODE == CACHE_BF16 ? ks * 32 + q * 8 : (ks >> 1) * 64 + q * 16 + (ks & 1) * 8));
  }

  const int len = paged_len(p, b);
  const int last = paged_seen(p, len, (min(m0 + A::ROWS, R) - 1) / G);   // keys that some row sees
  const int first = paged_seen(p, len, m0 / G);                          // ... that every row sees
  const int steps = (last + kStepKeys - 1) / kStepKeys;
  const int np = parts_of<D, RT>(steps, parts, each_cu);                          // parts of this block in use
  if (z >= np) return;
  const int j0 = (int)((uint32_t)steps * z / np), j1 = (int)((uint32_t)steps * (z + 1) / np);   // (steps <= 2^25, np <= 64)
  int seen[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) seen[rt] = paged_seen(p, len, min(m0 + 16 * rt + c, R - 1) / G);

  f32x4_t O[RT][A::DT] = {};
  float M[RT], L[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    M[rt] = kLowestF32;
    L[rt] = 0.0f;
  }
  const float cap = p.softcap, sl = (cap > 0.0f && !FAR ? 2.0f * p.scale / cap : p.scale) * 1.4426950408889634f;
  const float cap2 = cap * 1.4426950408889634f;

  // The pages of a step's two tiles (one where pages hold 32 tokens and more).  Their entries are asked for a step
  // before they are used, by scalar loads: they are the wave's.
  typedef const __attribute__((address_space(4))) int32_t* Table;
  const Table table = (Table)(uintptr_t)(p.table + b * p.ldt);
  const bool wide = p.c.shift > 4;
  struct Pages {
    int at[2];
  };
  auto look_up = [&](int j) {   // (any entry in use for a step behind the last)
    const int key = min(j, j1 - 1) * kStepKeys, e = table[key >> p.c.shift];
    return Pages{{e, wide ? e : table[min(key + 16, last - 1) >> 4]}};
  };
  auto resolve = [&](int j, Pages e) {   // -1: behind the last key, or an entry that names no page
    const int key = j * kStepKeys;
    const bool in = j < j1;
    return Pages{{in && (uint32_t)e.at[0] < (uint32_t)p.c.n_pages ? e.at[0] : -1,
                  in && key + 16 < last && (uint32_t)e.at[1] < (uint32_t)p.c.n_pages ? e.at[1] : -1}};
  };
  // A tile is read through a buffer that ends behind the last key that some row sees (of no bytes where there is no
  // page): what lies there comes back as 0, whatever it holds.  A step behind the last reads nothing, so that no branch hides
  // how many loads are under way.
  u32x4_t kf[2][A::KL];
  uint32_t vf[8][A::VW];
  f32x4_t ksc[2], vsc[2];
  [[maybe_unused]] const uint32_t klane = c * (uint32_t)p.c.k_l + q * 16;
  uint32_t vlane[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) vlane[i] = (4 * q + i) * (uint32_t)p.c.v_l + c * A::VW * 4;
#if defined(__HIP_DEVICE_COMPILE__)
  auto buffer = [](const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
  };
  // Byte offsets of a step's tiles: the page stride is below 2^32 bytes, a page's rows lie within 2^31.
  auto tiles = [&](int key, Pages pg, uint32_t page, uint32_t row, uint64_t (&at)[2]) {
    at[0] = (uint64_t)(uint32_t)pg.at[0] * page + ((uint32_t)key & ((1u << p.c.shift) - 1)) * row;
    at[1] = wide ? at[0] + 16 * row : (uint64_t)(uint32_t)pg.at[1] * page;
  };
  const char* const kbase = p.c.K + hk * p.c.k_h;
  const char* const vbase = p.c.V + hk * p.c.v_h;
  const char* const ksbase = reinterpret_cast<const char*>(p.c.Ks + hk * p.c.ks_h);
  const char* const vsbase = reinterpret_cast<const char*>(p.c.Vs + hk * p.c.vs_h);
#endif
  auto load_k = [&](int j, Pages pg, auto hint_t) {
    [[maybe_unused]] constexpr int kHint = decltype(hint_t)::value;
#if defined(__HIP_DEVICE_COMPILE__)
    const int key = j * kStepKeys;
    uint64_t at[2];
    tiles(key, pg, (uint32_t)p.c.k_p, (uint32_t)p.c.k_l, at);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const auto src = buffer(kbase + at[t], pg.at[t] < 0 ? 0 : min(16, last - key - 16 * t) * (uint32_t)p.c.k_l);
#pragma unroll
      for (int x = 0; x < A::KL; ++x)
        kf[t][x] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(src, klane + x * 64, 0, kHint));
    }
    if constexpr (CODE != CACHE_BF16) {
      tiles(key, pg, (uint32_t)p.c.ks_p * 4, 4, at);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        ksc[t] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer(ksbase + at[t], pg.at[t] < 0 ? 0 : 64), q * 16, 0, 0));
    }
#endif
  };
  auto load_v = [&](int j, Pages pg, auto hint_t) {
    [[maybe_unused]] constexpr int kHint = decltype(hint_t)::value;
#if defined(__HIP_DEVICE_COMPILE__)
    const int key = j * kStepKeys;
    uint64_t at[2];
    tiles(key, pg, (uint32_t)p.c.v_p, (uint32_t)p.c.v_l, at);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const auto src = buffer(vbase + at[t], pg.at[t] < 0 ? 0 : min(16, last - key - 16 * t) * (uint32_t)p.c.v_l);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (A::VW == 4) {
          const u32x4_t w = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(src, vlane[i], 0, kHint));
#pragma unroll
          for (int x = 0; x < 4; ++x) vf[4 * t + i][x] = w[x];
        } else if constexpr (A::VW == 2) {
          const u32x2_t w = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(src, vlane[i], 0, kHint));
          vf[4 * t + i][0] = w[0];
          vf[4 * t + i][1] = w[1];
        } else {
          vf[4 * t + i][0] = __builtin_amdgcn_raw_buffer_load_b32(src, vlane[i], 0, kHint);
        }
      }
    }
    if constexpr (CODE != CACHE_BF16) {
      tiles(key, pg, (uint32_t)p.c.vs_p * 4, 4, at);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        vsc[t] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer(vsbase + at[t], pg.at[t] < 0 ? 0 : 64), q * 16, 0, 0));
    }
#endif
  };

  // The way over the part's keys, a loop for each hint (branches around the loads: 64 x 8192 int8 keys 1 % slower, E4M3 4 %).
  auto walk = [&](auto hint) {
    Pages pages = {}, ahead = {};   // of the step whose rows are under way, and the entries of the one after it
    if (j0 + wave < j1) {
      pages = resolve(j0 + wave, look_up(j0 + wave));
      load_k(j0 + wave, pages, hint);
      load_v(j0 + wave, pages, hint);
      ahead = look_up(j0 + wave + kWaves);
    }
    for (int j = j0 + wave; j < j1; j += kWaves) {
      const int next = j + kWaves;
      const int k0 = j * kStepKeys;
      const bool bad0 = pages.at[0] < 0, bad1 = pages.at[1] < 0;
      const bool masked = k0 + kStepKeys > first || bad0 || bad1;
      pages = resolve(next, ahead);
      ahead = look_up(next + kWaves);
      // S^T, in log2 units; with a cap its 2 z first
      float s[RT][8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4_t a[A::KS];
#pragma unroll
        for (int ks = 0; ks < A::KS; ++ks) {
          if constexpr (CODE == CACHE_BF16) a[ks] = kf[t][ks];
          else {
            const uint32_t w0 = kf[t][ks >> 1][2 * (ks & 1)], w1 = kf[t][ks >> 1][2 * (ks & 1) + 1];
            a[ks] = u32x4_t{codes_bf16<CODE, 0>(w0), codes_bf16<CODE, 1>(w0), codes_bf16<CODE, 0>(w1), codes_bf16<CODE, 1>(w1)};
          }
        }
        f32x4_t sc = {sl, sl, sl, sl};
        if constexpr (CODE != CACHE_BF16)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[i] *= ksc[t][i];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          f32x4_t acc = {};
#pragma unroll
          for (int ks = 0; ks < A::KS; ++ks) acc = mfma16(a[ks], qf[rt][ks], acc);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[rt][4 * t + i] = acc[i] * sc[i];
        }
      }
      load_k(next, pages, hint);
      if (FAR) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float z2 = s[rt][e] * (2.0f / cap), y = z2 * z2 * 0.12011325347955035f;   // 2 z in log2 units, z^2
            const float series = s[rt][e] * fmaf(fmaf(fmaf(-17.0f / 315.0f, y, 2.0f / 15.0f), y, -1.0f / 3.0f), y, 1.0f);
            const float full = fmaf(-2.0f * cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z2)), cap2);
            s[rt][e] = y < 0.0625f ? series : full;
          }
      } else if (cap > 0.0f) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[rt][e] = fmaf(-2.0f * cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[rt][e])), cap2);
      }
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = k0 + 16 * (e >> 2) + 4 * q + (e & 3);
          const bool bad = e < 4 ? bad0 : bad1;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            if (bad || key >= seen[rt]) s[rt][e] = -INFINITY;
        }
      }
      u32x4_t pf[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float mx = s[rt][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[rt][e]);
        // The maximum is raised, and what was summed rescaled, only where a score passes it by 2^8.
        if (__any(mx > M[rt] + 8.0f)) {
          const float mn = fmaxf(M[rt], quad_max(mx)), f = __builtin_amdgcn_exp2f(M[rt] - mn);
          M[rt] = mn;
          L[rt] *= f;
#pragma unroll
          for (int d = 0; d < A::DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) O[rt][d][i] *= f;
        }
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = __builtin_amdgcn_exp2f(s[rt][e] - M[rt]);
          L[rt] += w[e];
          if constexpr (CODE != CACHE_BF16) {
            w[e] *= vsc[e >> 2][e & 3];
          }
        }
        if (CODE != CACHE_BF16 && masked)   // whatever the scale of a hidden row holds
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = s[rt][e] == -INFINITY ? 0.0f : w[e];
        pf[rt] = u32x4_t{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
      }
      // O^T += V^T P^T
      auto values = [&](int d) {
        u32x4_t a;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if constexpr (CODE == CACHE_I8) {
            a[x] = pack_bf16x2((float)(int8_t)(vf[2 * x][d / 4] >> (8 * (d % 4))), (float)(int8_t)(vf[2 * x + 1][d / 4] >> (8 * (d % 4))));
          } else if constexpr (CODE == CACHE_E4M3) {
            const uint32_t e0 = d % 4 / 2 ? codes_bf16<CODE, 1>(vf[2 * x][d / 4]) : codes_bf16<CODE, 0>(vf[2 * x][d / 4]);
            const uint32_t e1 = d % 4 / 2 ? codes_bf16<CODE, 1>(vf[2 * x + 1][d / 4]) : codes_bf16<CODE, 0>(vf[2 * x + 1][d / 4]);
            a[x] = __builtin_amdgcn_perm(e1, e0, d % 2 ? 0x07060302u : 0x05040100u);
          } else {
            a[x] = __builtin_amdgcn_perm(vf[2 * x + 1][d / 2], vf[2 * x][d / 2], d % 2 ? 0x07060302u : 0x05040100u);
          }
        }
        return a;
      };
      // MIXED: where rows of a step see different keys, an infinity or a NaN must not reach a row that does not see it (0 times
      // it would be NaN).  Such values are left out of the product; rows that see them are found by a product of ones.
      bool spoiled = false;
      if (MIXED && masked) {
        constexpr uint32_t kExp = CODE == CACHE_BF16 ? 0x7F807F80u : 0x7F7F7F7Fu, kOne = CODE == CACHE_BF16 ? 0x00800080u : 0x01010101u;
        uint32_t x = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int w = 0; w < A::VW; ++w) x |= (vf[i][w] & kExp) + kOne;
        spoiled = __any((x & (CODE == CACHE_BF16 ? 0x80008000u : 0x80808080u)) != 0);
      }
#pragma unroll
      for (int d = 0; d < A::DT; ++d) {
        u32x4_t a = values(d);
        if (MIXED && spoiled) {
          constexpr uint32_t kOnes = 0x3F803F80u;   // 1, 1
          u32x4_t up, down;                         // ones for + infinity and NaN, and for - infinity and NaN
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t all = ((((a[x] & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xFFFFu;   // not finite
            const uint32_t nan = ((((a[x] & 0x007F007Fu) + 0x007F007Fu) >> 7) & 0x00010001u) * 0xFFFFu;
            const uint32_t neg = ((a[x] >> 15) & 0x00010001u) * 0xFFFFu;
            up[x] = all & (nan | ~neg) & kOnes;
            down[x] = all & (nan | neg) & kOnes;
            a[x] &= ~all;
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            u32x4_t sees;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int key = k0 + 16 * (x >> 1) + 4 * q + 2 * (x & 1);
              sees[x] = (key < seen[rt] ? 0x00003F80u : 0u) | (key + 1 < seen[rt] ? 0x3F800000u : 0u);
            }
            const f32x4_t u = mfma16(up, sees, f32x4_t{}), n = mfma16(down, sees, f32x4_t{});
#pragma unroll
            for (int i = 0; i < 4; ++i) O[rt][d][i] += (u[i] > 0.0f ? INFINITY : 0.0f) + (n[i] > 0.0f ? -INFINITY : 0.0f);
          }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) O[rt][d] = mfma16(a, pf[rt], O[rt][d]);
      }
      load_v(next, pages, hint);
    }
  };
  if (ONCE && read_past((int64_t)p.B * len, p.Hk, D, CODE == CACHE_BF16)) walk(std::integral_constant<int, 2>{});
  else walk(std::integral_constant<int, 0>{});

  // The waves' results meet in LDS.  A lane holds d (4 q + i) D / 16 + t of row c: D / 4 neighbouring ones.
  float* const so = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float* mine = so + (wave * A::ROWS + 16 * rt + c) * A::PITCH;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < A::DT; d += 4)
        *reinterpret_cast<f32x4_t*>(mine + (4 * q + i) * A::DT + d) = f32x4_t{O[rt][d][i], O[rt][d + 1][i], O[rt][d + 2][i], O[rt][d + 3][i]};
    const float l = quad_sum(L[rt]);
    if (q == 0) {
      mine[D] = M[rt];
      mine[D + 1] = l;
    }
  }
  __syncthreads();
  constexpr int TPR = D / 8, RPP = 64 * kWaves / TPR;
  const int64_t rows = (int64_t)p.B * p.Hk * R;
  const int d0 = tid % TPR * 8;
  for (int r = tid / TPR; r < min(A::ROWS, R - m0); r += RPP) {
    Joined a;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float* other = so + (w * A::ROWS + r) * A::PITCH;
      a.add(other[D], other[D + 1], other + d0);
    }
    const int m = m0 + r;
    if (np == 1) {
      paged_store(p, b, hk * G + m % G, m / G, d0, a.o, a.L);
    } else {   // the partial results take less than 2^31 bytes
      const uint32_t at = (uint32_t)(z * rows + (int64_t)(b * p.Hk + hk) * R + m);
      const f32x4_t x = {a.o[0], a.o[1], a.o[2], a.o[3]}, y = {a.o[4], a.o[5], a.o[6], a.o[7]};
      coherent_store16(p.ws, at * (D * 4) + d0 * 4, __builtin_bit_cast(u32x4_t, x));
      coherent_store16(p.ws, at * (D * 4) + d0 * 4 + 16, __builtin_bit_cast(u32x4_t, y));
      if (d0 == 0)
        coherent_store8(p.ws, (uint32_t)(parts * rows) * (D * 4) + at * 8, u32x2_t{__float_as_uint(a.M), __float_as_uint(a.L)});
    }
  }
  if (np == 1) return;
  wait_vmcnt<0>();   // this wave's partial results are written
  __syncthreads();   // ... and every wave's
  if (tid == 0) {
    unsigned* const cnt = count + (b * p.Hk + hk) * nrb + rb;
    last_one = atomicInc(cnt, (unsigned)(np - 1)) == (unsigned)(np - 1);   // the last one wraps it to 0
  }
  __syncthreads();
  if (!last_one) return;
  // Join the block's rows: D / 8 threads a row; where there are few rows, others take the parts in turn.
  const int nr = min(A::ROWS, R - m0);
  int rs = 1;   // rows beside each other
  while (rs < nr && rs < RPP) rs *= 2;
  const int ways = RPP / rs, way = tid / TPR / rs;
  for (int r0 = 0; r0 < nr; r0 += rs) {
    const int r = r0 + tid / TPR % rs, m = m0 + min(r, nr - 1);
    Joined a;
    constexpr int AHEAD = 4;
    for (int s0 = way; s0 < np; s0 += AHEAD * ways) {
      u32x4_t x[AHEAD], y[AHEAD];
      u32x2_t v[AHEAD];
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        const uint32_t at = (uint32_t)(min(s0 + e * ways, np - 1) * rows + (int64_t)(b * p.Hk + hk) * R + m);
        x[e] = coherent_load16(p.ws, at * (D * 4) + d0 * 4);
        y[e] = coherent_load16(p.ws, at * (D * 4) + d0 * 4 + 16);
        v[e] = coherent_load8(p.ws, (uint32_t)(parts * rows) * (D * 4) + at * 8);
      }
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (s0 + e * ways < np) {
          float f[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            f[k] = __uint_as_float(x[e][k]);
            f[4 + k] = __uint_as_float(y[e][k]);
          }
          a.add(__uint_as_float(v[e][0]), __uint_as_float(v[e][1]), f);
        }
    }
    if (ways > 1) {   // (then one pass: rs >= nr)
      float* mine = so + tid / TPR * A::PITCH;
#pragma unroll
      for (int e = 0; e < 8; ++e) mine[d0 + e] = a.o[e];
      if (d0 == 0) {
        mine[D] = a.M;
        mine[D + 1] = a.L;
      }
      __syncthreads();
      if (way == 0)
        for (int w = 1; w < ways; ++w) {
          const float* other = so + (w * rs + tid / TPR) * A::PITCH;
          a.add(other[D], other[D + 1], other + d0);
        }
    }
    if (way == 0 && r < nr) paged_store(p, b, hk * G + m % G, m / G, d0, a.o, a.L);
  }
}

// How a call is cut: as many parts as the widest sequence that its table allows would take, and no more workgroups than a share
// of those that fit the chip at once.  So one long sequence in a batch of many short ones is cut into few parts.  For instance
// (us; parts 1, 4, 8, 16, 32):
//     1 x 4 key heads of 8 heads, 2944 keys, bf16, d 128        22   11  8.8  8.8
//     2 x 8 of 8, 9728 keys, int8, d 128                        78   26   17   16   20
//     40 x 8 of 4, 2176 keys, int8, d 128                       39   40   46   67
//     33 x 4 of 4, 6 queries, 6912 keys, int8, d 64             70   30   32   45   92
// Eight waves a workgroup in place of four were 1.4 % faster at their best over all calls, 20 % for some.
struct PagedPlan {
  int rt, nrb, parts;
  float each_cu;   // parts of a block with which every CU has a workgroup
  bool once;
};
constexpr size_t kCounterBytes = CF_PAGED_WS_HEADER_BYTES;
constexpr int kMaxParts = 64, kCUs = 256;
PagedPlan make_plan(const PagedParams& p) {
  const int64_t R = (int64_t)(p.H / p.Hk) * p.Lq;
  PagedPlan pl;
  pl.rt = R <= 16 ? 1 : 2;
  pl.nrb = (int)((R + 16 * pl.rt - 1) / (16 * pl.rt));
  const int64_t blocks = (int64_t)p.B * p.Hk * pl.nrb, keys = (int64_t)p.pages << p.c.shift, rows = (int64_t)p.B * p.Hk * R;
  const bool bf16 = p.c.code == CACHE_BF16;
  pl.once = pl.nrb == 1 && p.softcap <= kNearCap && read_past(p.B * keys, p.Hk, p.d, bf16);
  const int resident = kCUs * (p.d == 128 ? (pl.rt == 1 ? 3 : 2) : (pl.rt == 1 ? 5 : 3));   // workgroups, by registers (without MIXED)
  const double share = bf16 && p.d == 128 && pl.rt == 1 ? 0.35 : 0.7;
  const int64_t steps = (keys + kStepKeys - 1) / kStepKeys;
  const int64_t most = steps <= (p.d == 128 ? kOneSteps<128> : kOneSteps<64>) ? 1 : (int64_t)std::sqrt((double)steps * (2.0 / pl.rt));
  int64_t parts = std::min<int64_t>({kMaxParts, (int64_t)(resident * share) / blocks, most});
  parts = std::min<int64_t>(parts, ((int64_t)1 << 30) / (rows * (p.d + 2) * 4));   // the partial results are addressed in 32 bits
  if (blocks > (int64_t)kCounterBytes / 4) parts = 1;
  pl.parts = (int)std::max<int64_t>(1, parts);
  pl.each_cu = (float)kCUs / (float)blocks;
  return pl;
}

template <int D, int CODE, int RT, bool ONCE, bool MIXED, bool FAR>
hipError_t launch_kernel(PagedParams p, const PagedPlan& pl, hipStream_t st) {
  unsigned* const count = reinterpret_cast<unsigned*>(p.ws);
  if (pl.parts > 1) p.ws += kCounterBytes / 4;
  const int64_t wgs = (int64_t)p.B * p.Hk * pl.nrb * pl.parts;
  hipLaunchKernelGGL((paged_kernel<D, CODE, RT, ONCE, MIXED, FAR>), dim3((unsigned)wgs), dim3(64 * kWaves), 0, st, p, pl.nrb, pl.parts, p.B / pl.parts, pl.each_cu,
                     count);
  return hipGetLastError();
}
template <int D, int CODE, int RT, bool MIXED>
hipError_t launch_mixed(const PagedParams& p, const PagedPlan& pl, hipStream_t st) {
  if (p.softcap > kNearCap) return launch_kernel<D, CODE, RT, false, MIXED, true>(p, pl, st);
  return pl.once ? launch_kernel<D, CODE, RT, true, MIXED, false>(p, pl, st) : launch_kernel<D, CODE, RT, false, MIXED, false>(p, pl, st);
}
template <int D, int CODE, int RT>
hipError_t launch_rt(const PagedParams& p, const PagedPlan& pl, hipStream_t st) {
  if constexpr (CODE != CACHE_I8)   // (its codes are finite, and a scale is applied to the weights)
    if (p.causal && p.Lq > 1) return launch_mixed<D, CODE, RT, true>(p, pl, st);
  return launch_mixed<D, CODE, RT, false>(p, pl, st);
}
template <int D, int CODE>
hipError_t launch_code(const PagedParams& p, const PagedPlan& pl, hipStream_t st) {
  return pl.rt == 1 ? launch_rt<D, CODE, 1>(p, pl, st) : launch_rt<D, CODE, 2>(p, pl, st);
}
template <int D>
hipError_t launch_d(const PagedParams& p, const PagedPlan& pl, hipStream_t st) {
  return p.c.code == CACHE_BF16 ? launch_code<D, CACHE_BF16>(p, pl, st)
         : p.c.code == CACHE_I8 ? launch_code<D, CACHE_I8>(p, pl, st) : launch_code<D, CACHE_E4M3>(p, pl, st);
}

}  // namespace

size_t paged_workspace(const PagedParams& p) {
  const int parts = make_plan(p).parts;
  if (parts == 1) return 0;
  return kCounterBytes + (size_t)parts * (size_t)p.B * (size_t)p.H * (size_t)p.Lq * (size_t)(p.d + 2) * 4;
}

hipError_t launch_paged(const PagedParams& p, hipStream_t st) {
  const PagedPlan pl = make_plan(p);
  return p.d == 128 ? launch_d<128>(p, pl, st) : launch_d<64>(p, pl, st);
}

void paged_form(const PagedParams& p, char* text, size_t bytes) {
  const PagedPlan pl = make_plan(p);
  snprintf(text, bytes, "%d rows, %d blocks, %d parts%s", 16 * pl.rt, pl.nrb, pl.parts, pl.once ? ", read once" : "");
}

}  // namespace cf
