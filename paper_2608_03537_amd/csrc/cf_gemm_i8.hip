// Matrix product of 8-bit integers with a scale per token and per channel:
//     C[m, n] = act(float(sum_k A[m, k] B[n, k]) sa[m] sb[n] + bias[n]).
// The sum is exact in 32 bits for K <= 131056 (|product| <= 2^14), so the order
// of its terms is free: waves split K and tiles differ in shape without
// changing a bit of the result.
//
// An MFMA covers 32 bytes of k per operand row in 32 cycles, as the bf16 one does,
// so in bytes these loops are those of a bf16 product with half the k.  Tiles:
//   32 x 32 to 64 x 64   a wave each, with a ring of LDS stages of its own; the waves of a workgroup
//                split K and their sums meet in LDS.
//   64 x 128, 128 x 128  four waves share a tile and a ring; two such groups split K, one multiplying while
//                the other reads (1024 x 4096 x 4096 24.5 -> 22.7 us against one group of four waves,
//                512 x 4096 x 4096 17.7 -> 15.8 against two pairs, all in step).
//   128 x 128    four waves, two workgroups a CU, where there are more than 256 tiles.
//   256 x 256    big_product in cf_gemm_big.h.
// What bounds them: a CU's direct loads into LDS reach 90 to 100 GB/s with all CUs busy, so few tokens
// are the weights' stream.  In between it is how well a step's loads, LDS reads and MFMAs overlap (1024 x 4096
// x 4096 on 128 x 128 tiles: 13, 9 and 9 us by themselves, 18 together, and 5 of start and output).  256 x 256
// tiles run 16384 x 4096 x 4096 in 236 us, 2.3 POP/s; with operands of zeros, whose MFMAs draw
// less power, in 184: the clock that full power leaves bounds them.  kForms has
// the measurements of all.  A form that loads fragments straight into registers
// was slower from 16 tokens on (48 x 12288 x 4096 29 us against 12.8: rows of a power
// of two apart meet in the same sets of the first-level cache).
#include <algorithm>
#include <cstdio>

#include "cf_attn.h"
#include "cf_gemm_big.h"
#include "cf_serving.h"

namespace cf {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4_t;
typedef __attribute__((__vector_size__(16 * sizeof(int)))) int i32x16_t;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;

// D (32 n x 32 m) += W (32 n x 32 k) X (32 k x 32 m): lane l gives 16 k of row l % 32 of
// either operand, k group l / 32; layout of D as for the bf16 atom (acc_row).
struct MmaI8 {
  __device__ __forceinline__ static void run(i32x16_t& acc, u32x4_t w, u32x4_t x) {
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4_t, w), __builtin_bit_cast(i32x4_t, x), acc, 0,
                                                0, 0);
  }
};

template <int ACT>
__device__ __forceinline__ float act_i8(float x) {
  if constexpr (ACT == ACT_GELU) return gelu_erf(x);
  if constexpr (ACT == ACT_GELU_TANH) return 0.5f * x * (1.0f + tanh_exp(0.79788456080286536f * (x + 0.044715f * x * x * x)));
  if constexpr (ACT == ACT_RELU) return x < 0.0f ? 0.0f : x;
  return x;
}
// f(std::integral_constant<int, act>{})
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == ACT_GELU) f(std::integral_constant<int, ACT_GELU>{});
  else if (act == ACT_GELU_TANH) f(std::integral_constant<int, ACT_GELU_TANH>{});
  else if (act == ACT_RELU) f(std::integral_constant<int, ACT_RELU>{});
  else f(std::integral_constant<int, ACT_NONE>{});
}

// Output pass of a tile whose sums lie in LDS: KW planes of TM rows of TN int32 (pitch TN * 4 +
// 16 bytes), added here.  A thread takes 8 columns of a row at a time, always the same columns.
// Its scales and biases are loaded ahead (before the main loop, where registers allow: loaded
// here, they add a trip to memory to every tile).  AHEAD = false: all of the tile's lie in LDS (stage_scales),
// and the rows are not unrolled, for the 256 x 256 tiles, which have no registers to spare here.
template <int TM, int TN, int NT, bool AHEAD>
struct TileScales {
  static constexpr int CPR = TN / 8, STEP = NT / CPR, RPT = (TM + STEP - 1) / STEP;   // a thread's rows: STEP apart
  static_assert(NT % CPR == 0, "a thread keeps its columns");
  float sa[AHEAD ? RPT : 1], sb[8], bias[8];
  const float* rows;   // AHEAD = false: the rows' scales in LDS
  __device__ __forceinline__ void load(const GemmI8Params& p, int m0, int n0) {
    const int n = n0 + threadIdx.x % CPR * 8, r0 = threadIdx.x / CPR;
    auto eight = [&](const float* v, float none, float (&out)[8]) {
      if (v && n + 8 <= p.N) {
        const f32x4_t a = *reinterpret_cast<const f32x4_t*>(v + n), b = *reinterpret_cast<const f32x4_t*>(v + n + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          out[e] = a[e];
          out[4 + e] = b[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = v && n + e < p.N ? v[n + e] : none;
      }
    };
    eight(p.sb, 1.0f, sb);
    eight(p.bias, 0.0f, bias);
#pragma unroll
    for (int i = 0; i < RPT; ++i) sa[i] = p.sa ? p.sa[min(m0 + r0 + i * STEP, p.M - 1)] : 1.0f;
  }
  // From LDS: sa of the rows, and sb and bias of the tile's columns (only those that the call has).
  __device__ __forceinline__ void load_staged(const GemmI8Params& p, const float* la, const float* lb, const float* lbias) {
    const int c = threadIdx.x % CPR * 8;
    rows = la;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sb[e] = p.sb ? lb[c + e] : 1.0f;
      bias[e] = p.bias ? lbias[c + e] : 0.0f;
    }
  }
};

template <int TM, int TN, int KW, int NT, bool AHEAD>
__device__ __forceinline__ void finish_tile(const GemmI8Params& p, const TileScales<TM, TN, NT, AHEAD>& sc,
                                            const char* smem, int m0, int n0) {
  using Sc = TileScales<TM, TN, NT, AHEAD>;
  constexpr int PITCH = TN * 4 + 16;
  const int tid = threadIdx.x, c8 = tid % Sc::CPR * 8, left = p.N - n0 - c8;
  if (left <= 0) return;
  const int rows = min(TM, p.M - m0);
  with_act(p.act, [&](auto act_t) {
    constexpr int ACT = decltype(act_t)::value;
    auto row = [&](int r, float sa) {
      const char* src = smem + r * PITCH + c8 * 4;
      i32x4_t a = *reinterpret_cast<const i32x4_t*>(src), b = *reinterpret_cast<const i32x4_t*>(src + 16);
#pragma unroll
      for (int k = 1; k < KW; ++k) {
        a += *reinterpret_cast<const i32x4_t*>(src + k * TM * PITCH);
        b += *reinterpret_cast<const i32x4_t*>(src + k * TM * PITCH + 16);
      }
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = (float)(e < 4 ? a[e] : b[e - 4]) * sa * sc.sb[e];
        if (p.bias) x += sc.bias[e];
        y[e] = act_i8<ACT>(x);
      }
      const int64_t at = (int64_t)(m0 + r) * p.ldc + n0 + c8;
      if (left >= 8) {
        if (p.c_f32) {
          float* c = reinterpret_cast<float*>(p.C) + at;
          __builtin_nontemporal_store(f32x4_t{y[0], y[1], y[2], y[3]}, reinterpret_cast<f32x4_t*>(c));
          __builtin_nontemporal_store(f32x4_t{y[4], y[5], y[6], y[7]}, reinterpret_cast<f32x4_t*>(c + 4));
        } else {
          const u32x4_t w = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                             pack_bf16x2(y[6], y[7])};
          __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(reinterpret_cast<bf16_t*>(p.C) + at));
        }
      } else if (p.c_f32) {   // 4, 2 and 1 columns by the bits of `left` (one by one: 1699 x 5327 x 896 24.4 us, so 21.7)
        float* c = reinterpret_cast<float*>(p.C) + at;
        const bool h = left & 4;
        if (h) *reinterpret_cast<f32x4_t*>(c) = f32x4_t{y[0], y[1], y[2], y[3]};
        c += left & 4;
        const float z[3] = {h ? y[4] : y[0], h ? y[5] : y[1], h ? y[6] : y[2]};
        if (left & 2) *reinterpret_cast<f32x2_t*>(c) = f32x2_t{z[0], z[1]};
        if (left & 1) c[left & 2] = left & 2 ? z[2] : z[0];
      } else {
        bf16_t* c = reinterpret_cast<bf16_t*>(p.C) + at;
        const bool h = left & 4;
        if (h) *reinterpret_cast<u32x2_t*>(c) = u32x2_t{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        c += left & 4;
        const uint32_t z[2] = {pack_bf16x2(h ? y[4] : y[0], h ? y[5] : y[1]), pack_bf16x2(h ? y[6] : y[2], 0.0f)};
        if (left & 2) *reinterpret_cast<uint32_t*>(c) = z[0];
        if (left & 1) c[left & 2] = (bf16_t)(left & 2 ? z[1] : z[0]);
      }
    };
    const int r0 = tid / Sc::CPR;
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < Sc::RPT; ++i)
        if (r0 + i * Sc::STEP < rows) row(r0 + i * Sc::STEP, sc.sa[i]);
    } else {
#pragma unroll 2
      for (int r = r0; r < rows; r += Sc::STEP) row(r, p.sa ? sc.rows[r] : 1.0f);
    }
  });
}

// ---------------------------------------------------------------------------
// Tile.  A group of WM x WN waves (32 BM tokens x 32 BN channels each) shares a ring of
// NS stages of 128 bytes of k; KW groups take the stages in turn.  A group of one wave
// needs no barrier until the end.  ALT: two groups of four waves that read and multiply by turns
// (below).  The 16-byte chunk ch of row r of a stage sits at position ch ^ ((r >> 1) & 7), as in big_product.
// ---------------------------------------------------------------------------
template <int BM_, int BN_, int WM_, int WN_, int KW_, int NS_, bool ALT_ = false>
struct I8Tile {
  static constexpr bool ALT = ALT_;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KW = KW_, NS = NS_;
  static constexpr int GW = WM * WN, NW = GW * KW, NT = 64 * NW;
  static constexpr int TM = 32 * BM * WM, TN = 32 * BN * WN, STAGE = (TM + TN) * 128;
  static constexpr int RING = NS * STAGE, OUT = KW * TM * (TN * 4 + 16);
  static constexpr int LDS = KW * RING > OUT ? KW * RING : OUT;
  static constexpr int LPW = (TM + TN) / 8 / GW;   // wave-wide loads of a stage per wave
  static_assert(LDS <= 160 * 1024 && LPW * NS < 64, "LDS budget, vmcnt range");
  static_assert(!ALT || (KW == 2 && NW == 8), "two waves a SIMD");
};

// Fragments of a stage's four k steps of NB 32-row blocks at a[0..3], complete.
template <int NB>
__device__ __forceinline__ void read_blocks(u32x4_t (&f)[NB][4], const uint32_t (&a)[4]) {
  if constexpr (NB == 2) read_x_half<0>(f, a);
  else read_w_half_nk<0>(f[0], a);
}

// CUT: K ends inside a step (a kernel of its own: looking for that step costs whole K 0.3 us).
template <class S, bool CUT>
__global__ __launch_bounds__(S::NT) void gemm_i8_tile_kernel(GemmI8Params p) {
  __shared__ __attribute__((aligned(16))) char smem[S::LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int grp = wave / S::GW, gw = wave % S::GW, wm = gw / S::WN, wn = gw % S::WN;
  int rb, c;
  big_tile_order((p.M + S::TM - 1) / S::TM, (p.N + S::TN - 1) / S::TN, rb, c);
  const int m0 = rb * S::TM, n0 = c * S::TN;
  TileScales<S::TM, S::TN, S::NT, true> sc;
  sc.load(p, m0, n0);
  char* const ring = smem + grp * S::RING;
  const int KT = (p.K + 127) / 128, steps = grp < KT ? (KT - grp - 1) / S::KW + 1 : 0;   // steps; those of this group
  const int rem = p.K % 128, cut = (KT - 1) % S::KW == grp ? steps - 1 : -1;      // CUT: the group's step that K ends in

  // Stage rows 0 .. TM - 1 are tokens, then TN channels; load i of a wave fills rows
  // 8 (i GW + gw) .. + 7.  Rows past M and N are clamped (they feed nothing that is stored).
  const char* src[S::LPW];
#pragma unroll
  for (int i = 0; i < S::LPW; ++i) {
    const int row = 8 * (i * S::GW + gw) + (lane >> 3), ch = (lane & 7) ^ ((row >> 1) & 7);
    src[i] = (row < S::TM ? reinterpret_cast<const char*>(p.A) + (int64_t)min(m0 + row, p.M - 1) * p.lda
                          : reinterpret_cast<const char*>(p.B) + (int64_t)min(n0 + row - S::TM, p.N - 1) * p.ldb) +
             ch * 16 + grp * 128;
  }
  // Loads i0 .. i1 - 1 of the group's step s, into stage s % NS; of the step that K ends in, a lane whose
  // chunk lies behind K takes the step's first one (cleared when read).
  auto load = [&](int s, int i0, int i1) {
#pragma unroll
    for (int i = i0; i < i1; ++i) {
      const char* from = src[i] + (int64_t)s * (S::KW * 128);
      if (CUT && s == cut) {
        const int ch = ((lane & 7) ^ ((4 * (i * S::GW + gw) + (lane >> 4)) & 7)) * 16;
        if (ch >= rem) from -= ch;
      }
      dma16(from, ring + s % S::NS * S::STAGE + gw * 1024 + i * S::GW * 1024);
    }
  };
  const uint32_t s0 =
      (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem) + grp * S::RING;
  uint32_t xa[4], wa[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const int ch = ((2 * ks + lg) ^ ((lr >> 1) & 7)) << 4;
    xa[ks] = s0 + (wm * 32 * S::BM + lr) * 128 + ch;
    wa[ks] = s0 + (S::TM + wn * 32 * S::BN + lr) * 128 + ch;
  }
  i32x16_t acc[S::BM][S::BN] = {};
  u32x4_t xf[S::BM][4], wf[S::BN][4];
  auto mma = [&](int ks) {
#pragma unroll
    for (int bm = 0; bm < S::BM; ++bm)
#pragma unroll
      for (int bn = 0; bn < S::BN; ++bn) MmaI8::run(acc[bm][bn], wf[bn][ks], xf[bm][ks]);
  };
  auto read = [&](int s) {
    const uint32_t at = s % S::NS * S::STAGE;
    const uint32_t x[4] = {xa[0] + at, xa[1] + at, xa[2] + at, xa[3] + at};
    const uint32_t w[4] = {wa[0] + at, wa[1] + at, wa[2] + at, wa[3] + at};
    read_blocks<S::BM>(xf, x);
    read_blocks<S::BN>(wf, w);
    if (CUT && s == cut) {   // one operand's zeros do for both
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        if (ks * 32 + lg * 16 >= rem)
#pragma unroll
          for (int b = 0; b < S::BM; ++b) xf[b][ks] = u32x4_t{};
    }
  };
  // The MFMAs of a step; the loads of a later one go between them (in front of the reads they would hold
  // them up): a wave on its own issues them at once, waves that share a step in three parts, since together they
  // fill the load path (512 x 4096 x 4096 on 64 x 128 tiles without ALT 18.2 -> 16.8 us; 64 x 64 11.8 -> 12.2).
  auto multiply = [&](int later) {
    constexpr int PARTS = S::GW > 1 ? 3 : 1;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      __builtin_amdgcn_sched_barrier(0);
      mma(ks);
      __builtin_amdgcn_sched_barrier(0);
      if (ks < PARTS && later < steps) load(later, ks * S::LPW / PARTS, (ks + 1) * S::LPW / PARTS);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  const int all = (KT + S::KW - 1) / S::KW;   // every group passes every barrier
  constexpr int FIRST = S::ALT ? S::NS : S::NS - 1;   // steps loaded ahead
#pragma unroll
  for (int s = 0; s < FIRST; ++s)
    if (s < steps) load(s, 0, S::LPW);
  if constexpr (S::ALT) {
    // Read and MFMA sections with a barrier behind each; group 1 is one section behind, and its waves share the
    // SIMDs with those of group 0, so one of the two multiplies while the other reads.  In front of the
    // barrier that ends a read section a wave waits for its loads of the next step (one section later the
    // group reads them); a step's stage is free once that barrier is passed.
    if (S::NS <= steps) wait_vmcnt<S::LPW*(S::NS - 1)>();
    else wait_vmcnt<0>();
    lds_barrier();
    if (grp == 1) lds_barrier();
    for (int s = 0; s < all; ++s) {
      if (s < steps) read(s);
      if (s + S::NS - 1 < steps) wait_vmcnt<S::LPW*(S::NS - 2)>();
      else wait_vmcnt<0>();
      lds_barrier();
      if (s < steps) multiply(s + S::NS);
      lds_barrier();
    }
    if (grp == 0) lds_barrier();
  } else {
    for (int s = 0; s < all; ++s) {
      if (s + S::NS - 2 < steps) wait_vmcnt<S::LPW*(S::NS - 2)>();
      else wait_vmcnt<0>();
      if constexpr (S::GW > 1) lds_barrier();   // every wave's loads of step s are in, and step s - 1 has been read
      if (s >= steps) continue;
      read(s);
      multiply(s + S::NS - 1);
    }
  }
  __syncthreads();
  constexpr int PITCH = S::TN * 4 + 16;
  char* const out = smem + grp * S::TM * PITCH;
#pragma unroll
  for (int bm = 0; bm < S::BM; ++bm)
#pragma unroll
    for (int bn = 0; bn < S::BN; ++bn)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const i32x16_t& v = acc[bm][bn];
        *reinterpret_cast<i32x4_t*>(out + ((wm * S::BM + bm) * 32 + lr) * PITCH +
                                    ((wn * S::BN + bn) * 32 + 8 * g + 4 * lg) * 4) =
            i32x4_t{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
      }
  __syncthreads();
  finish_tile<S::TM, S::TN, S::KW, S::NT>(p, sc, smem, m0, n0);
}

// ---------------------------------------------------------------------------
// Big.
// ---------------------------------------------------------------------------
constexpr int kI8BigPitch = kBigT * 4 + 16;
constexpr int kI8BigVec = 128 * kI8BigPitch > 2 * kBigStep ? 128 * kI8BigPitch : 2 * kBigStep;   // sa, sb and bias of the tile
constexpr int kI8BigLds = kI8BigVec + 3 * kBigT * 4;

// Values at .. at + 63 of v (clamped to n) into LDS, by direct loads: no registers are held while the product
// runs, whose waits cover them.
__device__ __forceinline__ void stage_scales(const float* v, int at, int n, char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  if (v)
    __builtin_amdgcn_global_load_lds(v + min(at + (int)(threadIdx.x & 63), n - 1),
                                     (__attribute__((address_space(3))) void*)lds, 4, 0, 0);
#endif
}

__global__ __launch_bounds__(512, 1) __attribute__((amdgpu_waves_per_eu(2, 2)))
void gemm_i8_big_kernel(GemmI8Params p) {
  __shared__ __attribute__((aligned(16))) char smem[kI8BigLds];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3, lr = lane & 31, lg = lane >> 5;
  int rb, c;
  big_tile_order((p.M + kBigT - 1) / kBigT, (p.N + kBigT - 1) / kBigT, rb, c);
  const int m0 = rb * kBigT, n0 = c * kBigT, KT = p.K / 128;
  float* const vec = reinterpret_cast<float*>(smem + kI8BigVec);   // sa [256], sb [256], bias [256]
  if (wave < 4) stage_scales(p.sa, m0 + 64 * wave, p.M, smem + kI8BigVec + 256 * wave);
  else stage_scales(p.sb, n0 + 64 * (wave - 4), p.N, smem + kI8BigVec + 256 * wave);
  if (wave < 4) stage_scales(p.bias, n0 + 64 * wave, p.N, smem + kI8BigVec + 2048 + 256 * wave);
  i32x16_t acc[2][2][2] = {};   // [token half][32-token block][channel half]
  big_product<false, MmaI8>(acc, reinterpret_cast<const char*>(p.A) + (int64_t)m0 * p.lda, p.lda, p.M - m0,
                            reinterpret_cast<const char*>(p.B) + (int64_t)n0 * p.ldb, p.ldb, p.N - n0, KT, smem);
  // k behind the last whole step, straight from memory
#pragma unroll 1
  for (int k = KT * 128 + lg * 16; k - lg * 16 < p.K; k += 32) {
    u32x4_t w[2], x[2][2];
    const bool in = k < p.K;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      w[h] = u32x4_t{};
      if (in) w[h] = gload16(p.B + (int64_t)min(n0 + h * 128 + wn * 32 + lr, p.N - 1) * p.ldb + k);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[h][b] = u32x4_t{};
        if (in) x[h][b] = gload16(p.A + (int64_t)min(m0 + h * 128 + wm * 64 + b * 32 + lr, p.M - 1) * p.lda + k);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) MmaI8::run(acc[i >> 2][(i >> 1) & 1][i & 1], w[i & 1], x[i >> 2][(i >> 1) & 1]);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int nh = 0; nh < 2; ++nh)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const i32x16_t& v = acc[h][b][nh];
          *reinterpret_cast<i32x4_t*>(smem + (wm * 64 + b * 32 + lr) * kI8BigPitch + (nh * 128 + wn * 32 + 8 * g + 4 * lg) * 4) =
              i32x4_t{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        }
    TileScales<128, kBigT, 512, false> sc;
    sc.load_staged(p, vec + h * 128, vec + 256, vec + 512);
    __syncthreads();
    finish_tile<128, kBigT, 1, 512>(p, sc, smem, m0 + h * 128, n0);
    __syncthreads();
  }
}

template <class S>
hipError_t launch_tile(const GemmI8Params& p, hipStream_t st) {
  const int64_t wgs = (int64_t)((p.M + S::TM - 1) / S::TM) * ((p.N + S::TN - 1) / S::TN);
  if (p.K % 128 == 0) hipLaunchKernelGGL((gemm_i8_tile_kernel<S, false>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p);
  else hipLaunchKernelGGL((gemm_i8_tile_kernel<S, true>), dim3((unsigned)wgs), dim3(S::NT), 0, st, p);
  return hipGetLastError();
}
hipError_t launch_big(const GemmI8Params& p, hipStream_t st) {
  const int64_t wgs = (int64_t)((p.M + kBigT - 1) / kBigT) * ((p.N + kBigT - 1) / kBigT);
  hipLaunchKernelGGL(gemm_i8_big_kernel, dim3((unsigned)wgs), dim3(512), 0, st, p);
  return hipGetLastError();
}

// The tiles and their estimated time: rounds of `per` workgroups, each `step` us for
// every 128 bytes of k and `start` us besides.  Fitted to M x N of 1 to 16384 with K of 512
// to 16384; for instance (us, in this order):
//     1 x 4096 x 4096        5.9  7.2  7.4  9.8   13   15   27   36
//     16 x 12288 x 4096     12.3 14.0 10.7 11.5   13   16   28   36
//     48 x 12288 x 4096     15.6 14.3 14.6 12.0 13.5   16   28   37
//     128 x 4096 x 4096     11.2  8.4  8.6 10.7   14   17   30   38
//     512 x 4096 x 4096       38   27   26 19.8 15.8   18   30   42
//     1024 x 4096 x 4096      73   49   49   36   30 22.7   31   43
//     2048 x 4096 x 4096     141   94   95   69   57   43 37.7   48
//     4096 x 4096 x 4096     282  184  187  135  111   82   75 60.4
//     8192 x 1024 x 1024      77   51   49   34   25   22 13.4   20
// Over 300 calls of all sizes the form that the estimate takes is 0.4 % slower than the best one on average,
// 20 % at worst.
struct Form {
  int tm, tn, threads, per;
  double step, start;
  hipError_t (*launch)(const GemmI8Params&, hipStream_t);
};
constexpr int kCUs = 256;
template <class S>
constexpr Form tile_form(int per, double step, double start) {
  return {S::TM, S::TN, S::NT, per, step, start, launch_tile<S>};
}
const Form kForms[] = {
    tile_form<I8Tile<1, 1, 1, 1, 4, 4>>(kCUs, 0.093, 2.45),
    tile_form<I8Tile<2, 1, 1, 1, 4, 3>>(kCUs, 0.154, 4.15),
    tile_form<I8Tile<1, 2, 1, 1, 6, 2>>(kCUs, 0.17, 2.7),
    tile_form<I8Tile<2, 2, 1, 1, 4, 2>>(kCUs, 0.21, 3.55),
    tile_form<I8Tile<1, 2, 2, 2, 2, 3, true>>(kCUs, 0.365, 3.6),
    tile_form<I8Tile<2, 2, 2, 2, 2, 2, true>>(kCUs, 0.415, 5.5),
    tile_form<I8Tile<2, 2, 2, 2, 1, 2>>(2 * kCUs, 0.935, 4.55),
    {kBigT, kBigT, 512, kCUs, 0.86, 11.9, launch_big},
};
constexpr double kBigBusy = 0.55;   // added to the step of 256 x 256 tiles times the share of CUs at work (clocks)
// Rows whose pitch is no multiple of 128 bytes take two lines of memory a step; the smaller tiles, which the load
// path bounds, run slower by this (300 x 4096 x 4080 17.3 us, x 4096 13.7; 256 x 256 tiles 16384 x 4096 x 4080 271, 240).
constexpr double kOddPitch = 1.27;

const Form& choose_form(const GemmI8Params& p) {
  const Form* best = nullptr;
  double least = 0;
  const double kt = (double)((p.K + 127) / 128);
  const bool odd = p.lda % 128 != 0 || p.ldb % 128 != 0;
  for (const Form& f : kForms) {
    if (f.tm == kBigT && p.K < 256) continue;   // its loop needs two whole steps
    const int64_t wgs = (int64_t)((p.M + f.tm - 1) / f.tm) * ((p.N + f.tn - 1) / f.tn), rounds = (wgs + f.per - 1) / f.per;
    if (wgs * f.threads > UINT32_MAX) continue;   // a grid has less than 2^32 threads; 128 x 128 tiles of M N <= 2^37 fit
    double step = f.step;
    if (f.tm == kBigT) step += kBigBusy * std::min(1.0, (double)wgs / kCUs);
    else if (odd) step *= kOddPitch;
    const double t = (double)rounds * (step * kt + f.start);
    if (!best || t < least) {
      best = &f;
      least = t;
    }
  }
  return *best;
}

}  // namespace

hipError_t launch_gemm_i8(const GemmI8Params& p, hipStream_t st) { return choose_form(p).launch(p, st); }

void gemm_i8_form(const GemmI8Params& p, char* text, size_t bytes) {
  const Form& f = choose_form(p);
  snprintf(text, bytes, "%d x %d tiles of %d threads, %s K", f.tm, f.tn, f.threads, p.K % 128 == 0 ? "whole" : "cut");
}

}  // namespace cf
