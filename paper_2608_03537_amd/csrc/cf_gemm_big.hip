// Plain GEMM on 256 x 256 tiles for large bf16 products: C = alpha X W + bias.
//
// One workgroup of eight waves per tile, two waves per SIMD.  The wave tile is
// 128 x 64 (128 accumulator registers), so a 64-deep k step streams 64 KB of
// operands for 4.2 MMAC, half the bytes per MAC of the 128 x 256 tile, whose
// loop runs at the L2-to-LDS rate.
//
// The main loop is big_product (cf_gemm_big.h).
#include "cf_gemm_big.h"

namespace cf {

namespace {

constexpr int kBigPitch4 = kBigT * 4 + 16;       // staged output row, fp32
constexpr int kBigPitch2 = kBigT * 2 + 8;        // staged output row, bf16
constexpr int kBigLds = 128 * kBigPitch4 > 2 * kBigStep ? 128 * kBigPitch4 : 2 * kBigStep;

// Rows 0..127 or 128..255 of the tile through LDS to coalesced 16-byte stores.
template <int ESZ>
__device__ __forceinline__ void store_half(const f32x16_t (&x)[2][2], char* Y, int64_t ldy, int rows, int cols,
                                           char* smem, int tid, int lane, int wm, int wn) {
  constexpr int PITCH = ESZ == 4 ? kBigPitch4 : kBigPitch2;
  const int lr = lane & 31, lg = lane >> 5;
#pragma unroll
  for (int bm = 0; bm < 2; ++bm)
#pragma unroll
    for (int nh = 0; nh < 2; ++nh)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        char* dst = smem + (wm * 64 + bm * 32 + lr) * PITCH + (nh * 128 + wn * 32 + 8 * g + 4 * lg) * ESZ;
        const f32x16_t& v = x[bm][nh];
        if constexpr (ESZ == 4) {
          *reinterpret_cast<f32x4_t*>(dst) = f32x4_t{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        } else {
          *reinterpret_cast<u32x2_t*>(dst) =
              u32x2_t{pack_bf16x2(v[4 * g], v[4 * g + 1]), pack_bf16x2(v[4 * g + 2], v[4 * g + 3])};
        }
      }
  __syncthreads();
  constexpr int CPR = kBigT * ESZ / 16, EPC = 16 / ESZ, ITER = 128 * CPR / 512, BATCH = 8;
  static_assert(ITER % BATCH == 0, "store batches");
  const int64_t ldyb = ldy * ESZ;
  const bool full = rows >= 128 && cols >= kBigT;
#pragma unroll 1
  for (int j0 = 0; j0 < ITER; j0 += BATCH) {
    u32x4_t v[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int id = tid + (j0 + j) * 512;
      v[j] = *reinterpret_cast<const u32x4_t*>(smem + (id / CPR) * PITCH + (id % CPR) * 16);
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int id = tid + (j0 + j) * 512, r = id / CPR, cc = id % CPR;
      if (full || (r < rows && cc * EPC < cols))
        __builtin_nontemporal_store(v[j], reinterpret_cast<u32x4_t*>(Y + r * ldyb + cc * 16));
    }
  }
  __syncthreads();
}

}  // namespace

template <bool KN>
__global__ __launch_bounds__(512, 1) __attribute__((amdgpu_waves_per_eu(2, 2)))
void gemm_big_kernel(GemmRowsParams p) {
  __shared__ __attribute__((aligned(16))) char smem[kBigLds];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;          // waves 0..3: wm 0, waves 4..7: wm 1
  const int lg = lane >> 5;
  const int bz = blockIdx.y;

  int rb, c;
  big_tile_order(p.num_rb, p.cn, rb, c);
  const int m0 = rb * kBigT, n0 = c * kBigT;
  const bf16_t* X = reinterpret_cast<const bf16_t*>(p.X) + (int64_t)bz * p.sx;
  const bf16_t* W = reinterpret_cast<const bf16_t*>(p.W) + (int64_t)bz * p.sw;

  const char* xg = reinterpret_cast<const char*>(X + (int64_t)m0 * p.ldx);
  const char* wg = reinterpret_cast<const char*>(W) + (KN ? (int64_t)n0 : (int64_t)n0 * p.ldw) * 2;
  f32x16_t acc[2][2][2];   // [X half][32-row block][W half]
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i >> 2][(i >> 1) & 1][i & 1][e] = 0.0f;
  big_product<KN, Mma<bf16_t>>(acc, xg, p.ldx * 2, p.M - m0, wg, p.ldw * 2, p.N - n0, p.K / 64, smem);

  // C = alpha acc + bias; only a given bias is added (x + 0 would turn -0 into +0).
  const RowEpi& e = p.epi;
  if (e.alpha != 1.0f) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i >> 2][(i >> 1) & 1][i & 1][v] *= e.alpha;
  }
  if (e.bias) {
#pragma unroll
    for (int nh = 0; nh < 2; ++nh)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int n = min(n0 + nh * 128 + wn * 32 + 8 * g + 4 * lg, p.N - 4);   // columns past N are not stored
        const f32x4_t b = *reinterpret_cast<const f32x4_t*>(e.bias + n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[i >> 1][i & 1][nh][4 * g + q] += b[q];
      }
  }
  const int esz = e.y_f32 ? 4 : 2;
  char* Y = reinterpret_cast<char*>(e.Y) + ((int64_t)bz * e.sy + (int64_t)m0 * e.ldy + n0) * esz;
#pragma unroll
  for (int mh = 0; mh < 2; ++mh) {
    char* Yh = Y + (int64_t)mh * 128 * e.ldy * esz;
    const int rows = p.M - m0 - mh * 128, cols = p.N - n0;
    if (e.y_f32) store_half<4>(acc[mh], Yh, e.ldy, rows, cols, smem, tid, lane, wm, wn);
    else store_half<2>(acc[mh], Yh, e.ldy, rows, cols, smem, tid, lane, wm, wn);
  }
}

static const GemmKernel kTable[] = {
    {kBigT, kBigT, 0, 1, 0, 512, 3, 0, reinterpret_cast<const void*>(&gemm_big_kernel<false>),
     reinterpret_cast<const void*>(&gemm_big_kernel<false>)},
    {kBigT, kBigT, 0, 2, 0, 512, 3, 0, reinterpret_cast<const void*>(&gemm_big_kernel<true>),
     reinterpret_cast<const void*>(&gemm_big_kernel<true>)},
};

const GemmKernel* gemm_kernels_big(int* n) {
  *n = (int)(sizeof(kTable) / sizeof(kTable[0]));
  return kTable;
}

}  // namespace cf
