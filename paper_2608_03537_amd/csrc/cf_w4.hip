// 4-bit weights: the choice of the product's tile (kernels in cf_w4.h), and how codes and scales are laid out.
#include <algorithm>
#include <cstdio>

#include "cf_w4.h"

namespace cf {

namespace {

// The tiles and their estimated time (us): rounds of 256 workgroups, each `step` for every 64 k (and `busy` times the
// share of CUs at work) and `start` besides, and `once`; int4, then E2M1.  (The last tile fits a CU twice; two together
// take as long as one after the other.)  Fitted to 1 to 4096 tokens, 512 to 16384 channels and 512 to 8192 k, groups of 128;
// for instance (us, in this order; - not measured; single kernels with pauses, at a full clock):
//     1 x 4096 x 4096 int4       6.8  9.3  7.9  9.9  9.0   13   20    -
//     1 x 12288 x 4096 int4      9.7  9.9   14   10   16   13   20    -
//     16 x 12288 x 4096 E2M1      11  8.2   12  8.9   16   11   17    -
//     32 x 4096 x 4096 E2M1      8.5  7.3  7.0  8.2  8.8   11   17   31
//     48 x 12288 x 4096 E2M1      26   20   19   16   16 12.2   18   31
//     128 x 4096 x 4096 int4       -    -    -    - 10.0   14   21   40
//     512 x 4096 x 4096 int4       -    -    -    -   37   29 25.6   45
//     1024 x 4096 x 4096 int4      -    -    -    -   68   53 44.7 44.8
//     4096 x 4096 x 4096 int4      -    -    -    -  259  195  164  138
// Over the 1011 calls that were timed the tile that the estimate takes is 0.4 % slower than the best one on average, 42 %
// at worst (1024 x 512 x 8192).
struct Cost {
  double step, start, once, busy;
};
struct Form {
  int tm, tn, threads, blocks, groups;   // blocks of a wave, groups of waves
  Cost cost[2];
};
constexpr int kCUs = 256;
template <class S>
constexpr Form form_of(Cost int4, Cost e2m1) {
  return {S::TM, S::TN, S::NT, S::BM * S::BN, S::KW, {int4, e2m1}};
}
template <class... S>
constexpr int count_of(W4Tiles<S...>) { return (int)sizeof...(S); }
const Form kForms[] = {   // in the order of AllW4Tiles
    form_of<W4Tile<1, 1, 1, 1, 8, 4, 8>>({0.0355, 0.90, 3.20, 0.0138}, {0.0224, 1.10, 2.81, 0.0089}),
    form_of<W4Tile<1, 2, 1, 1, 8, 4, 16>>({0.0708, 1.35, 3.02, 0.0199}, {0.0396, 2.27, 1.92, 0.0263}),
    form_of<W4Tile<1, 1, 1, 1, 8, 4, 32>>({0.0505, 3.07, 1.48, 0.0090}, {0.0315, 3.16, 1.46, 0.0091}),
    form_of<W4Tile<1, 2, 1, 1, 8, 4, 32>>({0.0752, 3.57, 1.41, 0.0181}, {0.0443, 3.56, 1.39, 0.0248}),
    form_of<W4Tile<2, 1, 1, 1, 8, 2, 64>>({0.0723, 2.90, 1.38, 0.0127}, {0.0725, 2.60, 1.24, 0.0152}),
    form_of<W4Tile<2, 2, 1, 1, 4, 4, 64>>({0.1235, 3.93, 1.19, 0.0231}, {0.0957, 3.99, 1.00, 0.0253}),
    form_of<W4Tile<2, 2, 1, 2, 4, 2, 64>>({0.2431, 3.72, 0.58, 0.0535}, {0.1973, 3.80, 0.38, 0.0574}),
    form_of<W4Tile<2, 2, 2, 2, 1, 4, 128>>({0.5094, 1.29, 4.14, 0.0699}, {0.3973, 1.53, 3.66, 0.0913}),
};
static_assert(sizeof(kForms) / sizeof(Form) == count_of(AllW4Tiles{}), "a row for every tile");

int choose_form(const GemmW4Params& p) {
  int best = -1;
  double least = 0;
  const double kt = (double)((p.K + 63) / 64);
  for (int i = 0; i < count_of(AllW4Tiles{}); ++i) {
    const Form& f = kForms[i];
    const int64_t wgs = (int64_t)((p.M + f.tm - 1) / f.tm) * ((p.N + f.tn - 1) / f.tn);
    if (wgs * f.threads > UINT32_MAX) continue;   // a grid has less than 2^32 threads; 128 x 128 tiles of M N <= 2^37 fit
    const Cost& c = f.cost[p.e2m1];
    const double rounds = (double)((wgs + kCUs - 1) / kCUs);
    const double t = kt * (rounds * c.step + std::min(1.0, (double)wgs / kCUs) * c.busy) + rounds * c.start + c.once;
    if (best < 0 || t < least) {
      best = i;
      least = t;
    }
  }
  return best;
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

// `tg` threads (a power of two) take a group of a channel, 8 values each at a time, kept in registers between the maximum
// and the codes where the group has no more; one behind the last group, what the tiles have behind K.  Channels of a tile go
// first: their words lie beside each other (12288 x 4096 bf16 in groups of 128: 65 us; with one thread a group 1316).
__global__ __launch_bounds__(256) void w4_quant_kernel(W4QuantParams p, int tg) {
  const int KB = (p.K + 63) / 64, ng = p.K / p.group, per = ng + (p.K % 64 != 0);
  const int64_t all = (int64_t)((p.N + 31) / 32) * 32 * per;
  const float most = p.e2m1 ? 6.0f : 7.0f;
  const int lane = threadIdx.x % tg, own = 256 / tg;   // groups of a workgroup
  for (int64_t x = (int64_t)blockIdx.x * own + threadIdx.x / tg; x < all; x += (int64_t)gridDim.x * own) {
    const int64_t block = x / 32 / per;
    const int n = (int)(block * 32 + x % 32), g = (int)(x / 32 % per);
    const int k0 = g * p.group, words = g < ng ? p.group / 8 : (KB * 64 - k0) / 8;
    const bool real = n < p.N && g < ng;
    const char* const row = reinterpret_cast<const char*>(p.W) + (n * p.ldw + k0) * (p.f32 ? 4 : 2);
    auto get = [&](int j, float (&v)[8]) {
      if (p.f32) {
        const f32x4_t a = __builtin_bit_cast(f32x4_t, gload16(row + j * 32)), b = __builtin_bit_cast(f32x4_t, gload16(row + j * 32 + 16));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = a[e];
          v[4 + e] = b[e];
        }
      } else {
        const u32x4_t w = gload16(row + j * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[2 * e] = bf16_to_f32(w[e] & 0xFFFFu);
          v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
      }
    };
    float v[8] = {};
    uint32_t mb = 0;   // max |w| by its bits: a NaN is above infinity
    if (real)
      for (int j = (words - 1) / tg * tg + lane; j >= 0; j -= tg)   // (the first one stays)
        if (j < words) {
          get(j, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) mb = max(mb, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        }
    for (int o = 1; o < tg; o *= 2) mb = max(mb, (uint32_t)__shfl_xor((int)mb, o));
    const bool bad = mb >= 0x7F800000u;
    float s = __uint_as_float(mb) / most;
    if (!p.s_f32) s = bf16_to_f32(pack_bf16x2(s, 0.0f) & 0xFFFFu);
    if (real && lane == 0) {
      const float put = bad ? __uint_as_float(0x7FC00000u) : s;
      const int64_t at = g * p.lds + n;
      if (p.s_f32) reinterpret_cast<float*>(p.s)[at] = put;
      else reinterpret_cast<bf16_t*>(p.s)[at] = (bf16_t)(__float_as_uint(put) >> 16);
    }
    for (int j = lane; j < words; j += tg) {
      uint32_t w = 0;
      if (real && s > 0.0f && !bad) {
        if (j != lane) get(j, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = v[e] / s;
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
      }
      *tile_word(p.tiles, KB, n, k0 + 8 * j) = w;
    }
  }
}

}  // namespace

hipError_t launch_gemm_w4(const GemmW4Params& p, hipStream_t st) {
  return p.e2m1 ? launch_w4_e2m1(choose_form(p), p, st) : launch_w4_int4(choose_form(p), p, st);
}

void gemm_w4_form(const GemmW4Params& p, char* text, size_t bytes) {
  const Form& f = kForms[choose_form(p)];
  snprintf(text, bytes, "%d x %d tiles of %d threads, scales every %d", f.tm, f.tn, f.threads,
           w4_fold(f.blocks, f.groups, p.K, p.group));
}

hipError_t launch_w4_pack(int N, int K, const uint8_t* codes, int64_t ldc, uint8_t* tiles, hipStream_t st) {
  const int64_t threads = (int64_t)(N + 31) / 32 * 32 * ((K + 63) / 64) * 8;
  hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)std::min<int64_t>((threads + 255) / 256, 1 << 16)), dim3(256), 0, st, N, K, codes, ldc, tiles);
  return hipGetLastError();
}

hipError_t launch_w4_quant(const W4QuantParams& p, hipStream_t st) {
  int tg = 4;
  while (tg < 64 && tg * 8 < p.group) tg *= 2;
  const int64_t groups = (int64_t)(p.N + 31) / 32 * 32 * (p.K / p.group + 1), own = 256 / tg;
  hipLaunchKernelGGL(w4_quant_kernel, dim3((unsigned)std::min<int64_t>((groups + own - 1) / own, 1 << 20)), dim3(256), 0, st, p, tg);
  return hipGetLastError();
}

}  // namespace cf
