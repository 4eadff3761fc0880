// The product with 4-bit weights: kernels for E2M1.
#include "cf_w4.h"

namespace cf {

hipError_t launch_w4_e2m1(int tile, const GemmW4Params& p, hipStream_t st) { return AllW4Tiles::launch<true>(tile, p, st); }

}  // namespace cf
