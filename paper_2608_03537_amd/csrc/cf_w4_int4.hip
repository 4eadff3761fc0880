// The product with 4-bit weights: kernels for integers.
#include "cf_w4.h"

namespace cf {

hipError_t launch_w4_int4(int tile, const GemmW4Params& p, hipStream_t st) { return AllW4Tiles::launch<false>(tile, p, st); }

}  // namespace cf
