// Matrix products on tiles of 256 x 256 results, two steps of the reduction in LDS (linear_gemm.h).
#include "linear_gemm.h"

namespace purine {
namespace lin {
hipError_t gemm_256_2(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st) { return gemm_any<256, 256, 2>(p, a_in, b_in, act, st); }
}  // namespace lin
}  // namespace purine
