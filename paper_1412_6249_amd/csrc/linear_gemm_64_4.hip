// Matrix products on tiles of 64 x 64 results, four steps of the reduction in LDS (linear_gemm.h).
#include "linear_gemm.h"

namespace purine {
namespace lin {
hipError_t gemm_64_4(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st) { return gemm_any<64, 64, 4>(p, a_in, b_in, act, st); }
}  // namespace lin
}  // namespace purine
