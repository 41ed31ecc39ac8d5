// Launchers of the block operators (group_norm.hip, linear.hip, adamw.hip), called by block_api.cpp with checked arguments.
#pragma once
#include "common.h"
#include "purine_block.h"

namespace purine {

struct NormShape {
    int N, S, C, G;                 // images, positions, channels, groups
    int64_t x_ns, y_ns, dy_ns, dx_ns;   // elements between images
    float eps;
    int act;
};
size_t group_norm_ws_bytes(int64_t N, int64_t S, int64_t C, int64_t G);
hipError_t launch_group_norm_fwd(int dtype, const NormShape& s, const void* x, const float* scale, const float* shift, void* y, float* mean,
                                 float* rstd, void* ws, hipStream_t st);
hipError_t launch_group_norm_bwd(int dtype, const NormShape& s, const void* x, const float* scale, const float* shift, const float* mean,
                                 const float* rstd, const void* dy, void* dx, float* dscale, float* dshift, float beta, void* ws, hipStream_t st);

// out[i][j] = epilogue(sum over k of A(i, k) B(j, k)); an operand's reduction axis is its inner one (k_in: element (i, k) at i * ld + k)
// or its outer one (k * ld + i).
struct LinearCall {
    int64_t rows, cols, K;
    const void* a; int64_t a_ld; bool a_in;
    const void* b; int64_t b_ld; bool b_in;
    int dtype;                       // of the operands
    void* out; int64_t out_ld; int out_dtype;
    const void* bias;                // per column, of the operands' type; or null
    const void* res; int64_t res_ld; // added after the activation, of the operands' type; or null
    void* pre; int64_t pre_ld;       // receives the sum with its bias; or null
    const void* slope; int64_t slope_ld;   // the sum is multiplied by act'(slope); or null (act is applied otherwise)
    int act;
    bool accumulate;                 // out += ...
};
size_t linear_ws_bytes(int64_t rows, int64_t cols, int64_t K, bool a_in, bool b_in, int dtype);
hipError_t launch_linear(const LinearCall& c, void* ws, hipStream_t st);
size_t act_bwd_ws_bytes(int64_t N, int64_t K);
// g = dy act'(pre) (pre null: dy is read only, g may be null) and db (+)= column sums
hipError_t launch_act_bwd(int dtype, const void* pre, int64_t pre_ld, const void* dy, int64_t dy_ld, void* g, int64_t g_ld, void* db, int db_dtype,
                          bool accumulate, int64_t N, int64_t K, int act, void* ws, hipStream_t st);

hipError_t launch_adamw(const purine_adamw_desc& d, const purine_adamw_param* params, int n, int* done, hipStream_t st);

}  // namespace purine
