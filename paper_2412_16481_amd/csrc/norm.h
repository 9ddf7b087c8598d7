// Internal interface between the C ABI (flash3d_api.hip) and the layer norm kernels (norm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace f3d {

constexpr int NORM_MAX_CHANNELS = 8192;

struct NormArgs {
    const void* x;
    const int32_t* row_in;    // null, or [n]: row p of the results belongs to x[row_in[p]]
    const float* gamma;       // null: ones
    const float* beta;        // null: zeros
    float eps;
    int n, c;
    int type;                 // F3D_BF16 | F3D_F16 | F3D_F32
    int wide;                 // rows and weights begin at multiples of 16 bytes, rows are a multiple long
    void* y;
    float* mean;              // [n], may be null
    float* rstd;
};

struct NormBwdArgs {
    const void* dy;
    const void* x;
    const int32_t* row_in;
    const float* mean;
    const float* rstd;
    const float* gamma;
    const void* residual;     // null, or added to the stored row
    int n, c;
    int type;
    int wide;
    void* dx;
    float* dgamma;            // null: not wanted
    float* dbeta;
    float* part;              // [blocks][2][c]
};

// the most workgroups that leave sums of their own in the workspace
int64_t norm_bwd_max_blocks(int64_t n, int c);
hipError_t norm_launch(const NormArgs& a, hipStream_t stream);
hipError_t norm_bwd_launch(const NormBwdArgs& a, hipStream_t stream);

}  // namespace f3d
