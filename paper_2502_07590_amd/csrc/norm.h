// Layer norm of rows: what its kernels and their callers share.
#pragma once

#include "common.h"

namespace dsv {

// Strides in elements.  Row id = token * heads + head.
struct NormArgs {
    int32_t tokens, heads, n;
    float eps;
    int64_t x_row, x_head, y_row, y_head, dy_row, dy_head, dx_row, dx_head;
};
constexpr int kMaxNormWidth = 8192;  // 32 elements a lane of a block, and as many sums of dgamma and dbeta each, fit its registers; 64 do not
// wide: every row of every tensor begins on 16 bytes and n fills whole ones
dsv_status launch_norm_fwd(const NormArgs &a, int dtype, bool wide, const void *X, const void *gamma, const void *beta, void *Y, float *mean, float *rstd,
                           hipStream_t st);
int norm_bwd_blocks(const NormArgs &a, int dtype, bool wide);  // of the first kernel; each leaves two rows of n floats
dsv_status launch_norm_bwd(const NormArgs &a, int dtype, bool wide, const void *X, const void *gamma, const float *mean, const float *rstd, const void *dY,
                           void *dX, float *dgamma, float *dbeta, float *part, hipStream_t st);

}  // namespace dsv
