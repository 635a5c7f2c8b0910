// A block's gate, residual and norms of rows: what its kernels and their callers share.
#pragma once

#include "common.h"

namespace dsv {

// Strides from row to row (of the modulations: from segment to segment), in elements.
struct GatedNormArgs {
    const int32_t *cu;
    int32_t tokens, n, n_seg;
    int32_t rows;  // of a segment to a block
    float eps, residual;
    int32_t rms, post;
    int64_t x, y, h, z, dz, dh, dx, dy, gate, scale, shift, dgate, dscale, dshift;
};
struct GatedNormIn {
    const void *X, *Y, *gate, *scale, *shift;
};
dsv_status launch_gated_fwd(GatedNormArgs a, int dtype, bool wide, const GatedNormIn &in, void *Z, void *H, float4 *stats, hipStream_t st);
size_t gated_bwd_bytes(int64_t tokens, int n, int n_seg, int dtype);  // of the sums of segments that have several blocks
dsv_status launch_gated_bwd(GatedNormArgs a, int dtype, bool wide, const GatedNormIn &in, const float4 *stats, const void *dZ, const void *dH, void *dX, void *dY,
                            float *dgate, float *dscale, float *dshift, float *part, hipStream_t st);

}  // namespace dsv
