// vie_e2m1_logits.h - the product of two e2m1 matrices (vie_e2m1_logits.cu).
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "vie_head.h"

namespace vie {

struct E2m1Product {
    const uint8_t *x_codes, *w_codes, *x_scales, *w_scales;
    const float *x_row_scales, *w_row_scales;
    void *out;
    int64_t ld, n, V;
    int d;
    // The kernel before this one on the stream has let this one start after all
    // before it had ended, and does not write W: W may be read at once.
    int w_ready;
    uint32_t *flag;
};

// out[i, v] = sum_j x[i, j] w[v, j] (vie_e2m1_logits).
cudaError_t launch_e2m1_logits(const E2m1Product &p, vie_dtype dtype, cudaStream_t stream);

}  // namespace vie
