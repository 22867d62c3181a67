// The joint of two blocks (residual_norm.cu): r = rho x + gate * N_post(y), n = N_pre(r).
#pragma once
#include "internal.h"

namespace bigmac {

constexpr int kResNormMaxWidth = 8192;
constexpr int kResNormMaxRows = 1 << 30;    // row numbers and the step behind the last one are 32-bit

struct ResNorm {
    const bigmac_residual_norm_t* q;
    int T;
    bool vec;                          // every row of every tensor on a 16-byte boundary, d a multiple of 8
};

cudaError_t launch_residual_norm_forward(const ResNorm& a, cudaStream_t stream);
cudaError_t launch_residual_norm_backward(const ResNorm& a, float* partial, int accumulate, cudaStream_t stream);
// Most blocks of the backward pass: each leaves four vectors of d partial column sums.
int residual_norm_parts(int T, int d);

}  // namespace bigmac
