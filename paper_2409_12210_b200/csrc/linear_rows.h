// The weight-streaming form of modse_linear for a few tokens.
#pragma once

#include "dense_gemm.h"

namespace modse {

constexpr int kLinearRowsMax = 32;      // tokens up to which modse_linear streams the weights

cudaError_t launch_linear_rows(DenseType type, const void *x, const void *w, int T, int k, int n, const LinearEpilogue &lin,
                               int *status, cudaStream_t s);

}  // namespace modse
