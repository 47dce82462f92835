// What the two ways of modse_cross_entropy through the vocabulary share.
#pragma once

#include "dense_gemm.h"

namespace modse {

constexpr int kFewRows = 32;                     // at most, of the kernel that streams w past them
bool few_takes(int n, int d, int vocabulary);    // if that is the way to take
struct FewTiles { int height, count; };          // rows of a tile; each leaves one entry a row in LossEpilogue::part
FewTiles few_tiles(int vocabulary);
// Clears the status word and LossEpilogue::counter.
cudaError_t launch_loss_few(int n, int d, int vocabulary, const void *x, const void *w, const LossEpilogue &loss, int *status, cudaStream_t s);

}  // namespace modse
