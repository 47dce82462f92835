// The one-kernel form of modse_orthogonalize for matrices with a short side.
#pragma once

#include "modse_internal.h"

namespace modse {

// powers of two the fp16 factors of the iteration are stored with (see orthogonalize.cu)
constexpr float kOrthScaleX = 4096.f, kOrthScaleA = 1024.f, kOrthScaleB = 1024.f;
constexpr int kOrthSmallMax = 128;     // longest shorter side of this form
constexpr int kOrthSmallBatch = 32;    // matrices of a launch

// X0 = G pre inv holds kOrthScaleX G / (|G| + eps).  One fp32 factor would overflow where |G| + eps is below 1e-35 (a matrix of
// zeros would give NaN for a tiny eps) and lose digits above 1e41, so a power of two goes ahead of it there.
struct StartScale { float pre, inv; };
__device__ __forceinline__ StartScale start_scale(double norm, float eps)
{
    const double by = (double)kOrthScaleX / (norm + (double)eps);
    const float pre = by > 1e30 ? 0x1p80f : by < 1e-30 ? 0x1p-80f : 1.f;
    return {pre, (float)(by / (double)pre)};
}

struct SmallMatrix {
    const void *g;
    __nv_bfloat16 *out;
    long long ld_g, ld_out;
    int rows, cols;
    float scale;
};
struct SmallArgs {
    SmallMatrix m[kOrthSmallBatch];
    float k[3];
    float eps;
    int steps;
    int head_ints;       // words of the workspace head to zero (none: head is null)
    int *head;
};

// How a matrix of this shape is held: its number of blocks (a power of two up to `most`, 8 or 16; 0: not for this form) and
// whether the step works in place (of sixteen blocks only).
struct SmallForm { int blocks; bool in_place; };
SmallForm orthogonalize_small_form(int rows, int cols, int most);
cudaError_t launch_orthogonalize_small(bool f32, const SmallArgs &a, int n, int most, cudaStream_t s);

}  // namespace modse
