// Queries and keys normalised and rotated by positions, and the gradients: what the host side and the kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "arl2_rope_plan.h"

namespace arl2 {

enum { kNormNone = 0, kNormHead = 1, kNormRow = 2 };

struct RopeArgs {
    const void *x[2], *w[2];     // queries [B][L][H][D] and keys [B][L][Hk][D]; weights or nullptr
    const void *dy[2];           // the gradients only
    void *y[2];                  // rotated rows; the gradients of x
    float *dw[2];                // or nullptr
    const int32_t *pos;          // [L][axes] or [B][L][axes]
    const int32_t *len;          // [B], or nullptr: L for all
    float *part;                 // partial sums of dw [workgroups][rows' width]
    int B, L, D, heads[2];
    int axes, pos_per_stream, halves, norm, f32;
    int pairs;                   // that are rotated, of D / 2
    float eps;
    uint8_t axis[64];            // of each pair
    double turns[64];            // of each pair for one step of its position
};

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream);
hipError_t launch_rope_bwd(const RopeArgs &a, hipStream_t stream);

}  // namespace arl2
