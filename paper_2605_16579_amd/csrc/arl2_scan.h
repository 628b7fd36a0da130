// The causal recurrence over tokens and its gradients: what the host side and the kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace arl2 {

struct ScanArgs {
    const void *q, *k, *v;    // [B][L][H][D] bf16
    const void *dout;         // likewise; the gradients only
    const float *la;          // [B][L][H] logarithms of the gates, or nullptr: all gates are one
    const int32_t *len;       // [B], or nullptr: L for all
    const float *S0;          // [B][H][D][D], or nullptr: zeros
    const float *dS;          // gradient of the last state, or nullptr: zeros
    void *out, *dq, *dk, *dv;
    float *S, *dS0, *dla;     // each may be nullptr
    void *workspace;
    int B, H, L, D;
    int normalise;            // rows of q and k are divided by sqrt(|row|^2 + eps)
    float eps;
};

// A sequence in `nseg` segments of `seg` blocks of 64 tokens, whose states meet in the workspace.
struct ScanPlan {
    int step;                 // by the kernel of few tokens
    int nseg, seg;
    size_t back, decay, dots, bytes;     // of the workspace: the states of the way back, the segments' decays, the parts of E; all
};
ScanPlan scan_plan(int B, int H, int L, int D, bool backward);

hipError_t launch_scan_fwd(const ScanArgs &a, const ScanPlan &p, hipStream_t stream);
hipError_t launch_scan_bwd(const ScanArgs &a, const ScanPlan &p, hipStream_t stream);

}  // namespace arl2
