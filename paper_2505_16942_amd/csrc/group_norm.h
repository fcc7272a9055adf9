// Launchers of group_norm.hip, called by maps_api.hip after its checks.
#pragma once
#include "rows.h"

// B items of P rows of C channels in G groups.  `parts` shares of `share` rows of an item, for its sums over rows.
struct GroupNormArgs {
    corr_dtype type;
    int act;
    int B, C, G;
    int64_t P;
    float eps;
    const void* x; int64_t x_stride;
    const float* weight; const float* bias;
    void* y;
    float* stats;                  // [B][G][2]: mean, 1 / spread (written by the forward pass, read by the gradient)
    const void* d_y; int64_t d_y_stride;
    void* d_x; float* d_weight; float* d_bias;
    float* part;                   // forward: [B][parts][C][2] {mean, squares about it}; gradient: [B][parts][2][C] {sum of dz hat, sum of dz}
    float* sums;                   // gradient: [B][2][C]
    int parts; int64_t share;
    bool past;                     // y, d_x are stored past the caches
    int held;                      // a workgroup holds a group: threads across its channels; else 0
};
// fills in parts and share
void group_norm_plan(GroupNormArgs& a, bool gradient);
hipError_t launch_group_norm(const GroupNormArgs& a, hipStream_t s);
hipError_t launch_group_norm_backward(const GroupNormArgs& a, hipStream_t s);
