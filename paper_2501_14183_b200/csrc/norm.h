// What the parts of the norms share: parameters, launch interface of the element types.
#pragma once

#include "common.cuh"
#include "kernels.h"

namespace vardrop {

constexpr int kFwdPer = 16, kBwdPer = 8;  // elements of a row in a thread (backward the sums over tokens take as many registers again, or three times)
constexpr int kFwdPerFew = 10, kBwdPerFew = 6;
constexpr int kNormMaxC = 8192;

struct NormParams {
    const void *x, *y;
    const float *gate, *w_post, *b_post, *w_pre, *b_pre;
    const int32_t *sel_idx, *n_sel, *inv_idx;
    void *h, *u;
    float4* stats;
    const void *d_h, *d_u;
    void *dx, *dy;
    float* partial;                      // [2][slots, C], [2][CTAs, C]: sums over tokens of t o zy, t, du o zh, du
    int32_t* begin;                      // [B + 1], with a gate an instance: kept tokens of the instances ahead
    int B, N, C, pre, post, gate_rows, S;
    int slots;                           // rows of the first two sums
    int share, splits;                   // how tokens are shared out (NormShare); kSplit: CTAs of an instance
    float scale, eps, inv_c;
};

// How tokens are shared out among CTAs.
//   kFlat   neither a selection nor a gate tells instances apart: all tokens, by turns
//   kSplit  as many kept tokens in every instance: the same number of CTAs each, which take its tokens by turns
//   kRuns   as many as each instance keeps, one behind the other, in equal runs to the CTAs (7 x 4459 x 544 with 529 to 3195 kept took 108 us with CTAs per instance, 84 like this;
//           where turns can do it, they are the better: runs make 65536 x 1024, forward and backward, 245 us instead of 234, a call of one instance 4.3 instead of 3.2)
enum NormShare { kFlat, kSplit, kRuns };

inline int group_of(int C, int per) {
    int g = 8;
    while (g * per < C) g *= 2;
    return g;
}
// norm_bf16.cu, norm_fp16.cu, norm_fp32.cu
cudaError_t norm_launch_bf16(bool bwd, int grid, const NormParams& P, cudaStream_t s);
cudaError_t norm_launch_fp16(bool bwd, int grid, const NormParams& P, cudaStream_t s);
cudaError_t norm_launch_fp32(bool bwd, int grid, const NormParams& P, cudaStream_t s);

}  // namespace vardrop
