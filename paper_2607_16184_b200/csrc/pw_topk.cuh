// The layer call's own routing rule, for the kernels that route tokens themselves.
#pragma once

#include <stdint.h>

namespace pw {

constexpr int kMaxExpertsPerLane = 8;  // E <= 256

// Routing of one token by one warp.  Slot j holds the j-th largest logit; equal logits: lower expert index first.
// (The logits may be written by the kernel directly ahead, pw_scaled_linear's: plain pointers all the way.)
template <int NS>   // NS = 32-expert strides a lane holds (1, 2, 4 or 8): the loops below cost in proportion
__device__ __forceinline__ void route_token_n(const float* logits, int token, int E, int k,
                                              int32_t* __restrict__ topk_ids, float* __restrict__ gates, int lane) {
  const float* l = logits + (size_t)token * E;
  float v[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int e = lane + 32 * i;
    v[i] = e < E ? fmaxf(l[e], -INFINITY) : -INFINITY;   // a NaN loses every comparison: without k others no expert would be found
  }
  uint32_t taken = 0;
  float l0 = 0.f, S = 0.f, myp = 0.f;
  int myid = 0;
  for (int j = 0; j < k; ++j) {
    float bv = -INFINITY;
    int bi = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int e = lane + 32 * i;
      const bool ok = e < E && !((taken >> i) & 1u);
      if (ok && (v[i] > bv || (v[i] == bv && e < bi))) {
        bv = v[i];
        bi = e;
      }
    }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
      const float ov = __shfl_xor_sync(0xffffffffu, bv, d);
      const int oi = __shfl_xor_sync(0xffffffffu, bi, d);
      if (ov > bv || (ov == bv && oi < bi)) {
        bv = ov;
        bi = oi;
      }
    }
    if ((bi & 31) == lane) taken |= 1u << (bi >> 5);
    if (j == 0) l0 = bv;
    const float p = expf(__fsub_rn(bv, l0));
    S = __fadd_rn(S, p);  // summed in slot order, identically on every lane
    if (lane == j) {
      myp = p;
      myid = bi;
    }
  }
  // k <= 32: lane j owns slot j
  if (lane < k) {
    topk_ids[(size_t)token * k + lane] = myid;
    gates[(size_t)token * k + lane] = __fdiv_rn(myp, S);
  }
}

__device__ __forceinline__ void route_token(const float* logits, int token, int E, int k,
                                            int32_t* __restrict__ topk_ids, float* __restrict__ gates, int lane) {
  if (E <= 32) route_token_n<1>(logits, token, E, k, topk_ids, gates, lane);
  else if (E <= 64) route_token_n<2>(logits, token, E, k, topk_ids, gates, lane);
  else if (E <= 128) route_token_n<4>(logits, token, E, k, topk_ids, gates, lane);
  else route_token_n<kMaxExpertsPerLane>(logits, token, E, k, topk_ids, gates, lane);
}

}  // namespace pw
