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
  // Logits in an order-preserving form: a warp's largest whole number is one instruction.  Both zeros are the same logit.
  uint32_t v[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int e = lane + 32 * i;
    // a NaN loses every comparison: without k others no expert would be found
    const uint32_t bits = __float_as_uint((e < E ? fmaxf(l[e], -INFINITY) : -INFINITY) + 0.f);
    v[i] = e < E ? bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u) : 0u;   // 0: no expert, or taken (no float has it)
  }
  float l0 = 0.f, S = 0.f, myp = 0.f;
  int myid = 0;
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    uint32_t top = v[0];
#pragma unroll
    for (int i = 1; i < NS; ++i) top = max(top, v[i]);
    top = __reduce_max_sync(0xffffffffu, top);
    int best = 0;
#pragma unroll
    for (int i = NS - 1; i >= 0; --i) {
      const uint32_t has = __ballot_sync(0xffffffffu, v[i] == top);
      if (has) best = 32 * i + __ffs(has) - 1;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (best == lane + 32 * i) v[i] = 0u;
    const float logit = __uint_as_float(top & 0x80000000u ? top ^ 0x80000000u : ~top);
    if (j == 0) l0 = logit;
    const float p = expf(__fsub_rn(logit, l0));
    S = __fadd_rn(S, p);  // summed in slot order, identically on every lane
    if (lane == j) {
      myp = p;
      myid = best;
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
