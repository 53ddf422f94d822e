// Router of pw_route_tokens: scores (softmax or sigmoid), a bias on the choice, groups of experts, the k best, gates.
//
//   p = softmax(l) or 1 / (1 + exp(-l))      key = p + bias      gate = p [/ sum of the chosen p] * scale
//
// One warp per token, expert e in lane e mod 32.  A row of logits is read once and 8 k bytes are written per token:
// launch, one round trip to memory and the chain of k selections bound it.  Which of two near scores is larger decides
// whole numbers, so the order is exact where it can be: without a bias and without sums of scores the keys are the
// logits themselves (both scores grow with the logit); otherwise p and the key are computed in 64 bits.
#include "pw_scaled.cuh"

namespace pw {

constexpr int kMaxRouteExperts = 256;
constexpr int kMaxRouteTopK = 32;

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* ids;
  float* gates;
  int64_t stride;
  int T, E, k, type, sigmoid, groups, top_groups, group_best, renorm;
  float scale;
};

// Order-preserving integers; -0 has been made +0, and no number maps to 0, which marks "not to be chosen".
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return u >> 63 ? ~u : u | (1ull << 63);
}
__device__ __forceinline__ double from_ordered(uint64_t u) {
  return __longlong_as_double((long long)(u >> 63 ? u & ~(1ull << 63) : ~u));
}
__device__ __forceinline__ uint32_t warp_max_key(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ uint64_t warp_max_key(uint64_t v) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return (uint64_t)hi << 32 | lo;
}

// The largest key of the warp and the lowest expert that has it (key 0: nothing is left).
template <int NS, class K>
__device__ __forceinline__ K warp_best(const K* key, int lane, int* expert) {
  K best = 0;
  int at = 0;
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (key[i] > best) {           // strictly: the lane's lowest expert stays
      best = key[i];
      at = lane + 32 * i;
    }
  const K top = warp_max_key(best);
  *expert = (int)__reduce_min_sync(0xffffffffu, best == top ? (uint32_t)at : 0xffffffffu);
  return top;
}

// NS = 32-expert strides a lane holds; WIDE: keys in 64 bits.
template <int NS, bool WIDE>
__global__ void __launch_bounds__(256) score_kernel(const RouteArgs a) {
  using K = typename std::conditional<WIDE, uint64_t, uint32_t>::type;
  grid_dep_sync();
  grid_dep_trigger();
  const int64_t t = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.T) return;
  float l[NS];
  K key[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int e = lane + 32 * i;
    float v = e < a.E ? load1(a.logits, t * a.stride + e, a.type) : -INFINITY;
    if (!(v > -INFINITY)) v = -INFINITY;          // NaN counts as masked
    l[i] = fminf(v, 3.402823466e38f) + 0.f;       // +infinity as the largest number; -0 as +0
  }
  float top = -INFINITY;
  double total = 1.0;                             // softmax: sum of exp(l - top) over the experts that are not masked
  if (!a.sigmoid) {
#pragma unroll
    for (int i = 0; i < NS; ++i) top = fmaxf(top, l[i]);
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  }
  if (WIDE) {
    double p[NS];
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      p[i] = l[i] > -INFINITY ? (a.sigmoid ? 1.0 / (1.0 + exp(-(double)l[i])) : exp((double)l[i] - (double)top)) : 0.0;
      sum += p[i];
    }
    if (!a.sigmoid) {
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      total = sum;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int e = lane + 32 * i;
      const double b = a.bias && e < a.E ? (double)a.bias[e] : 0.0;
      const double v = p[i] / total + b;
      key[i] = l[i] > -INFINITY && v > -INFINITY ? (K)ordered(v + 0.0) : (K)0;
    }
  } else {
    if (!a.sigmoid && !a.renorm) {
      // the denominator only scales the gates: 32 bits are enough for it
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) sum += l[i] > -INFINITY ? expf(l[i] - top) : 0.f;
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      total = sum;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) key[i] = l[i] > -INFINITY ? (K)ordered(l[i]) : (K)0;
  }
  if (a.groups > 1) {
    // Score of a group: its best key, or the sum of its best two (of the one that is not masked).  Lane g keeps
    // group g's; then the top_groups best groups are taken and the keys of the others cleared.
    const int per = a.E / a.groups;
    int group[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) group[i] = (lane + 32 * i) / per;
    K mine[NS];                                   // scores of the groups lane, lane + 32, ..
#pragma unroll
    for (int i = 0; i < NS; ++i) mine[i] = 0;
    for (int g = 0; g < a.groups; ++g) {
      K sub[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) sub[i] = group[i] == g ? key[i] : (K)0;
      int e;
      K score = warp_best<NS>(sub, lane, &e);
      if (WIDE && a.group_best == 2 && score) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
          if (lane + 32 * i == e) sub[i] = 0;
        int e2;
        const K second = warp_best<NS>(sub, lane, &e2);
        if (second) score = (K)ordered(from_ordered((uint64_t)score) + from_ordered((uint64_t)second) + 0.0);
      }
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (lane + 32 * i == g) mine[i] = score;
    }
    uint32_t keep = 0;                            // bit i: the group of my expert i stays
    for (int j = 0; j < a.top_groups; ++j) {
      int g;
      if (!warp_best<NS>(mine, lane, &g)) break;  // only groups without an expert are left
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        if (lane + 32 * i == g) mine[i] = 0;
        if (group[i] == g) keep |= 1u << i;
      }
    }
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (!((keep >> i) & 1u)) key[i] = 0;
  }
  // slot j in lane j: the j-th best expert and its logit
  int my_id = -1;
  float my_l = -INFINITY, first = -INFINITY;
  for (int j = 0; j < a.k; ++j) {
    int e;
    const bool any = warp_best<NS>(key, lane, &e) != 0;
    if (!any) break;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (lane + 32 * i == e) {
        key[i] = 0;
        v = l[i];
      }
    v = __shfl_sync(0xffffffffu, v, e & 31);
    if (j == 0) first = v;
    first = fmaxf(first, v);
    if (lane == j) {
      my_id = e;
      my_l = v;
    }
  }
  // Gates in 64 bits (one exponential per lane), rounded once.  Renormalised softmax gates need no denominator over
  // the row: exp(l - largest chosen l) over their sum.
  double p = 0.0;
  if (my_id >= 0) {
    if (a.sigmoid) p = 1.0 / (1.0 + exp(-(double)my_l));
    else p = exp((double)my_l - (double)(a.renorm ? first : top)) / (a.renorm ? 1.0 : total);
  }
  if (a.renorm) {
    double sum = p;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    p = sum > 0.0 ? p / sum : 0.0;
  }
  if (lane < a.k) {
    a.ids[t * a.k + lane] = my_id;
    a.gates[t * a.k + lane] = (float)(p * (double)a.scale);
  }
}

template <bool WIDE>
static cudaError_t launch_score(const RouteArgs& a, cudaStream_t s) {
  const int ns = (a.E + 31) / 32;
  void (*k)(RouteArgs) = ns <= 1 ? score_kernel<1, WIDE> : ns <= 2 ? score_kernel<2, WIDE> : ns <= 4 ? score_kernel<4, WIDE> : score_kernel<8, WIDE>;
  // four tokens per CTA: a batch of a few hundred tokens still reaches every SM
  return launch_dependent(k, dim3((unsigned)(((int64_t)a.T + 3) / 4)), dim3(128), 0, s, a);
}

}  // namespace pw

using namespace pw;

extern "C" pw_status pw_route_tokens(pw_ctx* ctx, const pw_routing* rule, const void* router_logits, int logits_type,
                                     int64_t logits_stride, const float* bias, int T, int32_t* topk_ids, float* gates,
                                     pw_stream stream) {
  if (!ctx || !rule || T < 0 || !type_ok(logits_type)) return PW_ERR_INVALID_ARG;
  const pw_routing& r = *rule;
  if (r.n_experts < 1 || r.n_experts > kMaxRouteExperts || r.top_k < 1 || r.top_k > kMaxRouteTopK) return PW_ERR_INVALID_ARG;
  if (r.score != PW_SCORE_SOFTMAX && r.score != PW_SCORE_SIGMOID) return PW_ERR_INVALID_ARG;
  if (r.n_groups < 1 || r.n_groups > r.n_experts || r.n_experts % r.n_groups || r.top_groups < 1 || r.top_groups > r.n_groups)
    return PW_ERR_INVALID_ARG;
  if (r.group_best != 1 && r.group_best != 2) return PW_ERR_INVALID_ARG;
  if (r.top_k > r.n_experts / r.n_groups * r.top_groups) return PW_ERR_INVALID_ARG;
  if (!(r.scale == r.scale) || r.scale - r.scale != 0.f) return PW_ERR_INVALID_ARG;
  if (T == 0) return PW_OK;
  if (!router_logits || !topk_ids || !gates) return PW_ERR_INVALID_ARG;
  if (T > 1 && logits_stride < r.n_experts) return PW_ERR_SHAPE;
  if (!is_aligned(router_logits, 16) || !is_aligned(bias, 16) || !is_aligned(topk_ids, 16) || !is_aligned(gates, 16))
    return PW_ERR_ALIGN;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  RouteArgs a{};
  a.logits = router_logits;
  a.bias = bias;
  a.ids = topk_ids;
  a.gates = gates;
  a.stride = logits_stride;
  a.T = T;
  a.E = r.n_experts;
  a.k = r.top_k;
  a.type = logits_type;
  a.sigmoid = r.score == PW_SCORE_SIGMOID;
  a.groups = r.top_groups == r.n_groups ? 1 : r.n_groups;   // every group stays: nothing to choose
  a.top_groups = r.top_groups;
  a.group_best = r.group_best;
  a.renorm = r.renormalize != 0;
  a.scale = r.scale;
  const bool wide = bias || (a.groups > 1 && r.group_best == 2);
  PW_CUDA_OK(wide ? launch_score<true>(a, stream) : launch_score<false>(a, stream));
  ctx->launches++;
  return PW_OK;
}
