// Router of pw_route_tokens: scores (softmax or sigmoid), a bias on the choice, groups of experts, the k best, gates.
//
//   p = softmax(l) or 1 / (1 + exp(-l))      key = p + bias      gate = p [/ sum of the chosen p] * scale
//
// One warp per token, expert e in lane e mod 32.  A row of logits is read once and 8 k bytes are written per token: a
// batch of a few hundred tokens costs a launch, one round trip to memory and a chain of warp-wide steps of 30 cycles each,
// a long prompt the instructions of the selections.  Which of two near scores is larger decides whole numbers, so the
// choice has to be that of exact keys: without a bias the keys are the logits themselves (both scores grow with the
// logit); otherwise they are computed in 32 bits together with a bound of their error.  Where two keys or two groups that
// decide anything are closer than that, the few experts concerned are computed in 64 bits, one per lane, and where that
// does not settle it either the whole token is.
// 4096 tokens x 256 experts in 8 groups: 9 to 11 us, by the near ties among them (everything in 64 bits 28.4, every
// unsettled token in 64 bits 13.5), one token 4.7; without groups 9.2, without bias either 4.9; 4.2 MB read at the copy rate: 0.7.
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
  int group_lanes, group_pitch;    // groups of experts in shared memory: see keep_groups
  uint32_t per_inverse;
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
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
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
  const uint32_t holders = __ballot_sync(0xffffffffu, best == top);
  if ((holders & (holders - 1)) == 0) *expert = __shfl_sync(0xffffffffu, at, __ffs((int)holders) - 1);
  else *expert = (int)__reduce_min_sync(0xffffffffu, best == top ? (uint32_t)at : 0xffffffffu);
  return top;
}
// What the choice of one token needs beyond its keys.
struct Chooser {
  int groups, per, top_groups, group_best, k, lane;
  int lanes, pitch;               // lanes that look through a group, words from a group's keys to the next one's
  uint32_t per_inverse;           // e / (experts of a group) = e * per_inverse >> 32 for every e < 256; 0: groups of one
  __device__ __forceinline__ int group_of(int e) const { return per_inverse ? (int)__umulhi((uint32_t)e, per_inverse) : e; }
};

// Clears the keys of all but the best top_groups groups; equal scores: lower group first.  `score(first, second)`: a
// group's score, as a key, of its two best keys (second 0: none, or only the best counts).
template <int NS, class K, class Score>
__device__ __forceinline__ void keep_groups_exactly(const Chooser& c, K* key, Score score) {
  // scores of the groups lane, lane + 32, ..
  K mine[NS];
  int group[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    group[i] = c.group_of(c.lane + 32 * i);
    mine[i] = 0;
  }
#pragma unroll 1
  for (int g = 0; g < c.groups; ++g) {
    K b1 = 0, b2 = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const K k = group[i] == g ? key[i] : (K)0;
      b2 = k > b1 ? b1 : k > b2 ? k : b2;
      b1 = k > b1 ? k : b1;
    }
    const K first = warp_max_key(b1);
    const uint32_t holders = __ballot_sync(0xffffffffu, b1 == first);
    const K second = c.group_best == 2 ? warp_max_key(c.lane == __ffs((int)holders) - 1 ? b2 : b1) : (K)0;
    const K s = first ? score(first, second) : (K)0;
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (c.lane + 32 * i == g) mine[i] = s;
  }
  uint32_t keep = 0;                            // bit i: the group of my expert i stays
  for (int j = 0; j < c.top_groups; ++j) {
    int g;
    if (!warp_best<NS>(mine, c.lane, &g)) break;   // only groups without an expert are left
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (c.lane + 32 * i == g) mine[i] = 0;
      if (group[i] == g) keep |= 1u << i;
    }
  }
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (!((keep >> i) & 1u)) key[i] = 0;
}

// The same for up to 32 groups and keys that may be off.  The keys change places by way of shared memory: `lanes` lanes
// (32 over the groups' number, rounded up to a power of two) look through a group and join their two best; `pitch` is an
// odd multiple of `lanes`, so that all of them read different banks.  A group's rank is the number of groups before it.
// `far(a, b)`: whether the score a is larger than b beyond doubt.  When that does not settle the last group that stays
// against the first that does not, `settle` decides on those in doubt (score and group of a lane, the two scores at the
// cut, the groups that stay as bits lanes * group); false: it could not.
template <int NS, class Score, class Far, class Settle>
__device__ __forceinline__ bool keep_groups(const Chooser& c, uint32_t* key, uint32_t* mem, Score score, Far far, Settle settle) {
  int bit[NS];                                  // of my expert's group
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int e = c.lane + 32 * i, g = c.group_of(e);
    bit[i] = g < c.groups ? g * c.lanes : 0;
    if (g < c.groups) mem[g * c.pitch + e - g * c.per] = key[i];
  }
  __syncwarp();
  const int shift = __ffs(c.lanes) - 1, g = c.lane >> shift, part = c.lane & (c.lanes - 1);
  uint32_t b1 = 0, b2 = 0;
  if (g < c.groups) {
#pragma unroll 4
    for (int o = part; o < c.per; o += c.lanes) {
      const uint32_t k = mem[g * c.pitch + o];
      b2 = max(b2, min(b1, k));
      b1 = max(b1, k);
    }
  }
  for (int d = 1; d < c.lanes; d <<= 1) {
    const uint32_t o1 = __shfl_xor_sync(0xffffffffu, b1, d), o2 = __shfl_xor_sync(0xffffffffu, b2, d);
    b2 = max(min(b1, o1), max(b2, o2));
    b1 = max(b1, o1);
  }
  const uint32_t s = b1 ? score(b1, c.group_best == 2 ? b2 : 0u) : 0u;
  int rank = 0;
#pragma unroll 4
  for (int h = 0; h < c.groups; ++h) {
    const uint32_t o = __shfl_sync(0xffffffffu, s, h << shift);
    rank += o > s || (o == s && h < g);
  }
  const bool stays = s && rank < c.top_groups;
  uint32_t kept = __ballot_sync(0xffffffffu, stays && part == 0);
  const uint32_t last = __reduce_min_sync(0xffffffffu, stays ? s : 0xffffffffu), next = __reduce_max_sync(0xffffffffu, stays ? 0u : s);
  bool sure = !next || far(last, next);         // (a group is left out: then top_groups stay)
  if (!sure) sure = settle(s, g, part == 0, last, next, &kept);
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (!((kept >> bit[i]) & 1u)) key[i] = 0;
  return sure;
}

// The experts of slots 0 .. k - 1 and their keys (slot j in lane j; -1: none left), by k searches for the largest key.
// Consumes the keys.  Equal keys: lower expert first.
template <int NS, class K>
__device__ __forceinline__ void take_best(const Chooser& c, K* key, int* slot, K* slot_key) {
  *slot = -1;
  for (int j = 0; j < c.k; ++j) {
    int e;
    const K best = warp_best<NS>(key, c.lane, &e);
    if (!best) break;
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (c.lane + 32 * i == e) key[i] = 0;
    if (c.lane == j) {
      *slot = e;
      *slot_key = best;
    }
  }
}

// The same from sorted lists: a lane sorts its keys once (NS = 8: 19 comparisons, of which each takes two instructions),
// after that a step looks at one key per lane instead of NS.  The keys are kept.  Returns
//   kSure  every key was `far` enough above the next one, the first that is not taken among them
//   kNear  some were not, but the `count` slots filled (k or more) are far above whatever follows: the choice is among them
//   kEqual equal keys followed one another (the slots are not valid), or 32 slots did not separate the choice
enum { kSure, kNear, kEqual };
template <int NS, class Far>
__device__ __forceinline__ int take_best_sorted(const Chooser& c, const uint32_t* key, Far far, int* slot, uint32_t* slot_key, int* count) {
  static_assert(NS == 4 || NS == 8, "sorting networks");
  uint32_t s[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) s[i] = key[i];
  auto order = [&](int x, int y) {
    const uint32_t hi = max(s[x], s[y]);
    s[y] = min(s[x], s[y]);
    s[x] = hi;
  };
  if constexpr (NS == 8) {
    order(0, 1), order(2, 3), order(4, 5), order(6, 7);
    order(0, 2), order(1, 3), order(4, 6), order(5, 7);
    order(1, 2), order(5, 6), order(0, 4), order(3, 7);
    order(1, 5), order(2, 6);
    order(1, 4), order(3, 6);
    order(2, 4), order(3, 5);
    order(3, 4);
  } else {
    order(0, 1), order(2, 3);
    order(0, 2), order(1, 3);
    order(1, 2);
  }
  int how = kSure, source = 0, j = 0;             // source: lane that had slot j's key
  uint32_t mine = 0, last = 0;
  for (;; ++j) {
    const uint32_t best = __reduce_max_sync(0xffffffffu, s[0]);
    if (!best) break;
    if (j > 0) {
      const bool apart = far(last, best);
      if (j >= c.k && apart) break;               // the first that is not taken
      if (!apart) how = last == best || how == kEqual ? kEqual : kNear;
      if (how == kEqual) break;
    }
    if (j == 32) {
      how = kEqual;
      break;
    }
    last = best;
    const int w = __ffs((int)__ballot_sync(0xffffffffu, s[0] == best)) - 1;
    if (c.lane == w) {
#pragma unroll
      for (int i = 0; i + 1 < NS; ++i) s[i] = s[i + 1];
      s[NS - 1] = 0;
    }
    if (c.lane == j) {
      source = w;
      mine = best;
    }
  }
  *slot = -1;
  *slot_key = mine;
  *count = j;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const uint32_t v = __shfl_sync(0xffffffffu, key[i], source);
    if (mine && v == mine) *slot = source + 32 * i;
  }
  return how;
}

// Puts the first `count` slots in the order of exact keys; equal keys: lower expert first.
__device__ __forceinline__ void order_slots(double key, int count, int lane, int* slot) {
  int rank = lane < count ? 0 : 32;
  for (int i = 0; i < count; ++i) {
    const double k = __shfl_sync(0xffffffffu, key, i);
    const int e = __shfl_sync(0xffffffffu, *slot, i);
    if (lane < count && (k > key || (k == key && e < *slot))) ++rank;
  }
  const int had = *slot;
  *slot = -1;
  for (int i = 0; i < count; ++i) {
    const int r = __shfl_sync(0xffffffffu, rank, i), e = __shfl_sync(0xffffffffu, had, i);
    if (r == lane) *slot = e;
  }
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
template <class F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// A token's logits: masked ones (NaN too) -infinity, +infinity as the largest number, -0 as +0.
__device__ __forceinline__ float tidy(float v) { return v > -INFINITY ? fminf(v, 3.402823466e38f) + 0.f : -INFINITY; }
template <int NS>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t t, int lane, float* l) {
  auto row = [&](auto* p) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int e = lane + 32 * i;
      l[i] = e < a.E ? to_f32(p[e]) : -INFINITY;
    }
  };
  if (a.type == PW_F32) row(static_cast<const float*>(a.logits) + t * a.stride);
  else if (a.type == PW_F16) row(static_cast<const __half*>(a.logits) + t * a.stride);
  else row(static_cast<const __nv_bfloat16*>(a.logits) + t * a.stride);
#pragma unroll
  for (int i = 0; i < NS; ++i) l[i] = tidy(l[i]);
}

// The experts' biases, all loads in flight together.
template <int NS>
__device__ __forceinline__ void load_bias(const RouteArgs& a, int lane, float* b) {
#pragma unroll
  for (int i = 0; i < NS; ++i) b[i] = a.bias && lane + 32 * i < a.E ? a.bias[lane + 32 * i] : 0.f;
}

// The choice with everything in 64 bits.
template <int NS>
__device__ __noinline__ int choose_exactly(const RouteArgs& a, int64_t t, const Chooser& c, float top) {
  float l[NS], b[NS];
  load_bias<NS>(a, c.lane, b);
  load_logits<NS>(a, t, c.lane, l);
  double total = 0.0;
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (l[i] > -INFINITY && !a.sigmoid) total += exp((double)l[i] - (double)top);
  total = warp_sum(total);
  auto p_of = [&](double v) { return a.sigmoid ? 1.0 / (1.0 + exp(-v)) : exp(v - (double)top) / total; };
  uint64_t key[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    double v = l[i];
    if (a.bias && l[i] > -INFINITY) v = p_of(v) + (double)b[i];
    key[i] = l[i] > -INFINITY && v > -INFINITY ? ordered(v + 0.0) : 0ull;
  }
  if (c.groups > 1)
    keep_groups_exactly<NS>(c, key, [&](uint64_t first, uint64_t second) {
      if (c.group_best == 1 || (!second && a.bias)) return first;
      const double u = from_ordered(first), v = from_ordered(second);
      return ordered((a.bias ? u + v : second ? p_of(u) + p_of(v) : p_of(u)) + 0.0);
    });
  int slot;
  uint64_t slot_key;
  take_best<NS>(c, key, &slot, &slot_key);
  return slot;
}

// Exact score (and bias) of one expert per lane, e < 0: none (0 then).  Without a bias softmax scores keep their common
// denominator.
template <int NS>
__device__ __noinline__ double exact_key(const RouteArgs& a, int64_t t, int lane, float top, int e) {
  double total = 1.0;
  if (!a.sigmoid && a.bias) {
    float l[NS];
    load_logits<NS>(a, t, lane, l);
    total = 0.0;
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (l[i] > -INFINITY) total += exp((double)l[i] - (double)top);
    total = warp_sum(total);
  }
  double key = 0.0;
  if (e >= 0) {
    const double v = tidy(load1(a.logits, t * a.stride + e, a.type));
    key = a.sigmoid ? 1.0 / (1.0 + exp(-v)) : exp(v - (double)top) / total;
    if (a.bias) key += (double)a.bias[e];
  }
  return key;
}

// CTAs on an SM.  Sixteen of the PLAIN kernel: the CTAs of a call come to their SMs while those of the call before are
// there, if both fit (4096 tokens x 256 experts 6.3 -> 4.9 us; at 12 CTAs an SM everything above 3552 tokens took 1.9 us
// more).  Seven of the other: 4096 tokens are one wave, and only choose_exactly would want more than 72 registers (five
// CTAs of 96 registers 11.7 us, eight 10.6, seven 10.1).
// NS = 32-expert strides a lane holds.  PLAIN: no bias and no groups, nothing but the logits decides (a program a third
// as long: one token 1.9 us instead of 2.4, most of it instructions on their way to the SM).
template <int NS, bool PLAIN>
__global__ void __launch_bounds__(128, PLAIN ? 16 : 7) score_kernel(const __grid_constant__ RouteArgs a) {
  grid_dep_sync();
  grid_dep_trigger();
  const int64_t t = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.T) return;
  float l[NS], b[PLAIN ? 1 : NS];
  if constexpr (!PLAIN) load_bias<NS>(a, lane, b);
  load_logits<NS>(a, t, lane, l);
  const Chooser c{a.groups, a.E / a.groups, a.top_groups, a.group_best, a.k, lane, a.group_lanes, a.group_pitch, a.per_inverse};
  // softmax: the largest logit, and the sum of exp(l - top) where something needs it
  float top = -INFINITY, total = 1.f;
  if (!a.sigmoid) {
#pragma unroll
    for (int i = 0; i < NS; ++i) top = fmaxf(top, l[i]);
    top = warp_max(top);
    if (!a.renorm || (!PLAIN && (a.bias || a.groups > 1))) {
      total = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) total += l[i] > -INFINITY ? expf(l[i] - top) : 0.f;
      total = warp_sum(total);
    }
  }
  int my_id;
  uint32_t my_key = 0;
  if constexpr (PLAIN) {
    uint32_t key[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) key[i] = l[i] > -INFINITY ? ordered(l[i]) : 0u;
    if constexpr (NS >= 4) {
      int count;
      if (take_best_sorted<NS>(c, key, [](uint32_t x, uint32_t y) { return x > y; }, &my_id, &my_key, &count) != kSure)
        take_best<NS>(c, key, &my_id, &my_key);
    } else {
      take_best<NS>(c, key, &my_id, &my_key);
    }
  } else {
    // (one exponential and one division for both scores: a branch for each key is twice the code to fetch)
    const float sign = a.sigmoid ? -1.f : 1.f, shift = a.sigmoid ? 0.f : -top;
    auto p_of = [&](float v) {
      const float e = __expf(fmaf(sign, v, shift));
      return __fdividef(a.sigmoid ? 1.f : e, a.sigmoid ? 1.f + e : total);
    };
    // Error of p in 32 bits, in half steps of 1.  The fast exponential of x is (2 + 1.173 |x|) steps off, the fast division 2.
    //   sigmoid: p (1 - p) (4 + 2.35 |v|) + p + 4 p <= 1 + 0.53 + 1 + 4, below 8
    //   softmax: with d = how far a logit is below the largest, a term e^-d is off by 4 + 2.35 d + d of it (exponential and
    //            rounding of its argument), at most 5.3 in all for d e^-d <= 0.37.  The denominator's terms are off by 2 + d
    //            each (expf), 2 + 3.4 of the sum (the mean of d over the terms is largest for 255 of them at 4.2), and 13
    //            additions; the division 4: below 28, taken as 32, all of it relative to p, which is 1 / total at most
    // With the bias's addition a key is off by less than (8 or 32 / total, + |key|) half steps; two keys decide when they are
    // further apart than both errors together.
    constexpr float kHalfStep = 5.9604645e-8f;
    uint32_t key[NS];
    float size = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      float v = l[i];
      if (a.bias) {
        const float k = p_of(v) + b[i];
        v = v > -INFINITY && k > -INFINITY ? k : -INFINITY;   // a bias that is no number: never chosen
        size = v > -INFINITY ? fmaxf(size, fabsf(v)) : size;
      }
      key[i] = v > -INFINITY ? ordered(v + 0.f) : 0u;
    }
    if (a.bias) size = warp_max(size);
    const float apart = 2.f * ((a.sigmoid ? 8.f : __fdividef(32.f, total)) + size) * kHalfStep;
    auto far_keys = [&](uint32_t x, uint32_t y) { return a.bias ? from_ordered(x) - from_ordered(y) > apart : x > y; };
    // without a bias the keys are exact, and so is a group's best; a sum of two scores never is
    bool sure = a.groups <= 32;
    if (sure && a.groups > 1) {
      __shared__ uint32_t mem[4][kMaxRouteExperts + 64];
      auto far_scores = [&](uint32_t x, uint32_t y) {
        if (!a.bias && a.group_best == 1) return true;
        const float u = from_ordered(x), v = from_ordered(y);
        return u - v > 2.f * apart + (fabsf(u) + fabsf(v)) * kHalfStep;
      };
      sure = keep_groups<NS>(c, key, mem[threadIdx.x >> 5], [&](uint32_t first, uint32_t second) -> uint32_t {
        if (a.group_best == 1) return first;
        const float u = from_ordered(first), v = second ? from_ordered(second) : 0.f;
        const float x = a.bias ? (second ? u + v : u) : (second ? p_of(u) + p_of(v) : p_of(u));
        return ordered(x + 0.f);
      }, far_scores, [&](uint32_t s, int g, bool first_lane, uint32_t last, uint32_t next, uint32_t* kept) {
        // A group beyond doubt above the last that stays is above all that are not larger than it: it stays; one as far
        // below the first that does not stay goes.  Of the others the exact scores decide, from the exact keys of their
        // two best, two lanes each, if it is beyond doubt which two those are.
        const bool in_doubt = s && first_lane && !far_scores(s, last) && !far_scores(next, s);
        uint32_t left = __ballot_sync(0xffffffffu, in_doubt);
        const uint32_t above = *kept & ~left;
        if (__popc(left) > 16) return false;
        int my_expert = -1, my_bit = 0, n = 0;
#pragma unroll 1
        for (; left; left &= left - 1, ++n) {
          const int bit = __ffs((int)left) - 1, group = __shfl_sync(0xffffffffu, g, bit);
          uint32_t k[NS], best[3];
          int e[3];
#pragma unroll
          for (int i = 0; i < NS; ++i) k[i] = c.group_of(lane + 32 * i) == group ? key[i] : 0u;
#pragma unroll
          for (int j = 0; j < 3; ++j) {
            best[j] = warp_best<NS>(k, lane, &e[j]);
#pragma unroll
            for (int i = 0; i < NS; ++i)
              if (lane + 32 * i == e[j]) k[i] = 0;
          }
          const int taken = a.group_best - 1;
          if (a.bias && best[taken] && best[taken + 1] && !far_keys(best[taken], best[taken + 1])) return false;
          if ((lane >> 1) == n) {
            my_bit = bit;
            my_expert = !(lane & 1) ? e[0] : a.group_best == 2 && best[1] ? e[1] : -1;
          }
        }
        double exact = exact_key<NS>(a, t, lane, top, my_expert);
        exact += __shfl_xor_sync(0xffffffffu, exact, 1);
        int before = 0;
        for (int j = 0; j < n; ++j) {
          const double o = __shfl_sync(0xffffffffu, exact, 2 * j);
          before += o > exact || (o == exact && j < (lane >> 1));
        }
        const bool goes_in = (lane >> 1) < n && before < a.top_groups - __popc(above);
        *kept = above | __reduce_or_sync(0xffffffffu, goes_in ? 1u << my_bit : 0u);
        return true;
      });
    }
    if (sure) {
      if constexpr (NS >= 4) {
        int count;
        const int how = take_best_sorted<NS>(c, key, far_keys, &my_id, &my_key, &count);
        if (how != kSure) {
          if (!a.bias) {
            take_best<NS>(c, key, &my_id, &my_key);
          } else if (how == kNear) {
            // the scores of a few experts, one per lane
            order_slots(exact_key<NS>(a, t, lane, top, lane < count ? my_id : -1), count, lane, &my_id);
            if (lane >= a.k) my_id = -1;
          } else {
            sure = false;
          }
        }
      } else {
        // (two strides: k searches are as short; one more for the first that is not taken)
        Chooser more = c;
        more.k = c.k + 1;
        uint32_t copy[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) copy[i] = key[i];
        my_id = -1;
        take_best<NS>(more, copy, &my_id, &my_key);
        const uint32_t next = __shfl_down_sync(0xffffffffu, my_id >= 0 ? my_key : 0u, 1);
        const bool decided = !a.bias || lane >= c.k || my_id < 0 || !next || (lane < 31 && far_keys(my_key, next));   // (no lane has slot 32)
        sure = __all_sync(0xffffffffu, decided);
        if (lane >= c.k) my_id = -1;
      }
    }
    if (!sure) my_id = choose_exactly<NS>(a, t, c, top);
  }
  // the logit of the chosen, slot j in lane j: the key itself where no bias is in it
  float my_l = -INFINITY;
  if (my_id >= 0) my_l = PLAIN ? from_ordered(my_key) : tidy(load1(a.logits, t * a.stride + my_id, a.type));
  // Gates.  Renormalised softmax gates need no denominator over the row: exp(l - largest chosen l) over their sum.  In 32
  // bits while the exponents are small: a gate is a weight of the experts' outputs, whose operands have 11 bits (off by
  // 5.7e-8 of the gates' norm for 256 tokens x 64 experts, 2.4e-8 if everything is in 64 bits).  Else in 64 bits, where
  // neither the rounding of a large exponent nor an underflowing score of a sum of underflowing scores is lost; the
  // softmax's denominator over the row stays the sum in 32 bits, of positive terms, off by 13 roundings and their own.
  const bool chosen = my_id >= 0;
  const float base = a.sigmoid ? 0.f : a.renorm ? warp_max(my_l) : top;
  const float d = chosen ? my_l - base : 0.f;
  float gate;
  if (__any_sync(0xffffffffu, fabsf(d) > 16.f)) {
    double p = 0.0;
    if (chosen) {
      if (a.sigmoid) p = 1.0 / (1.0 + exp(-(double)my_l));
      else p = exp((double)my_l - (double)base) / (a.renorm ? 1.0 : (double)total);
    }
    if (a.renorm) {
      const double sum = warp_sum(p);
      p = sum > 0.0 ? p / sum : 0.0;
    }
    gate = (float)(p * (double)a.scale);
  } else {
    float p = 0.f;
    if (chosen) {
      const float e = expf(a.sigmoid ? -d : d);
      p = a.sigmoid ? __fdiv_rn(1.f, 1.f + e) : a.renorm ? e : __fdiv_rn(e, total);
    }
    if (a.renorm) {
      const float sum = warp_sum(p);
      p = sum > 0.f ? __fdiv_rn(p, sum) : 0.f;
    }
    gate = p * a.scale;
  }
  if (lane < a.k) {
    a.ids[t * a.k + lane] = my_id;
    a.gates[t * a.k + lane] = gate;
  }
}

static cudaError_t launch_score(const RouteArgs& a, cudaStream_t s) {
  const int ns = (a.E + 31) / 32, n = ns <= 1 ? 0 : ns <= 2 ? 1 : ns <= 4 ? 2 : 3;
  static void (*const table[2][4])(RouteArgs) = {{score_kernel<1, false>, score_kernel<2, false>, score_kernel<4, false>, score_kernel<8, false>},
                                                 {score_kernel<1, true>, score_kernel<2, true>, score_kernel<4, true>, score_kernel<8, true>}};
  void (*k)(RouteArgs) = table[!a.bias && a.groups == 1][n];
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
  const int per = r.n_experts / a.groups;
  a.group_lanes = 32;
  while (a.group_lanes > 1 && a.group_lanes * a.groups > 32) a.group_lanes /= 2;
  a.group_pitch = ((per + a.group_lanes - 1) / a.group_lanes | 1) * a.group_lanes;   // groups <= 32: below 256 + 64 words in all
  a.per_inverse = per > 1 ? (uint32_t)((0x100000000ull + per - 1) / per) : 0u;   // exact for numerators below 256
  a.group_best = r.group_best;
  a.renorm = r.renormalize != 0;
  a.scale = r.scale;
  PW_CUDA_OK(launch_score(a, stream));
  ctx->launches++;
  return PW_OK;
}
