// The whole layer for few tokens in one kernel (pw_moe_forward_few, pw_moe_forward_few_routed).
//
// The layer call for batches takes five or six launches, and its kernels work on tiles of 128 weight rows; one token of a
// layer with 60 + 4 experts takes them 45 us, where the pages' bytes need 16.  Here one CTA per SM
//   - routes the tokens (every CTA does, it is cheaper than to wait for one that does) and lists the experts that have any,
//   - phase 1: units of 32 rows of an expert's gate and up blocks -> 32 values h = silu(gate) * up of its tokens,
//   - waits for all CTAs (the kernel is launched cooperatively, so they run at the same time), having asked for the first
//     weights of
//   - phase 2: units of 32 rows of the output and a part of all down blocks' columns; where the columns are in parts, the
//     CTA that finishes last of a unit's parts adds them up.
// Bound by the pages' bytes; the inner loop and what bounds it below that are in pw_stream.cuh.  Sums are in fp32 in an order
// that depends on the routing alone.
#include "pw_scaled.cuh"
#include "pw_stream.cuh"
#include "pw_topk.cuh"

namespace pw {

constexpr int kFewParts = 8;                      // most parts of the down blocks' columns
constexpr uint32_t kFewPolls = 1u << 22;          // about 3 s

struct FewArgs {
  const DevRow* rows;                             // of the layer
  const char* hidden;
  const float* logits;                            // or null: ids and gates
  const int32_t* ids;
  const float* gates;
  void* out;
  char* h;                                        // [pair][F] pieces
  float* parts;                                   // [part][T][H]
  int32_t* sync;                                  // arrivals, generation; from 64 on: finished parts of every 32 output rows
  int32_t* status;
  int32_t* seen;                                  // for the observation taps (or null): see few_observe_kernel
  int T, k, E, n_shared, H, F, out_type;
  int segs, pairs, n_parts;                       // room for active experts and for their (expert, token) pairs
  int table_bytes, ring_bytes;
};

// Tables in shared memory, built once per call.
struct SegPage {
  const char* codes;
  const char* bit1;
  const char* bit0;
};
struct FewTables {
  SegPage* page;                                  // [segs][3]
  float* gate;                                    // [pairs]
  float* own_gates;                               // [T * k]
  int32_t* own_ids;                               // [T * k]
  uint32_t* mask;                                 // [E] tokens of an expert
  int32_t* unit0;                                 // [segs + 1] first unit of phase 1, by rank
  int32_t* step0;                                 // [segs + 1] first step of phase 2, of the segment's first pass
  int32_t* count;                                 // active segments, pairs
  uint16_t* seg;                                  // [segs] expert, ascending
  uint16_t* off;                                  // [segs + 1] first pair
  uint16_t* order;                                // [segs] by weight of a unit of phase 1, heaviest first
  uint8_t* fmt;                                   // [segs][4]
  uint8_t* token;                                 // [pairs]
};
__host__ __device__ inline size_t few_tables(FewTables* t, char* base, int segs, int pairs, int Tk, int E) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char* at = base + o;
    o += (bytes + 15) & ~(size_t)15;
    return at;
  };
  FewTables v;
  v.page = reinterpret_cast<SegPage*>(take(sizeof(SegPage) * 3 * segs));
  v.gate = reinterpret_cast<float*>(take(4 * (size_t)pairs));
  v.own_gates = reinterpret_cast<float*>(take(4 * (size_t)Tk));
  v.own_ids = reinterpret_cast<int32_t*>(take(4 * (size_t)Tk));
  v.mask = reinterpret_cast<uint32_t*>(take(4 * (size_t)E));
  v.unit0 = reinterpret_cast<int32_t*>(take(4 * (size_t)(segs + 1)));
  v.step0 = reinterpret_cast<int32_t*>(take(4 * (size_t)(segs + 1)));
  v.count = reinterpret_cast<int32_t*>(take(16));
  v.seg = reinterpret_cast<uint16_t*>(take(2 * (size_t)segs));
  v.off = reinterpret_cast<uint16_t*>(take(2 * (size_t)(segs + 1)));
  v.order = reinterpret_cast<uint16_t*>(take(2 * (size_t)segs));
  v.fmt = reinterpret_cast<uint8_t*>(take(4 * (size_t)segs));
  v.token = reinterpret_cast<uint8_t*>(take((size_t)pairs));
  if (t) *t = v;
  return (o + 127) & ~(size_t)127;
}

__device__ __forceinline__ int passes_of(const FewTables& t, int a) { return (t.off[a + 1] - t.off[a] + kUnitCols - 1) / kUnitCols; }

// Teams of a CTA that has m units to do (at most four at a time): log2 of the warps of one.
__device__ __forceinline__ int few_team_shift(int m) { return m == 1 ? 4 : m == 2 ? 3 : 2; }
// Every kind of team has barriers of its own: a warp may be in the next one's while others are in this one's.
__device__ __forceinline__ void few_team_sync(int team, int ts) {
  asm volatile("bar.sync %0, %1;" ::"r"((ts == 2 ? 1 : ts == 3 ? 5 : 7) + team), "r"(32 << ts) : "memory");
}

// A unit of phase 1 for one warp.
struct GateUp {
  int a, pass, slice, kind, lo, n;                // segment, tokens, rows; the warp's block (PW_GATE, PW_UP) and steps
  int gates;                                      // warps of the team on the gate block
};
__device__ __forceinline__ GateUp gate_up_unit(const FewTables& t, int segs, int u, int groups, int ts, int member) {
  int r = 0;
  for (int half = 256; half; half >>= 1)
    if (r + half < segs && t.unit0[r + half] <= u) r += half;
  GateUp g;
  g.a = t.order[r];
  const int local = u - t.unit0[r], passes = passes_of(t, g.a);
  g.slice = passes == 1 ? local : local / passes;
  g.pass = local - g.slice * passes;
  const int warps = 1 << ts, sg = step_shift(t.fmt[4 * g.a + PW_GATE]), su = step_shift(t.fmt[4 * g.a + PW_UP]);
  // warps in proportion to the steps of the two blocks, one at least
  g.gates = max(1, min(warps - 1, (2 * (warps << sg) + (1 << sg) + (1 << su)) / (2 * ((1 << sg) + (1 << su)))));
  g.kind = member < g.gates ? PW_GATE : PW_UP;
  const int mine = member < g.gates ? member : member - g.gates, share = member < g.gates ? g.gates : warps - g.gates;
  const int steps = groups << (member < g.gates ? sg : su);
  g.lo = steps * mine / share;
  g.n = steps * (mine + 1) / share - g.lo;
  return g;
}

// Where value f of a row of pieces lies; c: the row's column in its pass.
__device__ __forceinline__ uint32_t piece_offset(int f, int c) {
  const uint32_t j = f & 127, s = j >> 4, w = (j & 15) >> 1;
  return (uint32_t)(f >> 7) * 256 + piece_at(2 * s + ((w & 3) >> 1), c) * 16 + (2 * (w & 1) + (w >> 2)) * 4 + (j & 1) * 2;
}

// Walks the steps lo .. hi of the list of all down blocks, (segment, pass) after (segment, pass).
struct DownRun {
  int a, pass, lo, n;
};
__device__ __forceinline__ bool down_run(const FewTables& t, int segs, int groups, int& at, int hi, int& hint, DownRun& d) {
  if (at >= hi) return false;
  while (t.step0[hint + 1] <= at) ++hint;
  d.a = hint;
  const int per = groups << step_shift(t.fmt[4 * hint + PW_DOWN]), local = at - t.step0[hint];
  d.pass = local / per;
  d.lo = local - d.pass * per;
  d.n = min(per - d.lo, hi - at);
  at += d.n;
  return true;
}

template <int XC, int STAGES>
__global__ void __launch_bounds__(kStreamThreads, 1) few_layer_kernel(const __grid_constant__ FewArgs p) {
  extern __shared__ __align__(128) char smem[];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  FewTables t;
  few_tables(&t, smem, p.segs, p.pairs, p.T * p.k, p.E);
  float* const sums = reinterpret_cast<float*>(smem + p.table_bytes);
  const int hg = p.H / kGroup, fg = p.F / kGroup;

  // ---- routing ----
  // phase 1: sums [16 warps], rings, staged operand; phase 2: sums [16 warps][T tokens], rings
  char* const ring1 = smem + p.table_bytes + kStreamWarps * kSumFloats * 4;
  float* const xsum = reinterpret_cast<float*>(ring1 + kStreamWarps * STAGES * kSlotOf<0>);
  char* const pieces = reinterpret_cast<char*>(xsum) + ((hg * 3 * p.T * 4 + 127) & ~127);
  for (int e = tid; e < p.E; e += kStreamThreads) t.mask[e] = 0;
  const int P0 = p.T * p.k;
  if (p.logits) {
    if (warp < p.T) route_token(p.logits, warp, p.E, p.k, t.own_ids, t.own_gates, lane);
  } else {
    for (int i = tid; i < P0; i += kStreamThreads) {
      int id = p.ids[i];
      if (id < -1 || id >= p.E) {
        atomicMax(p.status, (int)PW_ERR_INVALID_ARG);
        id = -1;
      }
      t.own_ids[i] = id;
      t.own_gates[i] = p.gates[i];
    }
  }
  {
    const int idle = p.logits && p.T <= 8 ? p.T : 0;   // the warps that route leave the staging to the others
    if (warp >= idle) stage_operand(p.hidden, (size_t)p.H * 2, p.T, p.T, 0, hg, p.H * 2, pieces, xsum, tid - 32 * idle, kStreamThreads - 32 * idle);
  }
  __syncthreads();
  for (int i = tid; i < P0; i += kStreamThreads) {
    const int e = t.own_ids[i];
    if (e >= 0) atomicOr(&t.mask[e], 1u << (i / p.k));
  }
  __syncthreads();
  if (warp == 0) {                                // experts with tokens, ascending, then the shared ones
    int segs = 0, pairs = 0;
    for (int base = 0; base < p.E; base += 32) {
      const uint32_t m = base + lane < p.E ? t.mask[base + lane] : 0;
      const int n = __popc(m);
      int incl = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      const uint32_t any = __ballot_sync(0xffffffffu, n > 0);
      if (n) {
        const int i = segs + __popc(any & ((1u << lane) - 1));
        t.seg[i] = (uint16_t)(base + lane);
        t.off[i] = (uint16_t)(pairs + incl - n);
      }
      segs += __popc(any);
      pairs += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane < p.n_shared) {
      t.seg[segs + lane] = (uint16_t)(p.E + lane);
      t.off[segs + lane] = (uint16_t)(pairs + lane * p.T);
    }
    if (lane == 0) {
      t.off[segs + p.n_shared] = (uint16_t)(pairs + p.n_shared * p.T);
      t.count[0] = segs + p.n_shared;
      t.count[1] = pairs + p.n_shared * p.T;
    }
  }
  __syncthreads();
  const int segs = t.count[0];
  for (int i = tid; i < segs * 3; i += kStreamThreads) {
    const int a = i / 3, u = i - 3 * a;
    const DevRow row = p.rows[t.seg[a] * 3 + u];
    t.page[i] = SegPage{static_cast<const char*>(row.codes), static_cast<const char*>(row.bit1), static_cast<const char*>(row.bit0)};
    t.fmt[4 * a + u] = (uint8_t)stream_format((int)row.bits, row.valid == 2);
  }
  for (int i = tid; i < segs * 16; i += kStreamThreads) {
    const int a = i >> 4, tok = i & 15, e = t.seg[a];
    if (e >= p.E) {
      if (tok < p.T) {
        t.token[t.off[a] + tok] = (uint8_t)tok;
        t.gate[t.off[a] + tok] = 1.f;
      }
    } else if (t.mask[e] >> tok & 1) {            // an expert that a token names twice takes it once, with both gates
      const int at = t.off[a] + __popc(t.mask[e] & ((1u << tok) - 1));
      float g = 0.f;
      for (int j = 0; j < p.k; ++j)
        if (t.own_ids[tok * p.k + j] == e) g = __fadd_rn(g, t.own_gates[tok * p.k + j]);
      t.token[at] = (uint8_t)tok;
      t.gate[at] = g;
    }
  }
  __syncthreads();
  for (int a = tid; a < segs; a += kStreamThreads) {
    auto weight = [&](int s) { return (int)stream_tile_bytes(t.fmt[4 * s + PW_GATE]) + (int)stream_tile_bytes(t.fmt[4 * s + PW_UP]); };
    const int mine = weight(a);
    int rank = 0;
    for (int o = 0; o < segs; ++o) {
      const int w = weight(o);
      rank += w > mine || (w == mine && o < a);
    }
    t.order[rank] = (uint16_t)a;
  }
  __syncthreads();
  if (warp < 2) {                                 // first units of phase 1 by rank; first steps of phase 2
    int32_t* first = warp == 0 ? t.unit0 : t.step0;
    int carry = 0;
    for (int base = 0; base < segs; base += 32) {
      const int i = base + lane, a = i < segs ? (warp == 0 ? t.order[i] : i) : 0;
      const int n = i < segs ? passes_of(t, a) * (warp == 0 ? p.F / kUnitRows : fg << step_shift(t.fmt[4 * a + PW_DOWN])) : 0;
      int incl = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      if (i < segs) first[i] = carry + incl - n;
      carry += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) first[segs] = carry;
  }
  __syncthreads();
  if (p.seen && blockIdx.x == 0) {                // what the taps' kernel wants to know
    for (int a = tid; a <= segs; a += kStreamThreads) {
      if (a < segs) p.seen[2 + a] = t.seg[a];
      p.seen[2 + p.segs + a] = t.off[a];
    }
    for (int i = tid; i < t.count[1]; i += kStreamThreads) {
      p.seen[3 + 2 * p.segs + i] = t.token[i];
      reinterpret_cast<float*>(p.seen)[3 + 2 * p.segs + p.pairs + i] = t.gate[i];
    }
    if (tid == 0) p.seen[0] = segs;
  }

  const Fixed fixed;
  Feed f;
  f.left = 0;
  Ring r;
  r.lane = lane;

  // ---- phase 1: gate and up ----
  {
    const int G = (int)gridDim.x, b = (int)blockIdx.x;
    const int units = t.unit0[segs];
    // the units, heaviest first, are dealt out in turn, the turns in alternating order; four at a time, each to a team
    const int mine = units / G + ((units / G) & 1 ? G - 1 - b < units % G : b < units % G);
    auto unit_of = [&](int i) { return i * G + (i & 1 ? G - 1 - b : b); };
    r.base = smem_u32(ring1) + warp * STAGES * kSlotOf<0>;
    r.slot = r.base;
    int next = 0;                                 // first of the four units that the feed looks at next
    auto more = [&]() -> bool {
      while (next < mine) {
        const int m = min(4, mine - next), ts = few_team_shift(m), team = warp >> ts;
        const int i = next + team;
        next += m;
        if (team >= m) continue;
        const GateUp g = gate_up_unit(t, segs, unit_of(i), hg, ts, warp & ((1 << ts) - 1));
        const SegPage& page = t.page[3 * g.a + g.kind];
        feed_codes(f, lane, page.codes, page.bit1, page.bit0, t.fmt[4 * g.a + g.kind], hg, g.slice, g.lo, g.lo + g.n);
        if (f.left) return true;
      }
      return false;
    };
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) {
      if (f.left || more()) ask_any<0, true, false>(f, r.base + i * kSlotOf<0>, lane);
      cp_commit();
    }
#pragma unroll 1
    for (int first = 0; first < mine; first += 4) {
      const int m = min(4, mine - first), ts = few_team_shift(m), team = warp >> ts, member = warp & ((1 << ts) - 1);
      if (team >= m) continue;
      const GateUp g = gate_up_unit(t, segs, unit_of(first + team), hg, ts, member);
      const int pair0 = t.off[g.a] + g.pass * kUnitCols, cols = min(kUnitCols, t.off[g.a + 1] - pair0);
      const int x = t.token[pair0 + min(lane >> 2, cols - 1)];
      const int t0 = t.token[pair0 + min(2 * (lane & 3), cols - 1)], t1 = t.token[pair0 + min(2 * (lane & 3) + 1, cols - 1)];
      float tot[2][4] = {};
      Operand o{smem_u32(pieces) + x * 256, smem_u32(xsum + t0), smem_u32(xsum + t1), p.T, (uint32_t)(x & 1) << 2, g.lo};
      walk<kAnyFormat, 0, STAGES>(fixed, t.fmt[4 * g.a + g.kind], g.n, f, r, o, tot, more);
      put_sums(sums + warp * kSumFloats, lane, tot);
      few_team_sync(team, ts);
      const float* set = sums + (team << ts) * kSumFloats;
      for (int i = member * 32 + lane; i < kUnitRows * cols; i += 32 << ts) {
        const int row = i & (kUnitRows - 1), col = i >> 5;
        const float* at = set + col * kSumPitch + row;
        float gate = 0.f, up = 0.f;
        for (int w = 0; w < 1 << ts; ++w) {
          const float v = at[w * kSumFloats];
          if (w < g.gates) gate = __fadd_rn(gate, v);
          else up = __fadd_rn(up, v);
        }
        // rounded to fp16 as the operand of the down block, like the layer call for batches: the fast exponential and
        // division (relative error ~1e-6) change nothing that survives the rounding
        const float h = __fmul_rn(__fdividef(gate, __fadd_rn(1.0f, __expf(-gate))), up);
        *reinterpret_cast<__half*>(p.h + (size_t)(pair0 + col) * p.F * 2 + piece_offset(g.slice * kUnitRows + row, col)) = __float2half_rn(h);
      }
      few_team_sync(team, ts);                    // the sums are written again
    }
  }
  cp_wait<0>();
  __syncthreads();

  // ---- phase 2: down ----
  constexpr int kSlot2 = kSlotOf<XC>;
  char* const ring2 = smem + p.table_bytes + kStreamWarps * p.T * kSumPitch * 4;
  r.base = smem_u32(ring2) + warp * STAGES * kSlot2;
  r.slot = r.base;
  {
    const int G = (int)gridDim.x, b = (int)blockIdx.x;
    const int units = p.H / kUnitRows * p.n_parts, steps = t.step0[segs];
    const int mine = units / G + (b < units % G);
    int next = 0, at = 0, end = 0, hint = 0, slice = 0;
    f.left = 0;
    // steps of part `part` for warp `member` of 1 << ts
    auto range = [&](int unit, int ts, int member, int& lo, int& hi) {
      const int64_t share = (int64_t)p.n_parts << ts, i = ((int64_t)(unit % p.n_parts) << ts) + member;
      lo = (int)(steps * i / share);
      hi = (int)(steps * (i + 1) / share);
    };
    auto more = [&]() -> bool {
      DownRun d;
      while (!down_run(t, segs, fg, at, end, hint, d)) {
        if (next >= mine) return false;
        const int m = min(4, mine - next), ts = few_team_shift(m), team = warp >> ts;
        const int unit = (next + team) * G + b;
        next += m;
        at = end = 0;
        if (team >= m) continue;
        range(unit, ts, warp & ((1 << ts) - 1), at, end);
        hint = 0;
        slice = unit / p.n_parts;
      }
      const SegPage& page = t.page[3 * d.a + PW_DOWN];
      const int pair0 = t.off[d.a] + d.pass * kUnitCols;
      feed_codes(f, lane, page.codes, page.bit1, page.bit0, t.fmt[4 * d.a + PW_DOWN], fg, slice, d.lo, d.lo + d.n);
      feed_operand(f, lane, p.h + (size_t)pair0 * p.F * 2, (uint32_t)p.F * 2, min(kUnitCols, t.off[d.a + 1] - pair0), d.lo);
      return true;
    };
    // codes first, then, when every CTA has written its values, the operands that go with them
#pragma unroll 1
    for (int i = 0; i < STAGES && (f.left || more()); ++i) ask_any<XC, true, false>(f, r.base + i * kSlot2, lane);
    bool together = true;
    if (tid == 0) {
      const int32_t generation = *reinterpret_cast<volatile int32_t*>(p.sync + 1);
      __threadfence();
      if (atomicAdd(p.sync, 1) == G - 1) {
        p.sync[0] = 0;
        __threadfence();
        atomicAdd(p.sync + 1, 1);
      } else {
        together = false;
        for (uint32_t n = 0; n < kFewPolls && !together; ++n) {
          int32_t now;
          asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(now) : "l"(p.sync + 1) : "memory");
          together = now != generation;
        }
        if (!together) atomicMax(p.status, (int)PW_ERR_TIMEOUT);
      }
      __threadfence();
    }
    if (!__syncthreads_and(together)) {
      cp_commit();
      cp_wait<0>();
      return;
    }
    {
      const Feed ahead = f;
      const int a0 = next, a1 = at, a2 = end, a3 = hint, a4 = slice;
      next = at = end = hint = slice = 0;
      f.left = 0;
#pragma unroll 1
      for (int i = 0; i < STAGES; ++i) {
        if (f.left || more()) ask_any<XC, false, true>(f, r.base + i * kSlot2, lane);
        cp_commit();
      }
      const char* x = f.x;                        // (codes and operand have come to the same step)
      f = ahead;
      f.x = x;
      next = a0, at = a1, end = a2, hint = a3, slice = a4;
    }
    float* const own = sums + warp * p.T * kSumPitch;
#pragma unroll 1
    for (int first = 0; first < mine; first += 4) {
      const int m = min(4, mine - first), ts = few_team_shift(m), team = warp >> ts, member = warp & ((1 << ts) - 1);
      if (team >= m) continue;
      const int unit = (first + team) * G + b;
      int lo, hi, where = 0;
      range(unit, ts, member, lo, hi);
      for (int i = lane; i < p.T * kSumPitch; i += 32) own[i] = 0.f;
      __syncwarp();
      DownRun d;
      while (down_run(t, segs, fg, lo, hi, where, d)) {
        const int fmt = t.fmt[4 * d.a + PW_DOWN], ls = step_shift(fmt);
        const int pair0 = t.off[d.a] + d.pass * kUnitCols, cols = min(kUnitCols, t.off[d.a + 1] - pair0);
        const int xc = min(lane >> 2, cols - 1);
        float tot[2][4] = {};
        Operand o{r.base + kStepCodes + kStepMeta + xc * (256 >> ls), 0, 0, 0, (uint32_t)(xc & 1) << 2, d.lo};
        walk<kAnyFormat, XC, STAGES>(fixed, fmt, d.n, f, r, o, tot, more);
#pragma unroll
        for (int c = 0; c < 2; ++c) {             // the tokens of a run are different ones: no two lanes meet
          const int col = 2 * (lane & 3) + c;
          if (col < cols) {
            const float g = t.gate[pair0 + col];
            float4* to = reinterpret_cast<float4*>(own + t.token[pair0 + col] * kSumPitch + 4 * (lane >> 2));
            float4 v = *to;
            v.x = __fadd_rn(v.x, __fmul_rn(g, tot[0][c]));
            v.y = __fadd_rn(v.y, __fmul_rn(g, tot[0][c + 2]));
            v.z = __fadd_rn(v.z, __fmul_rn(g, tot[1][c]));
            v.w = __fadd_rn(v.w, __fmul_rn(g, tot[1][c + 2]));
            *to = v;
          }
        }
        __syncwarp();
      }
      few_team_sync(team, ts);
      const float* set = sums + (team << ts) * p.T * kSumPitch;
      const int row0 = unit / p.n_parts * kUnitRows, part = unit % p.n_parts;
      for (int i = member * 32 + lane; i < kUnitRows * p.T; i += 32 << ts) {
        const int row = i & (kUnitRows - 1), tok = i >> 5;
        float v = 0.f;
        for (int w = 0; w < 1 << ts; ++w) v = __fadd_rn(v, set[(w * p.T + tok) * kSumPitch + row]);
        if (p.n_parts == 1) store1(p.out, (int64_t)tok * p.H + row0 + row, p.out_type, v);
        else p.parts[((size_t)part * p.T + tok) * p.H + row0 + row] = v;
      }
      if (p.n_parts > 1) {
        // the last of the parts to finish adds all of them up, in their order
        __threadfence();
        few_team_sync(team, ts);
        int last = 0;
        if (lane == 0 && member == 0) last = atomicAdd(p.sync + 64 + row0 / kUnitRows, 1) == p.n_parts - 1;
        if (lane == 0 && member == 0) reinterpret_cast<int32_t*>(sums + (size_t)(team << ts) * p.T * kSumPitch)[0] = last;
        few_team_sync(team, ts);
        last = *reinterpret_cast<volatile int32_t*>(sums + (size_t)(team << ts) * p.T * kSumPitch);
        if (last) {
          __threadfence();
          for (int i = member * 32 + lane; i < kUnitRows * p.T; i += 32 << ts) {
            const int row = i & (kUnitRows - 1), tok = i >> 5;
            float v = 0.f;
            for (int q = 0; q < p.n_parts; ++q) v = __fadd_rn(v, __ldcg(p.parts + ((size_t)q * p.T + tok) * p.H + row0 + row));
            store1(p.out, (int64_t)tok * p.H + row0 + row, p.out_type, v);
          }
          if (lane == 0 && member == 0) p.sync[64 + row0 / kUnitRows] = 0;
        }
      }
      few_team_sync(team, ts);                    // the sums are written again
    }
  }
  cp_wait<0>();
}

// ---- observation taps ----------------------------------------------------------------------------
// One warp per expert with tokens adds the call's pairs to the expert's accumulators (PW_OBS_*), from what CTA 0 of the
// layer's kernel has noted in `seen`: [0] active experts, [2 ..] their numbers, [2 + segs ..] first pairs, then the pairs'
// tokens and gates.  Sums in a fixed order.
__device__ __forceinline__ float square_sum(const uint4* row, int n, int lane) {
  float a = 0.f;
  for (int i = lane; i < n; i += 32) {
    const uint4 v = __ldcg(row + i);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 h = __half22float2(u32_as_h2(w[j]));
      a = fmaf(h.x, h.x, a);
      a = fmaf(h.y, h.y, a);
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
  return a;
}
__global__ void __launch_bounds__(256) few_observe_kernel(const int32_t* seen, int room, int pairs, const uint4* hidden, const uint4* h, int H, int F, int E,
                                                          const int32_t* ids, int Tk, float* __restrict__ acc) {
  const int a = (int)(blockIdx.x * blockDim.x + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (a >= seen[0]) return;
  const int seg = seen[2 + a], p0 = seen[2 + room + a], p1 = seen[2 + room + a + 1];
  const int32_t* tokens = seen + 3 + 2 * room;
  const float* gates = reinterpret_cast<const float*>(seen) + 3 + 2 * room + pairs;
  float sr = 0.f, srx = 0.f, srx2 = 0.f, mx = 0.f, srh = 0.f, srh2 = 0.f, mh = 0.f;
  for (int i = p0; i < p1; ++i) {
    const float r = gates[i], x2 = square_sum(hidden + (size_t)tokens[i] * (H / 8), H / 8, lane), h2 = square_sum(h + (size_t)i * (F / 8), F / 8, lane);
    const float nx = sqrtf(x2), nh = sqrtf(h2);
    sr += r;
    srx = fmaf(r, nx, srx);
    srx2 = fmaf(r, x2, srx2);
    mx = fmaxf(mx, nx);
    srh = fmaf(r, nh, srh);
    srh2 = fmaf(r, h2, srh2);
    mh = fmaxf(mh, nh);
  }
  int n = p1 - p0;
  if (ids && seg < E) {                           // a pair that is named twice counts twice
    n = 0;
    for (int i = lane; i < Tk; i += 32) n += ids[i] == seg;
#pragma unroll
    for (int d = 16; d; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
  }
  if (lane == 0) {
    float* o = acc + (size_t)seg * PW_OBS_FIELDS;
    o[PW_OBS_SUM_R] += sr;
    o[PW_OBS_PAIRS] += (float)n;
    o[PW_OBS_SUM_R_NX] += srx;
    o[PW_OBS_SUM_R_NX2] += srx2;
    o[PW_OBS_MAX_NX] = fmaxf(o[PW_OBS_MAX_NX], mx);
    o[PW_OBS_SUM_R_NH] += srh;
    o[PW_OBS_SUM_R_NH2] += srh2;
    o[PW_OBS_MAX_NH] = fmaxf(o[PW_OBS_MAX_NH], mh);
  }
}

// ---- host ----------------------------------------------------------------------------------------
typedef void (*FewKernel)(FewArgs);
struct FewVariant {
  int xc, stages;
  FewKernel kernel;
};
// The most stages that fit are the fastest; the operand rows of a slot go by the tokens.
static const FewVariant kFewVariants[] = {{2, 4, few_layer_kernel<2, 4>}, {4, 3, few_layer_kernel<4, 3>}, {8, 3, few_layer_kernel<8, 3>}, {8, 2, few_layer_kernel<8, 2>}};

static size_t few_smem(const FewArgs& a, const FewVariant& v) {
  const size_t first = (size_t)kStreamWarps * (kSumFloats * 4 + v.stages * kSlotOf<0>) + (((size_t)a.H / kGroup * 3 * a.T * 4 + 127) & ~(size_t)127) +
                       (size_t)a.T * a.H * 2;
  const size_t second = (size_t)kStreamWarps * ((size_t)a.T * kSumPitch * 4 + (size_t)v.stages * (kStepCodes + kStepMeta + 256 * v.xc));
  return a.table_bytes + (first > second ? first : second);
}

static pw_status moe_forward_few(pw_ctx* ctx, int layer, const void* hidden, const Routing& routing, int T, int top_k, const pw_page_table* table,
                                 void* out, int out_type, cudaStream_t stream) {
  if (!type_ok(out_type)) return PW_ERR_INVALID_ARG;
  const pw_status as = check_forward(ctx, layer, hidden, routing, T, top_k, table, out, PW_MODE_TENSOR);
  if (as != PW_OK) return as;
  const pw_config& c = ctx->cfg;
  const WsMap& w = ctx->ws;
  if (T > PW_FEW_TOKENS) return PW_ERR_INVALID_ARG;
  FewArgs a{};
  a.T = T;
  a.k = top_k;
  a.E = c.n_experts;
  a.n_shared = c.n_shared;
  a.H = c.hidden;
  a.F = c.ffn;
  a.out_type = out_type;
  a.segs = (c.n_experts < T * top_k ? c.n_experts : T * top_k) + c.n_shared;
  a.pairs = T * (top_k + c.n_shared);
  a.table_bytes = (int)few_tables(nullptr, nullptr, a.segs, a.pairs, T * top_k, c.n_experts);
  const FewVariant* v = nullptr;
  for (const FewVariant& one : kFewVariants)
    if (!v && one.xc >= (T < kUnitCols ? T : kUnitCols) && few_smem(a, one) <= kSmemLimit) v = &one;
  if (!v) return PW_ERR_SHAPE;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  if (!ctx->few_layer_ready) {
    for (const FewVariant& one : kFewVariants) PW_CUDA_OK(cudaFuncSetAttribute(one.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
    ctx->few_layer_ready = true;
  }
  char* b = ctx->base;
  a.rows = reinterpret_cast<const DevRow*>(b + w.table) + (size_t)layer * w.S * 3;
  a.hidden = static_cast<const char*>(hidden);
  a.logits = routing.logits;
  a.ids = routing.ids;
  a.gates = routing.gates;
  a.out = out;
  a.h = b + w.few_h;
  a.parts = reinterpret_cast<float*>(b + w.y);
  a.sync = reinterpret_cast<int32_t*>(b + w.few_sync);
  a.status = reinterpret_cast<int32_t*>(b + w.status);
  a.seen = ctx->obs_acc ? reinterpret_cast<int32_t*>(b + w.few_seen) : nullptr;
  // parts of the down blocks' columns: as few as give every SM work, in rounds that are nearly full
  const int slices = c.hidden / kUnitRows;
  double best = -1.;
  for (int parts = 1; parts <= kFewParts; ++parts) {
    const int rounds = (slices * parts + ctx->num_sms - 1) / ctx->num_sms;
    const double cost = (double)rounds / parts * (1. + 0.02 * parts);
    if (best < 0 || cost < best) best = cost, a.n_parts = parts;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctx->num_sms);
  cfg.blockDim = dim3(kStreamThreads);
  cfg.dynamicSmemBytes = few_smem(a, *v);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  PW_CUDA_OK(cudaLaunchKernelEx(&cfg, v->kernel, a));
  ctx->launches++;
  if (ctx->obs_acc) {
    few_observe_kernel<<<(a.segs + 7) / 8, 256, 0, stream>>>(a.seen, a.segs, a.pairs, static_cast<const uint4*>(hidden), reinterpret_cast<const uint4*>(a.h),
                                                            a.H, a.F, a.E, routing.logits ? nullptr : routing.ids, T * top_k,
                                                            ctx->obs_acc + (size_t)layer * w.S * PW_OBS_FIELDS);
    ctx->launches++;
    PW_CUDA_OK(cudaGetLastError());
  }
  return PW_OK;
}

}  // namespace pw

using namespace pw;

extern "C" pw_status pw_moe_forward_few(pw_ctx* ctx, int layer, const void* hidden, const float* logits, int T, int top_k, const pw_page_table* table,
                                        void* out, int out_type, pw_stream stream) {
  return moe_forward_few(ctx, layer, hidden, Routing{logits, nullptr, nullptr}, T, top_k, table, out, out_type, stream);
}

extern "C" pw_status pw_moe_forward_few_routed(pw_ctx* ctx, int layer, const void* hidden, const int32_t* topk_ids, const float* gates, int T, int top_k,
                                               const pw_page_table* table, void* out, int out_type, pw_stream stream) {
  return moe_forward_few(ctx, layer, hidden, Routing{nullptr, topk_ids, gates}, T, top_k, table, out, out_type, stream);
}
