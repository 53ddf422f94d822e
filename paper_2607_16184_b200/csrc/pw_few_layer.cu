// The whole layer for few tokens in one kernel (pw_moe_forward_few, pw_moe_forward_few_routed).
//
// The layer call for batches takes five or six launches, and its kernels work on tiles of 128 weight rows; one token of a
// layer with 60 + 4 experts takes them 40 us, where the pages' bytes need 16.  Here (28 to 31 us) one CTA per SM
//   - routes the tokens (every CTA does, it is cheaper than to wait for one that does) and lists the experts that have any;
//     meanwhile it brings the tokens into shared memory and asks the L2 cache for the shared experts,
//   - phase 1: units of 32 rows of an expert's gate and up blocks -> 32 values h = silu(gate) * up of its tokens,
//   - waits for all CTAs (the kernel is launched cooperatively, so they run at the same time); each of its warps has gone on
//     by then to ask for its first weights of
//   - phase 2: units of 32 rows of the output and a part of all down blocks' columns; where the columns are in parts, the
//     CTA that finishes last of a unit's parts adds them up.
// Bound by the pages' bytes: phase 1 runs at the HBM rate (one token of the 8 x (4096, 14336) layer at mixed bitwidths, 350 MB:
// 233 MB in 31 us of 72), phase 2 of narrow formats by its instructions (a 4-bit step of 2 KB: about 300 of a warp), where
// the hidden size gives 128 of the 148 SMs a unit.  Besides that a call takes about 1 us to launch, 3 to route and make its
// tables (5 for 16 tokens of 128 experts), 2 for its first copies and 2.5 between the phases.  Asking the L2 cache for more of phase 2 while waiting was
// slower (one token of the 60 + 4 expert layer 30.3 us against 28.9).  Sums are in fp32 in an order that depends on the routing
// alone.
#include "pw_scaled.cuh"
#include "pw_stream.cuh"
#include "pw_topk.cuh"

namespace pw {

constexpr int kFewParts = 8;                      // most parts of the down blocks' columns
// The operand h of the down blocks is kept in two fp16 numbers: the nearest one, and what that leaves, times 2^11, so that
// the second has as many bits as the first wherever the first has all of its own: 22 bits of h, or 2^-36 where h is below
// 2^-14 (without the factor everything below 2^-25 was lost, 1.7e-4 of an h of 1e-4).  They stand in neighbouring columns of
// the matrix instructions, which most experts leave empty: an expert of more than four tokens takes a second pass.  (One
// number would save that, and cost 2e-4 of the output's norm: 16 tokens of the 8-expert layer 147 us against 177, of the
// 60 + 4 expert layer 79 against 88; 8 tokens 131 and 132, 51 and 55.)
constexpr int kHalves = 2;
constexpr int kDownCols = kUnitCols / kHalves;    // tokens of a pass of the second phase
constexpr float kRestUp = 2048.f, kRestDown = 1.f / kRestUp;
constexpr int kFewRouters = 8;                    // warps that route (2 / 4 / 8 / 12: 16 tokens of 128 + 1 experts 64.5 / 62.1 / 60.9 / 63.7 us)
// bytes of shared experts that are asked for while the tokens are routed: 2.5 us (none / 16 MB / 48 MB, 60 + 4 experts: one token
// 28.8 / 28.9 / 31.1 us, four 40.2 / 39.5 / 41.2)
constexpr size_t kFewAhead = 16 << 20;
constexpr uint32_t kFewAheadPiece = 4096;
constexpr uint32_t kFewPolls = 1u << 22;          // of the meeting's counter: about 3 s
constexpr uint32_t kFewPollsTest = 6400;          // about 4 ms, for the test of a wait that runs out (pw_debug_set_wait)

struct FewArgs {
  const DevRow* rows;                             // of the layer
  const char* hidden;
  const float* logits;                            // or null: ids and gates
  const int32_t* ids;
  const float* gates;
  void* out;
  char* h;                                        // [pair][kHalves][F] pieces
  float* parts;                                   // [part][T][H]
  int32_t* sync;                                  // arrivals; from 64 on: finished parts of every 32 output rows
  uint32_t polls, hook;                           // limit of the wait; test hook: the last CTA arrives when its own wait has run out
  int32_t* status;
  int32_t* seen;                                  // for the observation taps (or null): see few_observe_kernel
  int T, k, E, n_shared, H, F, out_type;
  int segs, pairs;                                // room for active experts and for their (expert, token) pairs
  int n_parts;                                    // parts of the down blocks' columns
  uint32_t per_part;                              // 2^32 / n_parts, rounded up
};

// Tables in shared memory, built once per call.
struct SegPage {
  const char* codes;
  const char* bit1;
  const char* bit0;
};
// at fixed places, so that a look into one is one instruction.  Two sizes: a few tokens of most layers, and every call.
template <int SEGS, int PAIRS, int CHOICES>
struct FewTables {
  static constexpr int kSegs = SEGS, kPairs = PAIRS, kChoices = CHOICES;
  SegPage page[SEGS * 3];
  float gate[PAIRS];
  float own_gates[CHOICES];                       // [T * k]
  int32_t own_ids[CHOICES];
  uint32_t mask[256];                             // tokens of an expert, and above them (16 bits) its first pair
  int32_t unit0[SEGS + 1];                        // first unit of phase 1, by rank
  int32_t step0[SEGS + 1];                        // first step of phase 2, of the segment's first pass
  uint2 weight[SEGS];                             // by which they are ordered, heaviest first, and their passes: see make_tables
  int32_t count[2];                               // active segments, pairs
  uint32_t done;                                  // warps that are through with phase 1
  uint16_t seg[SEGS];                             // expert, ascending
  uint16_t off[SEGS + 1];                         // first pair
  uint16_t order[SEGS];                           // shared experts first, then by weight, heaviest first
  uint8_t fmt[SEGS * 4];
  uint8_t token[PAIRS];
};
typedef FewTables<48, 96, 64> FewSmall;
typedef FewTables<256 + 16, PW_FEW_TOKENS * (32 + 16), PW_FEW_TOKENS * 32> FewAll;
template <class TAB>
constexpr int kTableBytes = (int)((sizeof(TAB) + 127) & ~(size_t)127);

template <class TAB>
__device__ __forceinline__ int passes_of(const TAB& t, int a) { return (t.off[a + 1] - t.off[a] + kUnitCols - 1) / kUnitCols; }

// A warp's team in a CTA that has m units to do, at most four at a time: the unit it takes, its first warp, log2 of its
// warps.  Of three units the first, which is the heaviest, has half of the warps.
struct Team {
  int unit, first, shift;
};
__device__ __forceinline__ Team few_team(int m, int warp) {
  Team w;
  w.shift = m == 1 ? 4 : m == 2 || (m == 3 && warp < 8) ? 3 : 2;
  w.first = warp >> w.shift << w.shift;
  w.unit = (warp >> w.shift) - (m == 3 && warp >= 8);
  return w;
}
// Every kind of team has barriers of its own: a warp may be in the next one's while others are in this one's.
__device__ __forceinline__ void few_team_sync(const Team& w) {
  asm volatile("bar.sync %0, %1;" ::"r"((w.shift == 2 ? 1 : w.shift == 3 ? 5 : 7) + (w.first >> w.shift)), "r"(32 << w.shift) : "memory");
}

// A unit of phase 1 for one warp.
struct GateUp {
  int a, pass, slice, kind, lo, n;                // segment, tokens, rows; the warp's block (PW_GATE, PW_UP) and steps
  int gates;                                      // warps of the team on the gate block
};
__constant__ uint32_t kPerShare[17] = {0, 1u << 20, 524289, 349526, 262145, 209716, 174763, 149797, 131073, 116509, 104858, 95326, 87382, 80660, 74899, 69906, 65537};
// How many of the n ascending numbers are at most v, by a warp.
__device__ __forceinline__ int count_up_to(const int32_t* number, int n, int v, int lane) {
  int c = 0;
#pragma unroll 1
  for (int base = 0; base < n; base += 32) c += __popc(__ballot_sync(0xffffffffu, base + lane < n && number[base + lane] <= v));
  return c;
}
template <class TAB>
__device__ __forceinline__ GateUp gate_up_unit(const TAB& t, int segs, int u, int groups, int ts, int member, int lane) {
  const int r = count_up_to(t.unit0 + 1, segs, u, lane);
  GateUp g;
  g.a = t.order[r];
  const int local = u - t.unit0[r], passes = passes_of(t, g.a);
  g.slice = passes == 1 ? local : local >> 1;     // (at most two passes)
  g.pass = passes == 1 ? 0 : local & 1;
  const int warps = 1 << ts, sg = step_shift(t.fmt[4 * g.a + PW_GATE]), su = step_shift(t.fmt[4 * g.a + PW_UP]);
  // warps in proportion to the steps of the two blocks, one at least
  const int both = (1 << sg) + (1 << su);
  g.gates = max(1, min(warps - 1, (int)((((warps << sg) + (both >> 1)) * kPerShare[both]) >> 20)));
  g.kind = member < g.gates ? PW_GATE : PW_UP;
  const int mine = member < g.gates ? member : member - g.gates, share = member < g.gates ? g.gates : warps - g.gates;
  const uint32_t steps = (uint32_t)groups << (member < g.gates ? sg : su);
  // steps * mine / share, rounded down: the product is below 2^20 / share for every block a context may have
  g.lo = (int)((uint64_t)(steps * mine) * kPerShare[share] >> 20);
  g.n = (int)((uint64_t)(steps * (mine + 1)) * kPerShare[share] >> 20) - g.lo;
  return g;
}

// Where value f of a row of pieces lies; c: the row's column in its pass.
__device__ __forceinline__ uint32_t piece_offset(int f, int c) {
  const uint32_t j = f & 127, s = j >> 4, w = (j & 15) >> 1;
  return (uint32_t)(f >> 7) * 256 + piece_at(2 * s + ((w & 3) >> 1), c) * 16 + (2 * (w & 1) + (w >> 2)) * 4 + (j & 1) * 2;
}

// Walks the steps lo .. hi of the list of all down blocks, (segment, pass) after (segment, pass); at most four passes of a
// segment, of kDownCols tokens.
struct DownRun {
  int a, pass, lo, n;
};
template <class TAB>
__device__ __forceinline__ bool down_run(const TAB& t, int groups, int& at, int hi, int& hint, DownRun& d) {
  if (at >= hi) return false;
#pragma unroll 1
  while (t.step0[hint + 1] <= at) ++hint;
  d.a = hint;
  const int per = groups << step_shift(t.fmt[4 * hint + PW_DOWN]);
  d.pass = 0;
  d.lo = at - t.step0[hint];
#pragma unroll 1
  for (; d.lo >= per; d.lo -= per) ++d.pass;
  d.n = min(per - d.lo, hi - at);
  at += d.n;
  return true;
}

// The tables of a call from its routing (own_ids, own_gates, and every expert's tokens in mask), by the first kFewRouters
// warps.  rows: the layer's, in shared memory.
__device__ __forceinline__ void routers_sync() { asm volatile("bar.sync 8, %0;" ::"n"(32 * kFewRouters) : "memory"); }
template <class TAB>
__device__ __forceinline__ void make_tables(const FewArgs& p, TAB& t, const DevRow* rows, int fg, int warp, int lane) {
  // Segment a: expert e with n tokens, pairs first .. first + n.  Its weight: shared or not, the bytes of a tile of its gate
  // and its up block, no two alike; beside it one in the upper half, for counting, and its passes.
  auto put = [&](int a, int e, int n, int first) {
    uint32_t tiles = 0, shift = 0;
    t.seg[a] = (uint16_t)e;
    t.off[a] = (uint16_t)first;
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      const DevRow& row = rows[e * 3 + u];
      const bool planes = row.valid == 2;
      if (u == PW_DOWN) shift = row.bits == 16 ? 2 : row.bits == 8 ? 1 : 0;
      else tiles += planes ? kPlaneTopTile : row.bits == 16 ? 32768 : row.bits * 2048 + 512;
      t.page[3 * a + u] = SegPage{static_cast<const char*>(row.codes), static_cast<const char*>(row.bit1), static_cast<const char*>(row.bit0)};
      t.fmt[4 * a + u] = (uint8_t)stream_format((int)row.bits, planes);
    }
    const uint32_t passes = (uint32_t)(n + kUnitCols - 1) / kUnitCols;
    t.weight[a] = make_uint2((e < p.E ? 0u : 1u << 31) | tiles << 9 | (511u - a), 1u << 16 | passes);
    t.step0[a] = (int32_t)((uint32_t)(n + kDownCols - 1) / kDownCols << shift);   // (summed up below)
  };
  // experts with tokens, ascending, then the shared ones: every warp counts all, and makes the segments of some
  int segs = 0, pairs = 0;
#pragma unroll 1
  for (int base = 0; base < p.E; base += 32) {
    const uint32_t m = base + lane < p.E ? t.mask[base + lane] & 0xffffu : 0;   // (another warp may have set the upper half)
    const uint32_t any = __ballot_sync(0xffffffffu, m != 0);
    if (!any) continue;
    const int n = __popc(m);                      // <= 16
    if ((base >> 5) % kFewRouters == warp) {
      const uint32_t below = (1u << lane) - 1;
      int before = pairs;
#pragma unroll
      for (int bit = 0; bit < 5; ++bit) before += __popc(__ballot_sync(0xffffffffu, n >> bit & 1) & below) << bit;
      if (n) {
        put(segs + __popc(any & below), base + lane, n, before);
        t.mask[base + lane] = m | (uint32_t)before << 16;
      }
    }
    segs += __popc(any);
    pairs += (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
  }
  if (warp == kFewRouters - 1) {
    if (lane < p.n_shared) put(segs + lane, p.E + lane, p.T, pairs + lane * p.T);
    if (lane == 0) {
      t.off[segs + p.n_shared] = (uint16_t)(pairs + p.n_shared * p.T);
      t.count[0] = segs + p.n_shared;
      t.count[1] = pairs + p.n_shared * p.T;
    }
  }
  routers_sync();
  // the experts' tokens, ascending; an expert that a token names twice takes it once, with both gates
  const int first = 32 * warp + lane, last = 32 * kFewRouters - 1 - first;
#pragma unroll 1
  for (int i = last; i < p.T * p.k; i += 32 * kFewRouters) {
    const int e = t.own_ids[i], tok = i / p.k, j0 = tok * p.k;
    if (e < 0) continue;
    const uint32_t m = t.mask[e];
    bool again = false;
    float g = 0.f;
#pragma unroll 1
    for (int j = j0; j < j0 + p.k; ++j)
      if (t.own_ids[j] == e) {
        again |= j < i;
        g = __fadd_rn(g, t.own_gates[j]);
      }
    if (again) continue;
    const int at = (int)(m >> 16) + __popc(m & ((1u << tok) - 1));
    t.token[at] = (uint8_t)tok;
    t.gate[at] = g;
  }
#pragma unroll 1
  for (int i = last; i < p.n_shared * p.T; i += 32 * kFewRouters) {
    t.token[pairs + i] = (uint8_t)(i % p.T);
    t.gate[pairs + i] = 1.f;
  }
  segs += p.n_shared;
  // first steps of phase 2
  if (warp == 1) {
    int carry = 0;
#pragma unroll 1
    for (int base = 0; base < segs; base += 32) {
      const int i = base + lane, n = i < segs ? t.step0[i] : 0;
      int incl = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      if (i < segs) t.step0[i] = (carry + incl - n) * fg;
      carry += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) t.step0[segs] = carry * fg;
  }
  // places in the order, first units of phase 1 by place
#pragma unroll 1
  for (int a = first; a <= segs; a += 32 * kFewRouters) {   // (a = segs: the end)
    const uint32_t mine = a < segs ? t.weight[a].x : 0;
    uint32_t heavier = 0;
#pragma unroll 4
    for (int o = 0; o < segs; ++o) {
      const uint2 w = t.weight[o];
      heavier += w.x > mine ? w.y : 0;
    }
    if (a < segs) t.order[heavier >> 16] = (uint16_t)a;
    t.unit0[heavier >> 16] = (int)(heavier & 0xffffu) * (p.F / kUnitRows);
  }
}

__device__ __forceinline__ void few_arrive(int32_t* sync, int b, int G) {
  asm volatile("red.add.release.gpu.global.u32 [%0], %1;" ::"l"(sync), "r"(b == 0 ? 0x80000000u - (uint32_t)(G - 1) : 1u) : "memory");
}

// (16 warps: 128 registers a thread, all of which it takes; 4 bytes are spilled, once)
template <class TAB, int XC, int STAGES>
__global__ void __launch_bounds__(kStreamThreads, 1) few_layer_kernel(const __grid_constant__ FewArgs p) {
  extern __shared__ __align__(128) char smem[];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  TAB& t = *reinterpret_cast<TAB*>(smem);
  float* const sums = reinterpret_cast<float*>(smem + kTableBytes<TAB>);
  const int hg = p.H / kGroup, fg = p.F / kGroup;

  // ---- routing ----
  // shared memory: tables, sums of 16 warps, rings of 16 warps; then in phase 1 the staged operand and its sums, in phase 2
  // slots of the streamed operand of 16 warps, and sums of 16 warps for all tokens, if those are more than a unit's
  char* const ring = smem + kTableBytes<TAB> + kStreamWarps * kSumFloats * 4;
  char* const rest = ring + kStreamWarps * STAGES * kSlotBytes;
  float* const xsum = reinterpret_cast<float*>(rest);
  char* const pieces = rest + ((hg * 3 * p.T * 4 + 127) & ~127);
  // a few warps route and make the tables; the others bring the layer's rows of the page table into shared memory (the rings
  // are still empty), ask the L2 cache for the shared experts, which are wanted whatever the routing is, and bring the tokens
  if (warp < kFewRouters) {
#pragma unroll 1
    for (int e = tid; e < 256; e += 32 * kFewRouters) t.mask[e] = 0;
    if (tid == 0) t.done = 0;
    routers_sync();
    if (p.logits) {
#pragma unroll 1
      for (int tok = warp; tok < p.T; tok += kFewRouters) {
        if (p.E <= 64) route_token_n<2>(p.logits, tok, p.E, p.k, t.own_ids, t.own_gates, lane);
        else route_token_n<kMaxExpertsPerLane>(p.logits, tok, p.E, p.k, t.own_ids, t.own_gates, lane);
        if (lane < p.k) atomicOr(&t.mask[t.own_ids[tok * p.k + lane]], 1u << tok);
      }
    } else {
#pragma unroll 1
      for (int i = tid; i < p.T * p.k; i += 32 * kFewRouters) {
        int id = p.ids[i];
        if (id < -1 || id >= p.E) {
          atomicMax(p.status, (int)PW_ERR_INVALID_ARG);
          id = -1;
        }
        t.own_ids[i] = id;
        t.own_gates[i] = p.gates[i];
        if (id >= 0) atomicOr(&t.mask[id], 1u << (i / p.k));
      }
    }
    asm volatile("bar.sync 9, %0;" ::"n"(kStreamThreads) : "memory");   // the rows are there (and the routing of all)
    make_tables(p, t, reinterpret_cast<const DevRow*>(ring), fg, warp, lane);
  } else {
    const int thread = tid - 32 * kFewRouters, threads = kStreamThreads - 32 * kFewRouters;
#pragma unroll 1
    for (int i = thread; i < (p.E + p.n_shared) * (3 * (int)sizeof(DevRow) / 16); i += threads)
      cp16(smem_u32(ring) + i * 16, reinterpret_cast<const char*>(p.rows) + i * 16);
    cp_commit();
    cp_wait<0>();
    asm volatile("bar.arrive 9, %0;" ::"n"(kStreamThreads) : "memory");
    if (warp == kFewRouters) {
      // (pages are whole tiles of 32 KB; asked for by the bulk copy engine, not by loads in front of everyone else's)
      const size_t pieces_of_page = (size_t)p.F * p.H * 2 / kFewAheadPiece;
      int64_t left = kFewAhead / kFewAheadPiece;
#pragma unroll 1
      for (int i = 0; i < p.n_shared * 2 && left > 0; ++i, left -= pieces_of_page) {
        const char* page = static_cast<const char*>(p.rows[(p.E + (i >> 1)) * 3 + (i & 1)].codes);
#pragma unroll 1
        for (size_t l = (size_t)lane * gridDim.x + blockIdx.x; l < pieces_of_page; l += 32 * (size_t)gridDim.x) prefetch_bytes(page + l * kFewAheadPiece, kFewAheadPiece);
      }
    }
    stage_operand<XC <= 2 ? 1 : 4>(p.hidden, (size_t)p.H * 2, p.T, p.T, 0, hg, p.H * 2, pieces, xsum, thread, threads);
  }
  __syncthreads();
  const int segs = t.count[0];
  if (p.seen && blockIdx.x == 0) {                // what the taps' kernel wants to know
#pragma unroll 1
    for (int a = tid; a <= segs; a += kStreamThreads) {
      if (a < segs) p.seen[2 + a] = t.seg[a];
      p.seen[2 + p.segs + a] = t.off[a];
    }
#pragma unroll 1
    for (int i = tid; i < t.count[1]; i += kStreamThreads) {
      p.seen[3 + 2 * p.segs + i] = t.token[i];
      reinterpret_cast<float*>(p.seen)[3 + 2 * p.segs + p.pairs + i] = t.gate[i];
    }
    if (tid == 0) p.seen[0] = segs;
  }

  const Fixed fixed;
  const int G = (int)gridDim.x, b = (int)blockIdx.x;
  if (p.n_parts > 1) {                            // counted from the meeting on: whatever a call before this one has left
#pragma unroll 1
    for (int i = b * kStreamThreads + tid; i < p.H / kUnitRows; i += G * kStreamThreads) p.sync[64 + i] = 0;
  }
  uint32_t before;                                // arrivals, seen before this CTA's: only the top bit matters
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(before) : "l"(p.sync) : "memory");
  Ring r{smem_u32(ring) + warp * STAGES * kSlotBytes, 0, smem_u32(rest) + warp * STAGES * 256 * XC, lane};
  r.slot = r.base;
  Feed f;
  f.left = 0;

  // ---- phase 1: gate and up ----
  {
    // the units, heaviest first, are dealt out in turn, the turns in alternating order; four at a time, each to a team
    const int units = t.unit0[segs], turns = units / G;
    const int mine = turns + (turns & 1 ? G - 1 - b < units - turns * G : b < units - turns * G);
    auto unit_of = [&](int i) { return i * G + (i & 1 ? G - 1 - b : b); };
    int next = 0;                                 // first of the four units that the feed looks at next
    auto ask_next = [&]() {
#pragma unroll 1
      while (f.left == 0) {
        if (next >= mine) return;
        const int m = min(4, mine - next);
        const Team w = few_team(m, warp);
        const int i = next + w.unit;
        next += m;
        const GateUp g = gate_up_unit(t, segs, unit_of(i), hg, w.shift, warp - w.first, lane);
        const SegPage& page = t.page[3 * g.a + g.kind];
        feed_codes(f, lane, page.codes, page.bit1, page.bit0, t.fmt[4 * g.a + g.kind], hg, g.slice, g.lo, g.lo + g.n);
      }
      ask_any<0>(f, r.slot, 0, lane);
    };
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) {
      ask_next();
      ring_on<0, STAGES>(r);
    }
#pragma unroll 1
    for (int first = 0; first < mine; first += 4) {
      const Team w = few_team(min(4, mine - first), warp);
      const int ts = w.shift, member = warp - w.first;
      const GateUp g = gate_up_unit(t, segs, unit_of(first + w.unit), hg, ts, member, lane);
      const int pair0 = t.off[g.a] + g.pass * kUnitCols, cols = min(kUnitCols, t.off[g.a + 1] - pair0);
      const int x = t.token[pair0 + min(lane >> 2, cols - 1)];
      const int t0 = t.token[pair0 + min(2 * (lane & 3), cols - 1)], t1 = t.token[pair0 + min(2 * (lane & 3) + 1, cols - 1)];
      float tot[2][4] = {};
      Operand o{smem_u32(pieces) + x * 256, smem_u32(xsum + t0), smem_u32(xsum + t1), p.T, (uint32_t)(x & 1) << 2, g.lo};
      walk<kAnyFormat, 0, STAGES>(fixed, t.fmt[4 * g.a + g.kind], g.n, f, r, o, tot, ask_next);
      put_sums(sums + warp * kSumFloats, lane, tot);
      few_team_sync(w);
      const float* set = sums + w.first * kSumFloats;
#pragma unroll 1
      for (int i = member * 32 + lane; i < kUnitRows * cols; i += 32 << ts) {
        const int row = i & (kUnitRows - 1), col = i >> 5;
        const float* from = set + col * kSumPitch + row;
        float gate = 0.f, up = 0.f;
#pragma unroll 4
        for (int w = 0; w < 1 << ts; ++w) {
          const float v = from[w * kSumFloats];
          gate = __fadd_rn(gate, w < g.gates ? v : 0.f);
          up = __fadd_rn(up, w < g.gates ? 0.f : v);
        }
        // (fast exponential and division: relative error ~1e-6)
        const float h = __fmul_rn(__fdividef(gate, __fadd_rn(1.0f, __expf(-gate))), up);
        // (beyond the largest fp16 number h is infinite, like the operand of the layer call for batches)
        const __half high = __float2half_rn(h);
        const float left = __hisinf(high) ? 0.f : __fmul_rn(__fsub_rn(h, __half2float(high)), kRestUp);
        char* const to = p.h + (size_t)(pair0 + col) * kHalves * p.F * 2;
        const int f = g.slice * kUnitRows + row;
        *reinterpret_cast<__half*>(to + piece_offset(f, 0)) = high;
        *reinterpret_cast<__half*>(to + (size_t)p.F * 2 + piece_offset(f, 1)) = __float2half_rn(left);
      }
      few_team_sync(w);                    // the sums are written again
    }
  }

  // ---- from phase 1 to phase 2 ----
  // The CTAs add up to 2^31 between them: the top bit turns when the last one has come, and again in the next call.  The last
  // warp of a CTA adds for it (the values of the others, released to this warp, are released with its own).  Each warp then
  // asks for its first codes of phase 2; the places that are written anew meanwhile are its own.
  __syncwarp();
  if (lane == 0) {
    uint32_t n;
    asm volatile("atom.acq_rel.cta.shared::cta.add.u32 %0, [%1], 1;" : "=r"(n) : "r"(smem_u32(&t.done)) : "memory");
    if (n == kStreamWarps - 1 && !(p.hook && b == G - 1)) few_arrive(p.sync, b, G);
  }

  // ---- phase 2: down ----
  {
    const int steps = t.step0[segs];              // of a slice
    const int units = p.H / kUnitRows * p.n_parts;
    const int mine = units / G + (b < units % G);
    auto slice_of = [&](int unit) { return p.n_parts == 1 ? unit : (int)__umulhi((uint32_t)unit, p.per_part); };   // unit / n_parts
    auto range = [&](int unit, int ts, int member, int& lo, int& hi) {
      // steps * i / (n_parts << ts), rounded down (steps * i is below 2^29: exact)
      const uint32_t i = ((uint32_t)(unit - slice_of(unit) * p.n_parts) << ts) + member;
      lo = slice_of((int)(steps * i >> ts));
      hi = slice_of((int)(steps * (i + 1) >> ts));
    };
    cp_wait<0>();
    r.slot = r.base;
    f.left = 0;
    // the feed's next four units, its place in the list of steps, and its slice
    int next = 0, at = 0, end = 0, hint = 0, slice = 0;
    auto more = [&]() -> bool {
      DownRun d;
#pragma unroll 1
      while (!down_run(t, fg, at, end, hint, d)) {
        if (next >= mine) return false;
        const int m = min(4, mine - next);
        const Team w = few_team(m, warp);
        const int unit = (next + w.unit) * G + b;
        next += m;
        at = end = 0;
        range(unit, w.shift, warp - w.first, at, end);
        hint = count_up_to(t.step0 + 1, segs, at, lane);
        slice = slice_of(unit);
      }
      const SegPage& page = t.page[3 * d.a + PW_DOWN];
      const int pair0 = t.off[d.a] + d.pass * kDownCols;
      feed_codes(f, lane, page.codes, page.bit1, page.bit0, t.fmt[4 * d.a + PW_DOWN], fg, slice, d.lo, d.lo + d.n);
      feed_operand(f, lane, p.h + (size_t)pair0 * kHalves * p.F * 2, (uint32_t)p.F * 2, min(kDownCols, t.off[d.a + 1] - pair0) * kHalves, d.lo);
      return true;
    };
    // The first steps are asked for without their operand, which is not there yet.  What a lane will copy of it is noted in
    // the warp's sums of phase 1: its place in p.h, the rows, and log2 of the steps of a group.
    const uint32_t notes = smem_u32(sums + warp * kSumFloats) + lane * 8;
    static_assert(STAGES * 256 <= kSumFloats * 4, "room for the notes");
    int asked = 0;
    auto ask_next = [&]() {
      if (f.left == 0 && !more()) return;
      const int copies = f.copies;
      if (asked < STAGES) {
        const int ls = step_shift(f.fmt);
        const char* x = f.x + (ls == 1 ? f.sub * 128 : ls == 2 ? (f.sub ^ ((lane >> 2) & 1)) * 64 : 0);
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(notes + asked * 256), "r"((uint32_t)(x - p.h)), "r"((uint32_t)(copies << 2 | ls)) : "memory");
        ++asked;
        f.copies = 0;
      }
      ask_any<XC>(f, r.slot, r.x, lane);
      f.copies = copies;
    };
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) {
      ask_next();
      ring_on<XC, STAGES>(r);
    }
    const int first_steps = asked;
    asked = STAGES;
    int place = 0, stop = 0, where = 0;           // of the warp's first unit
    if (mine) {
      const Team w = few_team(min(4, mine), warp);
      range(w.unit * G + b, w.shift, warp - w.first, place, stop);
      where = count_up_to(t.step0 + 1, segs, place, lane);
    }
    bool together = true;
    if (tid == 0) {
      uint32_t now;
      together = false;
#pragma unroll 1
      for (uint32_t i = 0; i < p.polls && !together; ++i) {
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(now) : "l"(p.sync) : "memory");
        together = (now ^ before) >> 31;
      }
      if (!together) atomicMax(p.status, (int)PW_ERR_TIMEOUT);
    }
    if (!__syncthreads_and(together)) {
      // every CTA arrives once, also one that has given up: the next call finds the counter as it should be
      if (p.hook && b == G - 1 && tid == 0) few_arrive(p.sync, b, G);
      cp_wait<0>();
      return;
    }
    uint2 note[STAGES];
#pragma unroll
    for (int i = 0; i < STAGES; ++i) note[i] = i < first_steps ? lds8(notes + i * 256) : make_uint2(0, 0);
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      const uint32_t to = r.x + i * (256 * XC) + lane * 16, step = (uint32_t)p.F * 2 << ((note[i].y & 3) + 1);
      const char* x = p.h + note[i].x;
#pragma unroll 1
      for (uint32_t j = 0; j < note[i].y >> 2; ++j) cp16(to + j * 512, x + (size_t)j * step);
      cp_commit();
    }
    __syncwarp();                                 // every lane has read its notes
    // (for no more tokens than a unit's where those of phase 1 were, and the notes: a warp's place is its own)
    const int set_floats = max(p.T, kUnitCols) * kSumPitch;
    float* const sums2 = p.T <= kUnitCols ? sums : reinterpret_cast<float*>(rest + kStreamWarps * STAGES * 256 * XC);
    float* const own = sums2 + warp * set_floats;
#pragma unroll 1
    for (int first = 0; first < mine; first += 4) {
      const Team w = few_team(min(4, mine - first), warp);
      const int ts = w.shift, member = warp - w.first;
      const int unit = (first + w.unit) * G + b;
      if (first) {
        range(unit, ts, member, place, stop);
        where = count_up_to(t.step0 + 1, segs, place, lane);
      }
#pragma unroll 1
      for (int i = lane; i < p.T * kSumPitch; i += 32) own[i] = 0.f;
      __syncwarp();
      DownRun d;
#pragma unroll 1
      while (down_run(t, fg, place, stop, where, d)) {
        const int fmt = t.fmt[4 * d.a + PW_DOWN], ls = step_shift(fmt);
        const int pair0 = t.off[d.a] + d.pass * kDownCols, cols = min(kDownCols, t.off[d.a + 1] - pair0);
        const int xc = min(lane >> 2, cols * kHalves - 1);
        float tot[2][4] = {};
        Operand o{(uint32_t)(xc * (256 >> ls)), 0, 0, 0, ls == 2 ? 0 : (uint32_t)(xc & 1) << 2, d.lo};
        walk<kAnyFormat, XC, STAGES>(fixed, fmt, d.n, f, r, o, tot, ask_next);
        // Columns 2t and 2t + 1 are the two numbers of token t.  The tokens of a run are different ones: no two lanes meet.
        const int col = lane & 3;
        if (col < cols) {
          const float gate = t.gate[pair0 + col];
          float4* to = reinterpret_cast<float4*>(own + t.token[pair0 + col] * kSumPitch + 4 * (lane >> 2));
          float4 v = *to;
          v.x = __fadd_rn(v.x, __fmul_rn(gate, fmaf(tot[0][1], kRestDown, tot[0][0])));
          v.y = __fadd_rn(v.y, __fmul_rn(gate, fmaf(tot[0][3], kRestDown, tot[0][2])));
          v.z = __fadd_rn(v.z, __fmul_rn(gate, fmaf(tot[1][1], kRestDown, tot[1][0])));
          v.w = __fadd_rn(v.w, __fmul_rn(gate, fmaf(tot[1][3], kRestDown, tot[1][2])));
          *to = v;
        }
        __syncwarp();
      }
      few_team_sync(w);
      float* const set = sums2 + w.first * set_floats;
      const int row0 = slice_of(unit) * kUnitRows, part = unit - slice_of(unit) * p.n_parts;
#pragma unroll 1
      for (int i = member * 32 + lane; i < kUnitRows * p.T; i += 32 << ts) {
        const int row = i & (kUnitRows - 1), tok = i >> 5;
        float v = 0.f;
#pragma unroll 4
        for (int w = 0; w < 1 << ts; ++w) v = __fadd_rn(v, set[w * set_floats + tok * kSumPitch + row]);
        if (p.n_parts == 1) store1(p.out, (int64_t)tok * p.H + row0 + row, p.out_type, v);
        else p.parts[((size_t)part * p.T + tok) * p.H + row0 + row] = v;
      }
      if (p.n_parts > 1) {
        // the last of the parts to finish adds all of them up, in their order
        few_team_sync(w);
        if (lane == 0 && member == 0) {
          uint32_t n;
          asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(n) : "l"(p.sync + 64 + row0 / kUnitRows) : "memory");
          *reinterpret_cast<uint32_t*>(set) = n == (uint32_t)p.n_parts - 1;
        }
        few_team_sync(w);
        if (*reinterpret_cast<volatile uint32_t*>(set)) {
#pragma unroll 1
          for (int i = member * 32 + lane; i < kUnitRows * p.T; i += 32 << ts) {
            const int row = i & (kUnitRows - 1), tok = i >> 5;
            const float* from = p.parts + (size_t)tok * p.H + row0 + row;
            float v = 0.f, part[kFewParts];
#pragma unroll
            for (int q = 0; q < kFewParts; ++q) part[q] = q < p.n_parts ? __ldcg(from + (size_t)q * p.T * p.H) : 0.f;
#pragma unroll
            for (int q = 0; q < kFewParts; ++q) v = __fadd_rn(v, part[q]);
            store1(p.out, (int64_t)tok * p.H + row0 + row, p.out_type, v);
          }
        }
      }
      few_team_sync(w);                    // the sums are written again
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
#pragma unroll 1
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
#pragma unroll 1
  for (int i = p0; i < p1; ++i) {
    const float r = gates[i], x2 = square_sum(hidden + (size_t)tokens[i] * (H / 8), H / 8, lane), h2 = square_sum(h + (size_t)i * kHalves * (F / 8), F / 8, lane);
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
#pragma unroll 1
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
  int segs, pairs, choices, table_bytes, rows, stages;
  FewKernel kernel;
};
template <class TAB, int XC, int STAGES>
static constexpr FewVariant few_variant() {
  return {TAB::kSegs, TAB::kPairs, TAB::kChoices, kTableBytes<TAB>, XC, STAGES, few_layer_kernel<TAB, XC, STAGES>};
}
// The first that fits is the fastest.
static const FewVariant kFewVariants[] = {few_variant<FewSmall, 2, 4>(), few_variant<FewSmall, 4, 3>(), few_variant<FewSmall, 8, 3>(),
                                          few_variant<FewAll, 8, 3>(),   few_variant<FewSmall, 8, 2>(), few_variant<FewAll, 8, 2>()};

static size_t few_smem(const FewArgs& a, const FewVariant& v) {
  const size_t first = (((size_t)a.H / kGroup * 3 * a.T * 4 + 127) & ~(size_t)127) + (size_t)a.T * a.H * 2;
  const size_t second = (size_t)kStreamWarps * (v.stages * 256 * v.rows + (a.T <= kUnitCols ? 0 : a.T * kSumPitch * 4));
  return v.table_bytes + (size_t)kStreamWarps * (kSumFloats * 4 + v.stages * kSlotBytes) + (first > second ? first : second);
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
  const int operand_rows = kHalves * T < kUnitCols ? kHalves * T : kUnitCols;
  const FewVariant* v = nullptr;
  for (const FewVariant& one : kFewVariants)
    if (!v && operand_rows <= one.rows && a.segs <= one.segs && a.pairs <= one.pairs && T * top_k <= one.choices && few_smem(a, one) <= kSmemLimit) v = &one;
  if (!v) return PW_ERR_SHAPE;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  if (!ctx->few_layer_ready.load(std::memory_order_acquire)) {
    for (const FewVariant& one : kFewVariants) PW_CUDA_OK(cudaFuncSetAttribute(one.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
    ctx->few_layer_ready.store(1, std::memory_order_release);
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
  a.polls = ctx->wait_polls ? kFewPollsTest : kFewPolls;
  a.hook = ctx->test_hook & 1u;
  a.status = reinterpret_cast<int32_t*>(b + w.status);
  a.seen = ctx->obs_acc ? reinterpret_cast<int32_t*>(b + w.few_seen) : nullptr;
  // Parts of the down blocks' columns: as few as give every SM work, in rounds that are nearly full.  By an estimate in us:
  // an SM streams 45 KB/us (routed blocks taken for 4 bits), and to add parts up takes about 1 us at the end (measured, 1 part
  // / 2 / 4: one token of 256 x 512 10.3 / 10.9 / 10.9, of 60 + 4 experts of 2048 x 1408 31.0 / 28.3 / 28.9, of 4096 x 14336
  // 71.5 / 75.4 / 75.5).
  const int slices = c.hidden / kUnitRows, routed = c.n_experts < T * top_k ? c.n_experts : T * top_k;
  const double slice_us = 32e-3 * c.ffn * (0.5 * routed + 2. * c.n_shared) / 45.;
  double best = -1.;
  for (int parts = 1; parts <= kFewParts; ++parts) {
    const int rounds = (slices * parts + ctx->num_sms - 1) / ctx->num_sms;
    const double us = slice_us * rounds / parts * (1. + 0.05 * parts) + (parts > 1 ? 1. : 0.);
    if (best < 0 || us < best) best = us, a.n_parts = parts;
  }
  // (see `range`: a place in the list of steps, times the parts of it, divided by multiplication)
  if (((int64_t)a.segs + a.pairs / kDownCols) * (c.ffn / kGroup) * 4 * (kFewParts * kStreamWarps) >= 1 << 29) return PW_ERR_SHAPE;
  a.per_part = a.n_parts > 1 ? (uint32_t)((0xffffffffull + a.n_parts) / a.n_parts) : 0;
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
