// Dense products on weight pages for few tokens (pw_page_linear).  The inner loop is in pw_stream.cuh.
//
// Bound: the pages' bytes for wide blocks (32003 x 4096 at 4 bits, one token: 16 us, 4.4 TB/s while the copy rate is 6.6),
// the launch and one round trip to memory for small ones (4096 x 4096, one token: 4.8 us, of which an empty launch takes
// 1.9 and the bytes 1.4), and with eight tokens of long rows the operand, which does not fit one SM (4096 x 14336, 3 of 4
// planes: 15.7 us; clusters of four CTAs share the columns, their launch alone takes 3 us more).  How a product is cut is
// decided by an estimate (cut_page_linear); of the cuts there are (24 to 48) it took the fastest, or one within 2 %, for all
// of ten shapes.
#include "pw_scaled.cuh"
#include "pw_stream.cuh"

namespace pw {

constexpr int kSumsBytes = kStreamWarps * kSumFloats * 4;
constexpr int kPartsBytes = 16384;                // sums of a batch of units from the CTAs of a cluster

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void store_to_rank(uint32_t own_s, uint32_t rank, float v) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own_s), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ void team_sync(int team, int ts) { asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 << ts) : "memory"); }

// ---- dense product -------------------------------------------------------------------------------
struct LinearPage {
  const char* codes;
  const char* bit1;
  const char* bit0;
  int fmt, rows;                                  // rows: output features
  int end;                                        // slices of 32 rows of the pages up to and with this one
  int col0;                                       // its first column of the output
};
struct PageLinearArgs {
  int T, groups, x_bytes;
  int width, passes, slices;                      // tokens of a pass
  int team_shift, split;                          // log2 of the warps that share a unit; CTAs of a cluster, which share the columns
  int room, split_groups;                         // tokens and groups that there is room for in a CTA
  int batch;                                      // units of a team between two exchanges of a cluster
  int pages, out_type, bias_type;
  const char* x;
  size_t x_pitch;                                 // bytes
  void* out;
  const void* bias;
  int64_t ld_out;
  LinearPage page[PW_LINEAR_PAGES];
};
struct LinearUnit {
  int page, slice;
};
__device__ __forceinline__ LinearUnit linear_unit(const PageLinearArgs& a, int u) {
  LinearUnit un{0, u};
  if (a.pages > 1) {
#pragma unroll 1
    while (u >= a.page[un.page].end) ++un.page;
    if (un.page) un.slice -= a.page[un.page - 1].end;
  }
  return un;
}

__device__ __forceinline__ void put_linear(const PageLinearArgs& a, const LinearUnit& un, int token, int row, float v) {
  const int m = un.slice * kUnitRows + row;
  if (m >= a.page[un.page].rows) return;
  const int at_col = a.page[un.page].col0 + m;
  if (a.bias) v = __fadd_rn(v, load1(a.bias, at_col, a.bias_type));
  store1(a.out, (int64_t)token * a.ld_out + at_col, a.out_type, v);
}

// A cluster takes a pass of up to eight tokens, stages their columns (each CTA its part) and goes through slices of 32
// rows.  Teams of 4, 8 or 16 warps take a slice each; the warps of a team share the CTA's columns and add their sums in
// warp order, the CTAs of a cluster theirs in rank order, a batch of slices at a time.
// F: the format of all pages, or kAnyFormat; a kernel for one format is a quarter of the code, and a call for one token
// spends a large part of its time on fetching code.
template <int F, int STAGES>
__global__ void __launch_bounds__(kStreamThreads, 1) page_linear_kernel(const __grid_constant__ PageLinearArgs a) {
  constexpr int kRing = STAGES * kSlotBytes;
  extern __shared__ __align__(128) char smem[];
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int ts = a.team_shift, team = warp >> ts, member = warp & ((1 << ts) - 1);
  float* const sums = reinterpret_cast<float*>(smem + kStreamWarps * kRing) + (team << ts) * kSumFloats;
  float* const parts = reinterpret_cast<float*>(smem + kStreamWarps * kRing + kSumsBytes);   // [rank][slot / split][token][32 rows], slots: [team][batch]
  float* const xsum = parts + (a.split > 1 ? kPartsBytes / 4 : 0);
  char* const pieces = reinterpret_cast<char*>(xsum) + ((a.split_groups * 3 * a.room * 4 + 127) & ~127);

  if (a.split > 1) cluster_arrive();              // this CTA has started: the others may write to its memory
  const int rank = a.split > 1 ? (int)cluster_rank() : 0;
  const int cluster = a.split > 1 ? (int)blockIdx.x / a.split : (int)blockIdx.x, clusters = a.split > 1 ? (int)gridDim.x / a.split : (int)gridDim.x;
  const int g0 = a.groups * rank / a.split, my_groups = a.groups * (rank + 1) / a.split - g0;
  // clusters deal out the passes among them; those with the same pass share its slices
  const int sharing = a.passes < clusters ? (clusters - cluster % a.passes + a.passes - 1) / a.passes : 1;
  const int first = a.passes < clusters ? cluster / a.passes : 0, stride = sharing << (4 - ts);   // of team 0; the others' lie `sharing` apart

  const Fixed fixed;
  const uint32_t ring = smem_u32(smem) + warp * kRing;
  Ring r{ring, ring, 0, lane};
  Feed f;
  f.left = 0;
  int next = 0;                                   // slice the feed takes next
  auto more = [&]() -> bool {
#pragma unroll 1
    while (next < a.slices) {
      const LinearUnit un = linear_unit(a, next);
      const LinearPage& p = a.page[un.page];
      const int fmt = F == kAnyFormat ? p.fmt : F;
      const int steps = my_groups << step_shift(fmt), from = g0 << step_shift(fmt);
      feed_codes(f, lane, p.codes, p.bit1, p.bit0, fmt, a.groups, un.slice, from + ((steps * member) >> ts), from + ((steps * (member + 1)) >> ts));
      next += stride;
      if (f.left) return true;
    }
    return false;
  };
  auto ask_next = [&]() {
    if (f.left == 0 && !more()) return;
    if constexpr (F == kAnyFormat) {
      ask_any<0>(f, r.slot, 0, lane);
    } else {
      f.left--;
      ask<F, 0>(f, r.slot, 0, lane);
    }
  };

  // The operand and the pages may be the work of the kernel directly ahead, which may still run: nothing is read before the
  // wait.  The first codes are only asked to come into the L2 cache, where what that kernel writes goes as well.
  next = first + sharing * team;
  if (more()) prefetch_steps<STAGES>(f, lane);
  grid_dep_sync();
  grid_dep_trigger();

  bool met = false, exchanged = false;
#pragma unroll 1
  for (int pass = cluster % a.passes; pass < a.passes; pass += clusters) {
    const int token0 = pass * a.width, cols = min(a.width, a.T - token0);
    __syncthreads();                              // the pass before has read its operand
    stage_operand<1>(a.x + (size_t)token0 * a.x_pitch, a.x_pitch, cols, a.room, g0, my_groups, a.x_bytes, pieces, xsum, threadIdx.x,
                  kStreamThreads);
    // (behind the operand, which has the longer way: 4096 x 4096 4.81 us, the other way round 5.06)
    r.slot = r.base;
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) {
      ask_next();
      ring_on<0, STAGES>(r);
    }
    __syncthreads();
    if (a.split > 1 && !met) {
      cluster_wait();                             // all CTAs of the cluster have started
      met = true;
    }
    // (tokens that there are not: any row and sum, their products are not used)
    const int xc = min(lane >> 2, cols - 1), c0 = min(2 * (lane & 3), cols - 1), c1 = min(2 * (lane & 3) + 1, cols - 1);
    const uint32_t x_lane = smem_u32(pieces) + xc * 256, sum0 = smem_u32(xsum + c0), sum1 = smem_u32(xsum + c1);
    const int batch = a.split > 1 ? a.batch : 1, slots = batch << (4 - ts);
#pragma unroll 1
    for (int u0 = first; u0 < a.slices; u0 += stride * batch) {
      if (a.split > 1 && exchanged) cluster_sync();   // the parts of the batch before have been read
#pragma unroll 1
      for (int j = 0; j < batch; ++j) {
        const int u = u0 + sharing * team + stride * j;
        if (u >= a.slices) break;
        const LinearUnit un = linear_unit(a, u);
        const int fmt = F == kAnyFormat ? a.page[un.page].fmt : F;
        const int steps = my_groups << step_shift(fmt), lo = (steps * member) >> ts;
        float tot[2][4] = {};
        Operand o{x_lane, sum0, sum1, a.room, (uint32_t)(xc & 1) << 2, lo};
        walk<F, 0, STAGES>(fixed, fmt, ((steps * (member + 1)) >> ts) - lo, f, r, o, tot, ask_next);
        put_sums(sums + member * kSumFloats, lane, tot);
        team_sync(team, ts);
#pragma unroll 1
        for (int i = member * 32 + lane; i < kUnitRows * cols; i += 32 << ts) {
          const int row = i & (kUnitRows - 1), col = i >> 5;
          float v = 0.f;
#pragma unroll 4
          for (int w = 0; w < 1 << ts; ++w) v = __fadd_rn(v, sums[w * kSumFloats + col * kSumPitch + row]);
          const int slot = team * batch + j;      // slot s is added up by rank s mod split
          if (a.split > 1) store_to_rank(smem_u32(parts + ((rank * slots + slot) / a.split * kUnitCols) * kUnitRows + i), slot % a.split, v);
          else put_linear(a, un, token0 + col, row, v);
        }
        team_sync(team, ts);                      // the sums are written again
      }
      if (a.split > 1) {
        cluster_sync();
        exchanged = true;
#pragma unroll 1
        for (int s = rank; s < slots; s += a.split) {
          const int u = u0 + sharing * (s / batch) + stride * (s % batch);
          if (u >= a.slices) continue;
          const LinearUnit un = linear_unit(a, u);
#pragma unroll 1
          for (int i = threadIdx.x; i < kUnitRows * cols; i += kStreamThreads) {
            float v = 0.f;
#pragma unroll 1
            for (int k = 0; k < a.split; ++k) v = __fadd_rn(v, parts[((k * slots + s) / a.split * kUnitCols) * kUnitRows + i]);
            put_linear(a, un, token0 + (i >> 5), i & (kUnitRows - 1), v);
          }
        }
      }
    }
    next = first + sharing * team;                // the feed starts again
  }
}

static size_t page_linear_smem(const PageLinearArgs& a, int stages) {
  return (size_t)kStreamWarps * stages * kSlotBytes + kSumsBytes + (a.split > 1 ? kPartsBytes : 0) +
         (((size_t)a.split_groups * 3 * a.room * 4 + 127) & ~(size_t)127) + (size_t)a.split_groups * a.room * 256;
}
typedef void (*PageLinearKernel)(PageLinearArgs);
template <int STAGES>
static PageLinearKernel page_linear_kernel_of(int fmt) {
  switch (fmt) {
    case kFmt16: return page_linear_kernel<kFmt16, STAGES>;
    case kFmt8: return page_linear_kernel<kFmt8, STAGES>;
    case kFmt4: return page_linear_kernel<kFmt4, STAGES>;
    case kFmt3: return page_linear_kernel<kFmt3, STAGES>;
    case kFmt2: return page_linear_kernel<kFmt2, STAGES>;
    case kFmtP4: return page_linear_kernel<kFmtP4, STAGES>;
    case kFmtP3: return page_linear_kernel<kFmtP3, STAGES>;
    case kFmtP2: return page_linear_kernel<kFmtP2, STAGES>;
    default: return page_linear_kernel<kAnyFormat, STAGES>;
  }
}
static PageLinearKernel page_linear_kernel_of(int fmt, int stages) { return stages == 4 ? page_linear_kernel_of<4>(fmt) : page_linear_kernel_of<2>(fmt); }
static cudaError_t launch_page_linear(const PageLinearArgs& a, PageLinearKernel kernel, int clusters, size_t smem, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(clusters * a.split));
  cfg.blockDim = dim3(kStreamThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Once per context (more than once does no harm): what the launches need of the device.
constexpr int kSplits = 3;                        // clusters of 2, 4, 8 CTAs
static pw_status few_setup(pw_ctx* ctx) {
  if (ctx->few_ready.load(std::memory_order_acquire)) return PW_OK;
  for (int fmt = kAnyFormat; fmt <= kFmtP2; ++fmt)
    for (int stages = 2; stages <= 4; stages += 2)
      PW_CUDA_OK(cudaFuncSetAttribute(page_linear_kernel_of(fmt, stages), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
  // how many clusters run at the same time, one CTA per SM: an SM left over in its group of SMs is of no use to a cluster
  for (int i = 0; i < kSplits; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2 << i;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.gridDim = dim3(2 << i);
    cfg.blockDim = dim3(kStreamThreads);
    cfg.dynamicSmemBytes = kSmemLimit;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    PW_CUDA_OK(cudaOccupancyMaxActiveClusters(&clusters, page_linear_kernel_of(kAnyFormat, 4), &cfg));
    ctx->few_clusters[i].store(clusters, std::memory_order_relaxed);
  }
  ctx->few_ready.store(1, std::memory_order_release);
  return PW_OK;
}

// How a product is cut: tokens to a pass, warps to a unit, CTAs to a cluster, stages of the rings.
struct PageLinearPlan {
  int stages, clusters;
  double cycles;                                  // estimate
};
// Fills in the fields of `a` that depend on the cut; cycles < 0: it has no room.
static PageLinearPlan cut_page_linear(PageLinearArgs& a, int width, int split, int ts, int sms, const int* max_clusters) {
  PageLinearPlan p{0, 0, -1.};
  a.width = a.room = width;
  a.split = split;
  a.split_groups = (a.groups + split - 1) / split;
  a.team_shift = ts;
  a.passes = (a.T + width - 1) / width;
  a.batch = kPartsBytes / (kUnitRows * 4 * kUnitCols) >> (4 - ts);
  for (int stages = 4; stages >= 2 && !p.stages; stages -= 2)
    if (page_linear_smem(a, stages) <= kSmemLimit) p.stages = stages;
  int most = sms;
  for (int i = 0; i < kSplits; ++i)
    if (split == 2 << i) most = max_clusters[i];
  if (!p.stages || most < 1) return p;
  const int64_t units = (int64_t)a.slices * a.passes, teams = 16 >> ts;
  p.clusters = (int)(units < most ? units : most);
  const int64_t sharing = a.passes < p.clusters ? p.clusters / a.passes : 1, passes = (a.passes + p.clusters - 1) / p.clusters;
  const int64_t rounds = (a.slices + sharing * teams - 1) / (sharing * teams);
  int64_t steps = 0;                              // of a warp, for a slice of the average page
  for (int i = 0; i < a.pages; ++i) steps += (int64_t)a.split_groups << step_shift(a.page[i].fmt);
  steps = (steps + ((int64_t)a.pages << ts) - 1) / ((int64_t)a.pages << ts);
  // Constants fitted to measured cuts, most of them of 4-bit blocks (not the time of a step, which is 1530 cycles there with
  // every warp at work): 1100 cycles of the SM for a step of each of the 16 warps, 400 for one of few warps; then the
  // hand-over of a unit, the exchange of a cluster, and the operands' way into shared memory.  Formats differ by what their
  // steps hold, which is all that the estimate knows of them: times at 16 bits come out 30 to 70 % too long.
  const double busy = (double)a.slices / (double)(sharing * teams);
  double c = (double)rounds * ((double)steps * (busy >= 1. ? 1100. : 1100. * busy > 400. ? 1100. * busy : 400.) + 1500.);
  if (split > 1) c += 4000. + (double)((rounds + a.batch - 1) / a.batch) * 3000.;
  c += (double)a.split_groups * width * 256 / 30.;
  p.cycles = c * (double)passes;
  return p;
}
// The cut that finishes soonest by that estimate.
static PageLinearPlan plan_page_linear(PageLinearArgs& a, int sms, const int* max_clusters) {
  PageLinearPlan best{0, 0, -1.};
  PageLinearArgs made = a;
  for (int width = a.T < kUnitCols ? a.T : kUnitCols; width; width /= 2)
    for (int split = 1; split <= 8; split *= 2)
      for (int ts = 4; ts >= 2; --ts) {
        PageLinearArgs b = a;
        const PageLinearPlan p = cut_page_linear(b, width, split, ts, sms, max_clusters);
        if (p.cycles >= 0 && (best.cycles < 0 || p.cycles < best.cycles)) best = p, made = b;
      }
  a = made;
  return best;
}

}  // namespace pw

using namespace pw;

// A page that a streaming kernel can read.
static pw_status check_page(const pw_page& p) {
  const bool planes = p.layout == PW_LAYOUT_PLANES;
  if (stream_format(p.bits, planes) < 0) return PW_ERR_BITS;
  if (p.rows < 1 || p.cols < 1 || p.rows % kTileRows || p.cols % kGroup || p.group != kGroup || p.rows > 1u << 30 || p.cols > 1u << 18) return PW_ERR_SHAPE;
  if (!planes && p.layout != PW_LAYOUT_TILED) return PW_ERR_STATE;
  if (!p.codes) return PW_ERR_INVALID_ARG;
  if (planes && ((p.bits >= 3 && !p.scales) || (p.bits == 4 && !p.zps))) return PW_ERR_STATE;
  if (!is_aligned(p.codes, 16) || (planes && (!is_aligned(p.scales, 16) || !is_aligned(p.zps, 16)))) return PW_ERR_ALIGN;
  return PW_OK;
}

// The fields of `a` that describe the operands; the pages have been checked.  Returns the columns of the output.
static int64_t set_pages(PageLinearArgs& a, int T, int K, const pw_page* pages, const int32_t* out_features, int n_pages) {
  int64_t slices = 0, columns = 0;
  for (int i = 0; i < n_pages; ++i) {
    const pw_page& p = pages[i];
    const int64_t n = out_features ? out_features[i] : (int64_t)p.rows;
    LinearPage& l = a.page[i];
    l.codes = static_cast<const char*>(p.codes);
    l.bit1 = static_cast<const char*>(p.scales);
    l.bit0 = static_cast<const char*>(p.zps);
    l.fmt = stream_format(p.bits, p.layout == PW_LAYOUT_PLANES);
    l.rows = (int)n;
    l.col0 = (int)columns;
    slices += (n + kUnitRows - 1) / kUnitRows;
    columns += n;
    l.end = (int)slices;
  }
  a.T = T;
  a.groups = (int)(pages[0].cols / kGroup);
  a.x_bytes = 2 * K;
  a.slices = (int)slices;
  a.pages = n_pages;
  return columns;
}
// Whether a call goes through the tensor-core kernel of the layer calls (three launches; outputs of 16 bits), and what of its
// cut does not depend on the device.  By estimates of both times in us: this kernel's from its cut; the other's as a sum of
// terms, 11 for the launches, for decoding 0.2 per million weights or 0.09 per group of columns, 2.3 per billion products, 4
// per million outputs (parts of sums, written and read).  Fitted to thirty shapes, where it takes the faster kernel or one
// within 5 %; of forty drawn afterwards, of all formats and mixed ones, the kernel it takes is 1 % slower than the faster one
// in the mean, 28 % at worst (13986 x 468 at 4 bits, 91 tokens 19.7 / 15.4).  Measured, here /
// there: 14336 x 4096 at 4 bits, 16 tokens 16.4 / 26.5, 32 tokens 27.0 / 27.6, 64 tokens 46.9 / 32.0, 256 tokens 188 / 72;
// 4096 x 4096 at 4 bits, 64 tokens 17.6 / 17.3; 4096 x 14336 at 8 bits, 64 tokens 61 / 32; 28672 x 8192 at 4 bits, 16 tokens
// 51 / 73; 1260 x 1000 in planes of 4 bits, 300 tokens 15.4 / 14.6, 600 tokens 37 / 17.7; 40 x 128 at 4 bits, 1200 tokens
// 5.4 / 11.5.
static bool many_tokens(DenseCall* d, const PageLinearArgs& call, const pw_page* pages, int out_type, int sms) {
  if (call.T <= kUnitCols || out_type == PW_F32) return false;
  double m = 0, width = 0;                         // millions of weights; columns, in whole tiles
  for (int i = 0; i < call.pages; ++i) {
    m += 1e-6 * pages[i].cols * call.page[i].rows;
    width += (call.page[i].rows + kTileRows - 1) / kTileRows * kTileRows;
  }
  // (about as many clusters as run at the same time: the workspace's size must not depend on the current device)
  int clusters[kSplits];
  for (int i = 0; i < kSplits; ++i) clusters[i] = sms * 7 / (8 * (2 << i));
  const double decode = 0.2 * m > 0.09 * call.groups ? 0.2 * m : 0.09 * call.groups;
  const double there = 11. + decode + 2.3e-3 * m * call.T + 4e-6 * call.T * width;
  PageLinearArgs a = call;
  const PageLinearPlan here = plan_page_linear(a, sms, clusters);
  if (here.stages && 2.5 + here.cycles / 1680. <= there) return false;
  *d = DenseCall{};
  d->T = call.T;
  d->cols = (int)pages[0].cols;
  d->n_pages = call.pages;
  for (int i = 0; i < call.pages; ++i) {
    d->page[i] = pages[i];
    d->features[i] = call.page[i].rows;
  }
  return true;
}
static pw_status check_pages(int T, int K, const pw_page* pages, const int32_t* out_features, int n_pages) {
  if (T < 0 || K < 1 || !pages || n_pages < 1 || n_pages > PW_LINEAR_PAGES) return PW_ERR_INVALID_ARG;
  if (T > 1 << 24) return PW_ERR_SHAPE;
  int64_t columns = 0;
  for (int i = 0; i < n_pages; ++i) {
    const pw_page& p = pages[i];
    const pw_status ps = check_page(p);
    if (ps != PW_OK) return ps;
    const int64_t n = out_features ? out_features[i] : (int64_t)p.rows;
    if (n < 1) return PW_ERR_INVALID_ARG;
    if (n > p.rows || K > (int64_t)p.cols || K <= (int64_t)p.cols - kGroup || p.cols != pages[0].cols) return PW_ERR_SHAPE;
    columns += n;
    if (columns > 1 << 30) return PW_ERR_SHAPE;
  }
  return PW_OK;
}

extern "C" size_t pw_page_linear_workspace(pw_ctx* ctx, int T, int K, const pw_page* pages, const int32_t* out_features, int n_pages, int out_type) {
  if (!ctx || !type_ok(out_type) || check_pages(T, K, pages, out_features, n_pages) != PW_OK) return 0;
  PageLinearArgs a{};
  set_pages(a, T, K, pages, out_features, n_pages);
  DenseCall d;
  return many_tokens(&d, a, pages, out_type, ctx->num_sms) ? dense_plan(&d, ctx->num_sms) : 0;
}

extern "C" pw_status pw_page_linear(pw_ctx* ctx, int T, int K, const void* x_fp16, int64_t x_stride, const pw_page* pages,
                                    const int32_t* out_features, int n_pages, const void* bias, int bias_type, void* out,
                                    int out_type, int64_t out_stride, void* workspace, size_t workspace_bytes, pw_stream stream) {
  if (!ctx || !type_ok(out_type) || (bias && !type_ok(bias_type))) return PW_ERR_INVALID_ARG;
  const pw_status cs = check_pages(T, K, pages, out_features, n_pages);
  if (cs != PW_OK) return cs;
  PageLinearArgs a{};
  const int64_t columns = set_pages(a, T, K, pages, out_features, n_pages);
  if (T == 0) return PW_OK;
  if (!x_fp16 || !out) return PW_ERR_INVALID_ARG;
  if (T > 1 && (x_stride < K || out_stride < columns)) return PW_ERR_SHAPE;
  if (!is_aligned(x_fp16, 16) || !is_aligned(out, 16) || !is_aligned(bias, 16) || !is_aligned(workspace, 256) || (T > 1 && x_stride % 8)) return PW_ERR_ALIGN;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  DenseCall d;
  if (workspace && many_tokens(&d, a, pages, out_type, ctx->num_sms)) {
    const size_t need = dense_plan(&d, ctx->num_sms);
    if (need && need <= workspace_bytes)
      return launch_dense(ctx, d, x_fp16, (size_t)x_stride * 2, 2 * K, bias, bias_type, out, out_type, out_stride, workspace, stream);
  }
  const pw_status fs = few_setup(ctx);
  if (fs != PW_OK) return fs;
  a.x = static_cast<const char*>(x_fp16);
  a.x_pitch = T > 1 ? (size_t)x_stride * 2 : 0;
  a.out = out;
  a.bias = bias;
  a.ld_out = out_stride;
  a.out_type = out_type;
  a.bias_type = bias_type;
  int max_clusters[kSplits];
  for (int i = 0; i < kSplits; ++i) max_clusters[i] = ctx->few_clusters[i].load(std::memory_order_relaxed);
  const PageLinearPlan p = plan_page_linear(a, ctx->num_sms, max_clusters);
  if (!p.stages) return PW_ERR_SHAPE;
  const size_t smem = page_linear_smem(a, p.stages);
  int fmt = a.page[0].fmt;
  for (int i = 1; i < n_pages; ++i)
    if (a.page[i].fmt != fmt) fmt = kAnyFormat;
  PW_CUDA_OK(launch_page_linear(a, page_linear_kernel_of(fmt, p.stages), p.clusters, smem, stream));
  ctx->launches++;
  return PW_OK;
}
