// The calls for few tokens: dense products on weight pages (pw_page_linear) and the whole layer in one kernel
// (pw_moe_forward_few).  The inner loop is in pw_stream.cuh.
#include "pw_scaled.cuh"
#include "pw_stream.cuh"

namespace pw {

constexpr int kSmemLimit = 232448;                // 227 KB
constexpr int kSumsBytes = kStreamWarps * kSumFloats * 4;
constexpr int kUnitOut = kUnitRows * kUnitCols;

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
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
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
  LinearPage page[PW_LINEAR_PAGES];
  const char* x;
  size_t x_pitch;                                 // bytes
  void* out;
  const void* bias;
  int64_t ld_out;
  int T, groups, x_bytes;
  int width, passes, slices;                      // tokens of a pass (8, fewer for very long rows)
  int team_shift, split;                          // log2 of the warps that share a unit; CTAs of a cluster, which share the columns
  int rows, split_groups;                         // most tokens of a pass, most groups of a CTA: what is staged
  int out_type, bias_type;
};
struct LinearUnit {
  int page, slice;
};
__device__ __forceinline__ LinearUnit linear_unit(const PageLinearArgs& a, int u) {
  LinearUnit un{0, u};
  while (u >= a.page[un.page].end) ++un.page;
  if (un.page) un.slice -= a.page[un.page - 1].end;
  return un;
}

// A cluster takes a pass of up to eight tokens, stages their columns (each CTA its part) and goes through slices of 32
// rows.  Teams of 4, 8 or 16 warps take a slice each; the warps of a team share the CTA's columns and add their sums in
// warp order, the CTAs of a cluster (whose team is the whole CTA) theirs in rank order.
template <int STAGES>
__global__ void __launch_bounds__(kStreamThreads, 1) page_linear_kernel(const __grid_constant__ PageLinearArgs a) {
  constexpr int kRing = STAGES * kSlotOf<0>;
  extern __shared__ __align__(128) char smem[];
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int ts = a.team_shift, team = warp >> ts, member = warp & ((1 << ts) - 1);
  float* const sums = reinterpret_cast<float*>(smem + kStreamWarps * kRing) + (team << ts) * kSumFloats;
  float* const parts = reinterpret_cast<float*>(smem + kStreamWarps * kRing + kSumsBytes);   // [2][split][kUnitOut] of rank 0
  float* const xsum = parts + (a.split > 1 ? 2 * a.split * kUnitOut : 0);
  char* const pieces = reinterpret_cast<char*>(xsum) + ((a.split_groups * 2 * a.rows * 4 + 127) & ~127);

  const int rank = a.split > 1 ? (int)cluster_rank() : 0;
  const int cluster = a.split > 1 ? (int)blockIdx.x / a.split : (int)blockIdx.x, clusters = a.split > 1 ? (int)gridDim.x / a.split : (int)gridDim.x;
  const int g0 = a.groups * rank / a.split, my_groups = a.groups * (rank + 1) / a.split - g0;
  // clusters deal out the passes among them; those with the same pass share its slices
  const int sharing = a.passes < clusters ? (clusters - cluster % a.passes + a.passes - 1) / a.passes : 1;
  const int first = (a.passes < clusters ? cluster / a.passes : 0) + sharing * team, stride = sharing << (4 - ts);

  Ring r{smem + warp * kRing, 0, 0, lane};
  r.base_s = smem_u32(r.base);
  Feed f;
  f.left = 0;
  int next = first;                               // slice the feed takes next
  auto more = [&]() -> bool {
    while (next < a.slices) {
      const LinearUnit un = linear_unit(a, next);
      const LinearPage& p = a.page[un.page];
      const int steps = my_groups << step_shift(p.fmt), from = g0 << step_shift(p.fmt);
      feed_codes(f, lane, p.codes, p.bit1, p.bit0, p.fmt, a.groups, un.slice, from + ((steps * member) >> ts), from + ((steps * (member + 1)) >> ts));
      next += stride;
      if (f.left) return true;
    }
    return false;
  };

  int buf = 0;
  bool waited = false;
#pragma unroll 1
  for (int pass = cluster % a.passes; pass < a.passes; pass += clusters) {
    // pages are final when this kernel is placed, the operand may be written by the kernel ahead: codes first
    next = first;
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) {
      if (f.left || more()) ask_any<0, true, false>(f, r.base_s + i * kSlotOf<0>, lane);
      cp_commit();
    }
    r.slot = 0;
    if (!waited) {
      grid_dep_sync();
      grid_dep_trigger();
      waited = true;
    }
    const int cols = min(a.width, a.T - pass * a.width);
    __syncthreads();                              // the pass before has read its operand
    stage_operand(a.x + (size_t)pass * a.width * a.x_pitch, a.x_pitch, cols, g0, my_groups, a.x_bytes, pieces, xsum);
    __syncthreads();
    const int xc = min(lane >> 2, cols - 1), c0 = min(2 * (lane & 3), cols - 1), c1 = min(2 * (lane & 3) + 1, cols - 1);
#pragma unroll 1
    for (int u = first; u < a.slices; u += stride, buf ^= 1) {
      const LinearUnit un = linear_unit(a, u);
      const int fmt = a.page[un.page].fmt;
      const int steps = my_groups << step_shift(fmt), lo = (steps * member) >> ts;
      float tot[2][4] = {};
      Operand o{pieces + xc * 256, xsum + c0, c1 - c0, cols, (uint32_t)(xc & 1) << 2, lo};
      walk<0, STAGES>(fmt, ((steps * (member + 1)) >> ts) - lo, f, r, o, tot, more);
      put_sums(sums + member * kSumFloats, lane, tot);
      team_sync(team, ts);
      for (int i = member * 32 + lane; i < kUnitRows * cols; i += 32 << ts) {
        const int row = i & (kUnitRows - 1), col = i >> 5;
        float v = 0.f;
#pragma unroll 4
        for (int w = 0; w < 1 << ts; ++w) v = __fadd_rn(v, sums[w * kSumFloats + col * kSumPitch + row]);
        if (a.split > 1) {
          store_to_rank(smem_u32(parts + (buf * a.split + rank) * kUnitOut + i), 0, v);
        } else {
          const int m = un.slice * kUnitRows + row;
          if (m < a.page[un.page].rows) {
            const int at_col = a.page[un.page].col0 + m;
            if (a.bias) v = __fadd_rn(v, load1(a.bias, at_col, a.bias_type));
            store1(a.out, (int64_t)(pass * a.width + col) * a.ld_out + at_col, a.out_type, v);
          }
        }
      }
      if (a.split > 1) {
        cluster_sync();                           // (the other buffer is written next: whoever writes this one again has seen rank 0 past it)
        if (rank == 0)
          for (int i = threadIdx.x; i < kUnitRows * cols; i += kStreamThreads) {
            const int row = i & (kUnitRows - 1), col = i >> 5, m = un.slice * kUnitRows + row;
            float v = 0.f;
            for (int k = 0; k < a.split; ++k) v = __fadd_rn(v, parts[(buf * a.split + k) * kUnitOut + i]);
            if (m < a.page[un.page].rows) {
              const int at_col = a.page[un.page].col0 + m;
              if (a.bias) v = __fadd_rn(v, load1(a.bias, at_col, a.bias_type));
              store1(a.out, (int64_t)(pass * a.width + col) * a.ld_out + at_col, a.out_type, v);
            }
          }
      } else {
        team_sync(team, ts);                      // the sums are written again by the next unit
      }
    }
  }
}

static size_t page_linear_smem(const PageLinearArgs& a, int stages) {
  return (size_t)kStreamWarps * stages * kSlotOf<0> + kSumsBytes + (a.split > 1 ? 2 * a.split * kUnitOut * 4 : 0) +
         (((size_t)a.split_groups * 2 * a.rows * 4 + 127) & ~(size_t)127) + (size_t)a.split_groups * a.rows * 256;
}
template <int STAGES>
static cudaError_t launch_page_linear(const PageLinearArgs& a, int clusters, size_t smem, cudaStream_t s) {
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
  return cudaLaunchKernelEx(&cfg, page_linear_kernel<STAGES>, a);
}

// Once per context (more than once does no harm): what the launches need of the device.
static pw_status few_setup(pw_ctx* ctx) {
  if (ctx->few_ready.load(std::memory_order_acquire)) return PW_OK;
  PW_CUDA_OK(cudaFuncSetAttribute(page_linear_kernel<3>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
  PW_CUDA_OK(cudaFuncSetAttribute(page_linear_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
  ctx->few_ready.store(1, std::memory_order_release);
  return PW_OK;
}

// How a product is cut: warps to a unit, CTAs to a cluster, stages of the rings, clusters.  `clusters_of`: how many of a
// size run at the same time.
struct PageLinearPlan {
  int stages, clusters;
};
static PageLinearPlan plan_page_linear(PageLinearArgs& a, int sms) {
  PageLinearPlan p{0, 0};
  int steps = 0, pages = 0;
  for (; pages < PW_LINEAR_PAGES && a.page[pages].codes; ++pages) steps += a.groups << step_shift(a.page[pages].fmt);
  for (a.width = kUnitCols; a.width && !p.stages; a.width >>= p.stages ? 0 : 1) {
    a.rows = a.T < a.width ? a.T : a.width;
    for (a.split = 1; a.split <= 8; a.split *= 2) {
      a.split_groups = (a.groups + a.split - 1) / a.split;
      for (int stages = 4; stages >= 3 && !p.stages; --stages)
        if (page_linear_smem(a, stages) <= kSmemLimit) p.stages = stages;
      if (p.stages) break;
    }
  }
  if (!p.stages) return p;
  a.passes = (a.T + a.width - 1) / a.width;
  const int64_t most = sms / a.split;
  const int64_t units = (int64_t)a.slices * a.passes;
  p.clusters = (int)(units < most ? units : most);
  a.team_shift = 4;
  if (a.split > 1) return p;
  // warps to a unit: what finishes first, where a warp's share of a unit costs its steps plus about three (the hand-over
  // at its end), and a CTA's teams work at the same time
  int64_t least = -1;
  for (int ts = 4; ts >= 2; --ts) {
    const int64_t teams = (int64_t)sms << (4 - ts);
    const int64_t cost = (units + teams - 1) / teams * (3 * pages + ((steps + (1 << ts) - 1) >> ts));
    if (least < 0 || cost < least) least = cost, a.team_shift = ts;
  }
  return p;
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

extern "C" pw_status pw_page_linear(pw_ctx* ctx, int T, int K, const void* x_fp16, int64_t x_stride, const pw_page* pages,
                                    const int32_t* out_features, int n_pages, const void* bias, int bias_type, void* out,
                                    int out_type, int64_t out_stride, pw_stream stream) {
  if (!ctx || T < 0 || K < 1 || !pages || n_pages < 1 || n_pages > PW_LINEAR_PAGES || !type_ok(out_type) || (bias && !type_ok(bias_type)))
    return PW_ERR_INVALID_ARG;
  if (T > 1 << 24) return PW_ERR_SHAPE;
  PageLinearArgs a{};
  int64_t slices = 0, columns = 0;
  for (int i = 0; i < n_pages; ++i) {
    const pw_page& p = pages[i];
    const pw_status ps = check_page(p);
    if (ps != PW_OK) return ps;
    const int64_t n = out_features ? out_features[i] : (int64_t)p.rows;
    if (n < 1) return PW_ERR_INVALID_ARG;
    if (n > p.rows || K > (int64_t)p.cols || K <= (int64_t)p.cols - kGroup || p.cols != pages[0].cols) return PW_ERR_SHAPE;
    LinearPage& l = a.page[i];
    l.codes = static_cast<const char*>(p.codes);
    l.bit1 = static_cast<const char*>(p.scales);
    l.bit0 = static_cast<const char*>(p.zps);
    l.fmt = stream_format(p.bits, p.layout == PW_LAYOUT_PLANES);
    l.rows = (int)n;
    l.col0 = (int)columns;
    slices += (n + kUnitRows - 1) / kUnitRows;
    columns += n;
    if (columns > 1 << 30) return PW_ERR_SHAPE;
    l.end = (int)slices;
  }
  if (T == 0) return PW_OK;
  if (!x_fp16 || !out) return PW_ERR_INVALID_ARG;
  if (T > 1 && (x_stride < K || out_stride < columns)) return PW_ERR_SHAPE;
  if (!is_aligned(x_fp16, 16) || !is_aligned(out, 16) || !is_aligned(bias, 16) || (T > 1 && x_stride % 8)) return PW_ERR_ALIGN;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  const pw_status fs = few_setup(ctx);
  if (fs != PW_OK) return fs;
  a.x = static_cast<const char*>(x_fp16);
  a.x_pitch = T > 1 ? (size_t)x_stride * 2 : 0;
  a.out = out;
  a.bias = bias;
  a.ld_out = out_stride;
  a.T = T;
  a.groups = (int)(pages[0].cols / kGroup);
  a.x_bytes = 2 * K;
  a.slices = (int)slices;
  a.out_type = out_type;
  a.bias_type = bias_type;
  const PageLinearPlan p = plan_page_linear(a, ctx->num_sms);
  if (!p.stages) return PW_ERR_SHAPE;
  const size_t smem = page_linear_smem(a, p.stages);
  PW_CUDA_OK(p.stages == 4 ? launch_page_linear<4>(a, p.clusters, smem, stream) : launch_page_linear<3>(a, p.clusters, smem, stream));
  ctx->launches++;
  return PW_OK;
}
