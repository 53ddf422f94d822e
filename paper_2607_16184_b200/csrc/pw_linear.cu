// Product of two matrices in the scaled 8-bit format.
//
//   out[t, n] = sum over blocks g of 128 columns:  sa[t, g] * sw[n / 128, g] * (sum over k in g of a[t, k] * w[n, k])
//
// The inner sums run on the tensor cores (tcgen05.mma, kind::f8f6f4: products of e4m3 codes, fp32 sums in tensor
// memory), one fresh accumulator per block of 128 columns; the scales are applied in fp32 on its way from tensor memory
// to registers, where the sums over the blocks stay.
#include <cuda.h>

#include "pw_ptx.cuh"
#include "pw_scaled.cuh"

namespace pw {

constexpr int kBlockK = 128;                    // columns of a scale block = bytes of an operand row in a stage
constexpr int kWaitPolls = 100000;              // x 20 us suspend time = 2 s
constexpr int kWaitPollsTest = 200;             // 4 ms (pw_debug_set_wait)

struct LinearArgs {
  CUtensorMap ma, mw;                           // codes of a [T, K] and of w [N, K]
  const float* sa;
  const float* sw;
  void* out;
  int32_t* status;
  int64_t ld_out;
  int T, N, G, out_type;
  int polls;
  uint32_t hook;
};

// ---- bounded waits -------------------------------------------------------------------------------
__device__ __forceinline__ bool mbar_try(uint32_t bar_s, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar_s), "r"(parity), "r"(20000u)
      : "memory");
  return ok != 0;
}
// False when the limit ran out or another role of the CTA has given up.
__device__ __forceinline__ bool mbar_wait(uint32_t bar_s, uint32_t parity, volatile int* gave_up, int polls, int32_t* status) {
  if (mbar_try(bar_s, parity)) return true;
  for (int n = 0; n < polls; ++n) {
    if (mbar_try(bar_s, parity)) return true;
    if (*gave_up) return false;
  }
  *gave_up = 1;
  atomicMax(status, (int)PW_ERR_TIMEOUT);
  return false;
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar_s, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar_s), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst_s, const CUtensorMap* map, int x, int y, uint32_t bar_s) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst_s),
               "l"(map), "r"(x), "r"(y), "r"(bar_s)
               : "memory");
}
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar_s) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar_s) : "memory");
}
// Waits for the tensor-memory loads into v[0 .. 15]; the registers pass through, so that no use moves ahead of it.
__device__ __forceinline__ void tmem_wait16(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                 "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :
               : "memory");
}
// Operand tile in shared memory: rows of 128 bytes along K, 128-byte swizzle, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3fffu) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__host__ __device__ constexpr uint32_t e4m3_idesc(int m, int n) {
  return 1u << 4 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;   // fp32 sums, both operands e4m3 and K-major
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float load_cluster(uint32_t addr_s, uint32_t rank) {
  float v;
  asm volatile("{\n\t.reg .b32 p;\n\tmapa.shared::cluster.u32 p, %1, %2;\n\tld.shared::cluster.f32 %0, [p];\n\t}"
               : "=f"(v)
               : "r"(addr_s), "r"(rank)
               : "memory");
  return v;
}

// ---- few rows: the weights on the M side ---------------------------------------------------------
// D[128 weight rows, NT tokens].  A CTA takes one 128-row tile of w, up to NT tokens and a range of the blocks; the
// CTAs of a cluster share the tile and the tokens, each with a range of its own, and add their sums through distributed
// shared memory in rank order (no workspace, the same bits on every run).
//   warps 0-3  tensor memory -> registers, scales, output; thread = weight row
//   warp 4     copies (one stage = a 128 x 128 tile of w and the same columns of NT tokens)
//   warp 5     MMAs; owns tensor memory (two accumulators of NT columns in turn)
constexpr int kFewThreads = 192;
template <int NT>
struct FewCfg {
  static constexpr int kStage = 16384 + NT * 128;
  static constexpr int kStages = NT <= 16 ? 5 : NT <= 32 ? 5 : NT <= 64 ? 4 : 3;   // two CTAs fit on an SM
  static constexpr int kSmem = kStages * kStage + 1024;
  static constexpr int kCols = 2 * NT;
};

template <int NT>
__global__ void __launch_bounds__(kFewThreads) linear_few_kernel(const __grid_constant__ LinearArgs a, int split, int token_tiles) {
  using C = FewCfg<NT>;
  constexpr int S = C::kStages;
  extern __shared__ char smem_raw[];
  __shared__ unsigned long long full[S], empty[S], acc_full[2], acc_empty[2];
  __shared__ uint32_t tmem_base;
  __shared__ volatile int gave_up;
  __shared__ alignas(16) float col_scale[4][2][NT];      // read four at a time
  const uint32_t ring_s = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x % split);
  const int unit = (int)(blockIdx.x / split);
  const int row_tile = unit / token_tiles, tok0 = (unit % token_tiles) * NT;
  const int g0 = (int)((int64_t)a.G * rank / split), g1 = (int)((int64_t)a.G * (rank + 1) / split);
  const int n_blocks = g1 - g0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 4);
    }
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(C::kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  grid_dep_sync();          // codes and scales may come from the kernel directly ahead
  grid_dep_trigger();

  float acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = 0.f;

  if (warp == 4) {
    bool ok = true;
    int i = 0;
    for (; ok && i < n_blocks; ++i) {
      if ((a.hook & 2u) && i == 1) break;          // test hook: the waits on the second stage run out
      const int s = i % S;
      if (i >= S) ok = mbar_wait(smem_u32(&empty[s]), (i / S - 1) & 1, &gave_up, a.polls, a.status);
      if (!ok) break;
      if (lane == 0) {
        const uint32_t bar = smem_u32(&full[s]), dst = ring_s + s * C::kStage;
        mbar_expect_tx(bar, C::kStage);
        tma_load_2d(dst, &a.mw, (g0 + i) * kBlockK, row_tile * 128, bar);
        tma_load_2d(dst + 16384, &a.ma, (g0 + i) * kBlockK, tok0, bar);
      }
      __syncwarp();
    }
    if (!ok)                                       // leave nothing in flight
      for (int j = i < S ? 0 : i - S; j < i; ++j)
        for (int n = 0; n < 200 && !mbar_try(smem_u32(&full[j % S]), (j / S) & 1); ++n) {
        }
  } else if (warp == 5) {
    bool ok = true;
    for (int i = 0; ok && i < n_blocks; ++i) {
      const int s = i % S, b = i & 1;
      if (i >= 2) ok = mbar_wait(smem_u32(&acc_empty[b]), ((i >> 1) - 1) & 1, &gave_up, a.polls, a.status);
      if (ok) ok = mbar_wait(smem_u32(&full[s]), (i / S) & 1, &gave_up, a.polls, a.status);
      if (!ok) break;
      tc_fence_after();
      if (lane == 0) {
        const uint32_t w_s = ring_s + s * C::kStage;
        const uint64_t wd = swizzled_desc(w_s), xd = swizzled_desc(w_s + 16384);
#pragma unroll
        for (int k = 0; k < 4; ++k)                // 32 columns (bytes) per instruction
          mma_e4m3(tmem + b * NT, wd + 2 * k, xd + 2 * k, e4m3_idesc(128, NT), k > 0);
        mma_commit(smem_u32(&empty[s]));
        mma_commit(smem_u32(&acc_full[b]));
      }
      __syncwarp();
    }
  } else {
    const float* sw = a.sw + (int64_t)row_tile * a.G + g0;
    constexpr int M = (NT + 31) / 32;
    float next[M];
    auto fetch = [&](int i) {                      // scales of block i for the columns lane, lane + 32, ..
      const float w = sw[i];
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int j = lane + 32 * m;
        next[m] = j < NT && tok0 + j < a.T ? a.sa[(int64_t)(tok0 + j) * a.G + g0 + i] * w : 0.f;
      }
    };
    if (n_blocks > 0) fetch(0);
    bool ok = true;
    for (int i = 0; ok && i < n_blocks; ++i) {
      const int b = i & 1;
      float* cs = col_scale[warp][b];
      __syncwarp();
#pragma unroll
      for (int m = 0; m < M; ++m)
        if (lane + 32 * m < NT) cs[lane + 32 * m] = next[m];
      __syncwarp();
      if (i + 1 < n_blocks) fetch(i + 1);
      ok = mbar_wait(smem_u32(&acc_full[b]), (i >> 1) & 1, &gave_up, a.polls, a.status);
      if (!ok) break;
      tc_fence_after();
      constexpr int W = NT < 64 ? NT : 64;
#pragma unroll
      for (int h = 0; h < NT; h += W) {
        float v[W];
#pragma unroll
        for (int c = 0; c < W; c += 16) tmem_ld16(tmem + ((uint32_t)(warp * 32) << 16) + b * NT + h + c, v + c);
#pragma unroll
        for (int c = 0; c < W; c += 16) tmem_wait16(v + c);
        if (h + W == NT) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&acc_empty[b]);
        }
#pragma unroll
        for (int j = 0; j < W; j += 4) {
          const float4 f = *reinterpret_cast<const float4*>(cs + h + j);
          acc[h + j] = fmaf(v[j], f.x, acc[h + j]);
          acc[h + j + 1] = fmaf(v[j + 1], f.y, acc[h + j + 1]);
          acc[h + j + 2] = fmaf(v[j + 2], f.z, acc[h + j + 2]);
          acc[h + j + 3] = fmaf(v[j + 3], f.w, acc[h + j + 3]);
        }
      }
    }
  }

  const int n = row_tile * 128 + (int)threadIdx.x;       // threads 0 .. 127: my weight row
  if (split == 1) {
    if (warp < 4 && n < a.N) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
        if (tok0 + j < a.T) store1(a.out, (int64_t)(tok0 + j) * a.ld_out + n, a.out_type, acc[j]);
    }
  } else {
    // every copy has landed and every MMA has read its operands (the last accumulator was complete): the ring is free
    const uint32_t mine_s = ring_s + threadIdx.x * 4;
    if (warp < 4) {
#pragma unroll
      for (int j = 0; j < NT; ++j) asm volatile("st.shared.f32 [%0], %1;" ::"r"(mine_s + j * 512), "f"(acc[j]) : "memory");
    }
    __syncwarp();
    cluster_sync();
    if (warp < 4 && n < a.N) {
      for (int j = NT * rank / split; j < NT * (rank + 1) / split && tok0 + j < a.T; ++j) {
        float v = 0.f;
        for (int r = 0; r < split; ++r) v += load_cluster(mine_s + j * 512, r);
        store1(a.out, (int64_t)(tok0 + j) * a.ld_out + n, a.out_type, v);
      }
    }
    __syncwarp();
    cluster_sync();                                      // nobody leaves while its sums are being read
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 5) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::kCols));
}

// ---- host side -----------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Map of an 8-bit matrix [rows, cols]: boxes of 128 columns, rows and columns past the end read as zero codes.
static bool codes_map(void* encode, const void* base, int rows, int cols, int64_t stride, int box_rows, CUtensorMap* m) {
  const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t pitch[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {(cuuint32_t)kBlockK, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return reinterpret_cast<EncodeTiledFn>(encode)(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dim, pitch, box, step,
                                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static pw_status linear_setup(pw_ctx* ctx) {
  if (ctx->encode_tiled) return PW_OK;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  PW_CUDA_OK(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found));
  if (!fn || found != cudaDriverEntryPointSuccess) return PW_ERR_CUDA;
  PW_CUDA_OK(cudaFuncSetAttribute(linear_few_kernel<16>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<16>::kSmem));
  PW_CUDA_OK(cudaFuncSetAttribute(linear_few_kernel<32>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<32>::kSmem));
  PW_CUDA_OK(cudaFuncSetAttribute(linear_few_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<64>::kSmem));
  PW_CUDA_OK(cudaFuncSetAttribute(linear_few_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<128>::kSmem));
  ctx->encode_tiled = fn;
  return PW_OK;
}

static cudaError_t launch_cluster(void (*kernel)(LinearArgs, int, int), unsigned ctas, unsigned cluster, int threads, size_t smem,
                                  cudaStream_t s, const LinearArgs& a, int p0, int p1) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a, p0, p1);
}

template <int NT>
static pw_status launch_few(pw_ctx* ctx, LinearArgs& a, int64_t row_tiles, int64_t token_tiles, cudaStream_t s) {
  // Split the blocks over a cluster until there are two CTAs per SM, and at least two blocks per CTA.
  int split = 1;
  while (split < 8 && row_tiles * token_tiles * split * 2 <= 2 * ctx->num_sms && a.G >= split * 4) split *= 2;
  const int64_t ctas = row_tiles * token_tiles * split;
  if (ctas > 0x7fffffff) return PW_ERR_SHAPE;
  PW_CUDA_OK(launch_cluster(linear_few_kernel<NT>, (unsigned)ctas, split, kFewThreads, FewCfg<NT>::kSmem, s, a, split, (int)token_tiles));
  return PW_OK;
}

}  // namespace pw

using namespace pw;

extern "C" pw_status pw_scaled_linear(pw_ctx* ctx, int T, int N, int K, const void* a_codes, int64_t a_stride,
                                      const float* a_scales, const void* w_codes, int64_t w_stride, const float* w_scales,
                                      void* out, int out_type, int64_t out_stride, pw_stream stream) {
  if (!ctx || T < 0 || N < 1 || K < 1 || !type_ok(out_type)) return PW_ERR_INVALID_ARG;
  if (N > 1 << 30 || K > 1 << 30) return PW_ERR_SHAPE;
  if (T == 0) return PW_OK;
  if (!a_codes || !a_scales || !w_codes || !w_scales || !out) return PW_ERR_INVALID_ARG;
  if ((T > 1 && (a_stride < K || out_stride < N)) || (N > 1 && w_stride < K)) return PW_ERR_SHAPE;
  const void* ptrs[5] = {a_codes, a_scales, w_codes, w_scales, out};
  for (const void* p : ptrs)
    if (!is_aligned(p, 16)) return PW_ERR_ALIGN;
  if (a_stride % 16 || w_stride % 16) return PW_ERR_ALIGN;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  pw_status st = linear_setup(ctx);
  if (st != PW_OK) return st;
  LinearArgs a;
  a.sa = a_scales;
  a.sw = w_scales;
  a.out = out;
  a.status = reinterpret_cast<int32_t*>(ctx->base + ctx->ws.status);
  a.ld_out = out_stride;
  a.T = T;
  a.N = N;
  a.G = (K + kBlockK - 1) / kBlockK;
  a.out_type = out_type;
  a.polls = ctx->wait_polls ? kWaitPollsTest : kWaitPolls;
  a.hook = ctx->test_hook;
  const int64_t row_tiles = ((int64_t)N + 127) / 128;
  const int nt = T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128;
  const int64_t token_tiles = ((int64_t)T + nt - 1) / nt;
  // a single row's stride is never used: give the map one that it accepts
  const int64_t min_pitch = ((int64_t)K + 15) / 16 * 16;
  const int64_t pa = a_stride < min_pitch ? min_pitch : a_stride, pwgt = w_stride < min_pitch ? min_pitch : w_stride;
  if (!codes_map(ctx->encode_tiled, a_codes, T, K, pa, nt, &a.ma) || !codes_map(ctx->encode_tiled, w_codes, N, K, pwgt, 128, &a.mw))
    return PW_ERR_CUDA;
  st = nt == 16   ? launch_few<16>(ctx, a, row_tiles, token_tiles, stream)
       : nt == 32 ? launch_few<32>(ctx, a, row_tiles, token_tiles, stream)
       : nt == 64 ? launch_few<64>(ctx, a, row_tiles, token_tiles, stream)
                  : launch_few<128>(ctx, a, row_tiles, token_tiles, stream);
  if (st == PW_OK) ctx->launches++;
  return st;
}
