// Product of two matrices in the scaled 8-bit format.
//
//   out[t, n] = sum over blocks g of 128 columns:  sa[t, g] * sw[n / 128, g] * (sum over k in g of a[t, k] * w[n, k])
//
// The inner sums run on the tensor cores (tcgen05.mma, kind::f8f6f4: products of e4m3 codes, fp32 sums in tensor
// memory), one fresh accumulator per block of 128 columns; the scales are applied in fp32 on its way from tensor memory
// to registers, where the sums over the blocks stay.  Their product is rounded once; where it leaves fp32's range, or has
// fewer than 24 bits there, a power of two goes onto the block's sum instead (split_factor).
#include <cuda.h>

#include "pw_ptx.cuh"
#include "pw_scaled.cuh"

namespace pw {

constexpr int kBlockK = 128;                    // columns of a scale block = bytes of an operand row in a stage
constexpr int kScaleRun = 8;                    // scales of a row travel eight blocks (a 32-byte sector) at a time
constexpr int kWaitPolls = 100000;              // x 20 us suspend time = 2 s
constexpr int kWaitPollsTest = 200;             // 4 ms (pw_debug_set_wait)

struct LinearArgs {
  CUtensorMap ma, mw;                           // codes of a [T, K] and of w [N, K]
  CUtensorMap mo;                               // the output, in boxes of 32 rows x 128 bytes (with tma_out)
  const float* sa;
  const float* sw;
  void* out;
  int32_t* status;
  int64_t ld_out;
  int T, N, G, out_type;
  int tma_out;
  int polls;
  uint32_t hook;
};

// ---- bounded waits -------------------------------------------------------------------------------
// One look at a phase, with the suspend time of a poll or without any.  CLUSTER: what the phase counted was written by
// other CTAs of the cluster, so its completion is acquired at that scope (the instruction's own is the CTA).
template <bool SUSPEND, bool CLUSTER = false>
__device__ __forceinline__ bool mbar_look(uint32_t bar_s, uint32_t parity) {
  uint32_t ok;
  if constexpr (CLUSTER)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar_s), "r"(parity), "r"(20000u)
        : "memory");
  else if constexpr (SUSPEND)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar_s), "r"(parity), "r"(20000u)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar_s), "r"(parity)
        : "memory");
  return ok != 0;
}
// Whether any lane has seen the phase.  A lane that has not goes on all the same, and reads what was written before the
// phase by order of the one that has: a vote orders no memory, __syncwarp does.
__device__ __forceinline__ bool warp_saw(bool ok) {
  const bool any = __any_sync(0xffffffffu, ok);
  __syncwarp();
  return any;
}
// Called by a whole warp, with the same answer for all lanes: the lanes of one poll may see the phase flip at different
// moments, and what follows a wait (tensor-memory loads, cluster barriers) must not be run by a part of the warp.
// False when the limit ran out or another role of the CTA has given up.  (The first look goes without a suspend time: a
// phase that is complete costs 79 cycles, with one 105.)
template <bool CLUSTER = false>
__device__ __forceinline__ bool mbar_wait(uint32_t bar_s, uint32_t parity, volatile int* gave_up, int polls, int32_t* status) {
  if (warp_saw(mbar_look<false, CLUSTER>(bar_s, parity))) return true;
#pragma unroll 1
  for (int n = 0; n < polls; ++n) {
    if (warp_saw(mbar_look<true, CLUSTER>(bar_s, parity))) return true;
    if (__any_sync(0xffffffffu, *gave_up != 0)) return false;
  }
  *gave_up = 1;
  atomicMax(status, (int)PW_ERR_TIMEOUT);
  return false;
}
// The forms of a copy warp: the whole warp runs its loop on the same values and the lane with on != 0 acts, so that the
// operands stay in uniform registers, where these instructions take them from.  (From one lane inside a branch an
// expected count and a copy took 300 cycles, and one warp could not ask for more than 71 GB/s.)
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar_s, uint32_t bytes, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar_s), "r"(bytes), "r"(on)
      : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst_s, const CUtensorMap* map, int x, int y, uint32_t bar_s, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(dst_s),
      "l"(map), "r"(x), "r"(y), "r"(bar_s), "r"(on)
      : "memory");
}
// The MMAs of one block (four steps of 32 columns) and the commit behind them, on the stage's `done` barrier: the stage
// is free again and its accumulators complete.  The whole warp runs this on the same values and the lane with on != 0
// issues: the operands can then live in uniform registers, which a single lane inside a branch would have to fill for
// every instruction.  PAIR: the forms of a CTA pair, whose commit arrives on the barrier at this offset in both CTAs.
template <bool PAIR>
__device__ __forceinline__ void mma_block(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t done, uint32_t on) {
  if constexpr (PAIR) {
    asm volatile(
        "{\n\t.reg .pred q, f, t;\n\t.reg .b32 x, y;\n\t.reg .b64 ad, bd;\n\t.reg .b16 both;\n\tmov.b16 both, 3;\n\t"
        "setp.ne.b32 q, %6, 0;\n\tsetp.ne.b32 f, 0, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
        "mov.b64 ad, {%1, %3};\n\tmov.b64 bd, {%2, %3};\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], ad, bd, %4, f;\n\t"
        "add.u32 x, %1, 2;\n\tadd.u32 y, %2, 2;\n\tmov.b64 ad, {x, %3};\n\tmov.b64 bd, {y, %3};\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], ad, bd, %4, t;\n\t"
        "add.u32 x, %1, 4;\n\tadd.u32 y, %2, 4;\n\tmov.b64 ad, {x, %3};\n\tmov.b64 bd, {y, %3};\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], ad, bd, %4, t;\n\t"
        "add.u32 x, %1, 6;\n\tadd.u32 y, %2, 6;\n\tmov.b64 ad, {x, %3};\n\tmov.b64 bd, {y, %3};\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], ad, bd, %4, t;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], both;\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(done), "r"(on)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred q, f, t;\n\t.reg .b32 x, y;\n\t.reg .b64 ad, bd;\n\t"
        "setp.ne.b32 q, %6, 0;\n\tsetp.ne.b32 f, 0, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
        "mov.b64 ad, {%1, %3};\n\tmov.b64 bd, {%2, %3};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, f;\n\t"
        "add.u32 x, %1, 2;\n\tadd.u32 y, %2, 2;\n\tmov.b64 ad, {x, %3};\n\tmov.b64 bd, {y, %3};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, t;\n\t"
        "add.u32 x, %1, 4;\n\tadd.u32 y, %2, 4;\n\tmov.b64 ad, {x, %3};\n\tmov.b64 bd, {y, %3};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, t;\n\t"
        "add.u32 x, %1, 6;\n\tadd.u32 y, %2, 6;\n\tmov.b64 ad, {x, %3};\n\tmov.b64 bd, {y, %3};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, t;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(done), "r"(on)
        : "memory");
  }
}
// Arrives on `done` once the MMAs that this thread has issued so far are complete.
__device__ __forceinline__ void mma_commit(uint32_t done, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(done),
      "r"(on)
      : "memory");
}
// Waits for the tensor-memory loads into v[0 .. 15]; the registers pass through, so that no use moves ahead of it.
__device__ __forceinline__ void tmem_wait16(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                 "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :
               : "memory");
}
// Two fp32 multiply-adds in one instruction, each rounded once.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  return r;
}
// Operand tile in shared memory: rows of 128 bytes along K, 128-byte swizzle, groups of eight rows 1024 bytes apart.
// The descriptor's low word is the address (and a leading offset that this layout ignores), 32 columns = 2 further on;
// the high word: offset between the groups, version of sm_100, swizzle mode.
__device__ __forceinline__ uint32_t swizzled_lo(uint32_t saddr) { return ((saddr >> 4) & 0x3fffu) | 1u << 16; }
constexpr uint32_t kSwizzledHi = (1024u >> 4) | 1u << 14 | 2u << 29;
__host__ __device__ constexpr uint32_t e4m3_idesc(int m, int n) {
  return 1u << 4 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;   // fp32 sums, both operands e4m3 and K-major
}
// (all lanes of a warp together)
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr_s, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr_s), "r"(rank));
  return r;
}
// What a block's sum is multiplied with: the product of two scales, as f * m with m a power of two.  Scales are 2^-126 or
// more and sums 2^-18 to 2^24.7 (or 0), so that the product of two scales can leave fp32's range on either side where the
// result does not.  m goes onto the sum first, exactly, and f keeps its 24 bits: below the range down to 2^-174, where even
// the largest sum underflows, above it up to 2^176, where the smallest one overflows.
struct Factor {
  float f, m;
};
__device__ __forceinline__ Factor split_factor(float x, float y) {
  Factor r{x * y, 1.f};
  if (x == 0.f || y == 0.f || !(fabsf(x) <= 3.402823466e38f && fabsf(y) <= 3.402823466e38f)) return r;
  if (fabsf(r.f) < 1.17549435e-38f) {
    r.f = (x * 16777216.f) * (y * 16777216.f);                  // 2^24 each
    r.m = 3.5527137e-15f;                                       // 2^-48
  } else if (fabsf(r.f) > 3.402823466e38f) {
    r.f = fminf(fmaxf((x * 5.9604645e-8f) * (y * 5.9604645e-8f), -3.402823466e38f), 3.402823466e38f);
    r.m = 2.8147498e14f;
  }
  return r;
}
// Scales of ROWS rows and the blocks g .. g + 7, one warp: a sector of 32 bytes per row, all loads in flight together,
// stored as [block][row] (rows padded by four, which keeps both sides free of bank conflicts).  Rows and blocks past the
// end, whose codes read as 0, get `past`.
template <int ROWS, class Store>
__device__ __forceinline__ void load_scales(const float* sa, int64_t row0, int T, int G, int g, int g_end, float past, int lane, Store store) {
  constexpr int kLoads = ROWS / 4 < 16 ? ROWS / 4 : 16;      // in flight at a time
  const int j = lane & 7, r0 = lane >> 3;
  const bool in = g + j < g_end;
#pragma unroll 1
  for (int base = 0; base < ROWS; base += kLoads * 4) {
    float v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int64_t r = row0 + base + i * 4 + r0;
      v[i] = in && r < T ? sa[r * G + g + j] : past;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) store(j * (ROWS + 4) + base + i * 4 + r0, v[i]);
  }
}
// The same times w, a lane's scale of the weights for block g + lane % 8 (1 past the end).  Returns whether one of the
// products is 0, subnormal or no number; then they are split_factor's, with the powers of two beside them.
template <int ROWS>
__device__ __forceinline__ bool load_products(const float* sa, int64_t row0, int T, int G, int g, int g_end, float w, float* dst, float* powers,
                                              int lane) {
  uint32_t worst = 0;                              // an exponent of 0 wraps round to the top
  load_scales<ROWS>(sa, row0, T, G, g, g_end, 1.f, lane, [&](int at, float v) {
    const float f = v * w;
    worst = max(worst, 2 * __float_as_uint(f) - 0x01000000u);
    dst[at] = f;
  });
  const bool any = __any_sync(0xffffffffu, worst >= 0xfe000000u);
  if (any)
    load_scales<ROWS>(sa, row0, T, G, g, g_end, 1.f, lane, [&](int at, float v) {
      const Factor x = split_factor(v, w);
      dst[at] = x.f;
      powers[at] = x.m;
    });
  return any;
}
// Whether a product of one of ROWS x 8 scales in shared memory and a scale between two others can leave the range.
template <int ROWS>
__device__ __forceinline__ bool products_leave(const float* scales, float w_low, float w_high, int lane) {
  static_assert(ROWS == 128, "four rows a lane");
  uint32_t least = 0xffffffffu;                    // twice the smallest magnitude's bits, less one: 0 is the largest
  float high = 0.f;
#pragma unroll
  for (int j = 0; j < kScaleRun; ++j) {
    const float4 q = *reinterpret_cast<const float4*>(scales + j * (ROWS + 4) + lane * 4);
    least = min(min(least, 2 * __float_as_uint(q.x) - 1), 2 * __float_as_uint(q.y) - 1);
    least = min(min(least, 2 * __float_as_uint(q.z) - 1), 2 * __float_as_uint(q.w) - 1);
    high = fmaxf(fmaxf(high, fabsf(q.x)), fabsf(q.y));
    high = fmaxf(fmaxf(high, fabsf(q.z)), fabsf(q.w));
  }
  const float low = __uint_as_float((least >> 1) + 1);
  return __any_sync(0xffffffffu, high > 0.f && (low * w_low < 1.17549435e-38f || high * w_high > 3.402823466e38f));
}

// ---- few rows: the weights on the M side ---------------------------------------------------------
// D[128 weight rows, NT tokens].  A CTA takes one 128-row tile of w, up to NT tokens and a range of the blocks; the
// CTAs of a cluster share the tile and the tokens, each with a range of its own.  Every four tokens have an owner among
// them: the others store their sums for those into its shared memory (counted on a barrier there), and it adds them in
// rank order: no workspace, the same bits on every run.  One CTA per SM, its ring as deep as shared memory, for the weights
// come from HBM; persistent where there are more tiles than SMs (a cluster takes one unit only).
// A stage holds two blocks: what every role spends per barrier phase (a look 80 cycles, a copy or an MMA 70 to 90) is
// what bounds it where the weights are in L2.
//   warps 0 .. kSum - 1  tensor memory -> registers, scales, output; thread = weight row, four warps for 16 tokens (with
//              32 tokens to a warp 64 x 14336 x 4096 took 15.8 us instead of 14.6)
//   then one   copies (128 x 128 tiles of w and the same columns of NT tokens)
//   then two   MMAs, the first and the second block of every stage; the first owns tensor memory: an accumulator of NT
//              columns per block of the ring, so a stage that has been filled again says that its accumulators have been
//              read.  (Stages in turn between the two would need an even number of them: a warp that sees every other phase
//              of a barrier can take an old one for the one it waits for.)
//   then one   scales, eight blocks at a time, multiplied, into shared memory: loaded by the warps that use them they
//              were 16 times as many requests as they are sectors, and the bound of the kernel
// 64 x 14336 x 4096: 14.4 us (weights once from HBM: 8.9; the rest is the launch, filling and draining), one token 12.1;
// one token x 4096 x 4096: 5.1.
template <int NT, bool SPLIT>
struct FewCfg {
  static constexpr int kSum = NT / 4;              // four warps for 16 tokens each
  static constexpr int kThreads = (kSum + 4) * 32;
  static constexpr int kBlock = 16384 + NT * 128;  // bytes of a block in the ring
  static constexpr int kStages = NT <= 32 ? 5 : SPLIT ? 3 : 4;
  static constexpr int kChunks = NT / 4;           // of four tokens
  // what a CTA receives at most: its share of the chunks, rounded up, from every CTA of a cluster of 2 to 5, or 8
  static constexpr int kSums = SPLIT ? (NT <= 16 ? 8 : NT <= 32 ? 10 : 20) * 2048 : 0;
  static_assert(!SPLIT || ((kChunks + 2) / 3 * 3 * 2048 <= kSums && (kChunks + 4) / 5 * 5 * 2048 <= kSums && (kChunks + 7) / 8 * 8 * 2048 <= kSums), "");
  static constexpr int kSmem = kStages * 2 * kBlock + kSums + 1024;
  static constexpr int kCols = NT <= 16 ? 256 : 512;
  static_assert(kStages * 2 * NT <= kCols, "an accumulator per block of the ring");
};
// 16 bytes into the shared memory of a CTA of the cluster, counted on a barrier there.
__device__ __forceinline__ void send4(uint32_t dst, float x, float y, float z, float w, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst), "f"(x), "f"(y), "f"(z),
               "f"(w), "r"(bar)
               : "memory");
}
__device__ __forceinline__ float lo_of(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi_of(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }

template <int NT, bool SPLIT>
__global__ void __launch_bounds__(FewCfg<NT, SPLIT>::kThreads, 1)
    linear_few_kernel(const __grid_constant__ LinearArgs a, int token_tiles, int n_units, int split) {
  using C = FewCfg<NT, SPLIT>;
  constexpr int S = C::kStages, NW = C::kSum, QC = 16;   // columns of a summing warp
  extern __shared__ char smem_raw[];
  __shared__ unsigned long long full[S], done[S], freed[S], sc_full[2], sc_empty[2], sums_in;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int gave_up;
  __shared__ alignas(16) float scales[2][kScaleRun][NT + 4], powers[2][kScaleRun][NT + 4];   // read four at a time
  __shared__ int extreme_run[2];                                 // whether there are powers
  const uint32_t ring_s = (smem_u32(smem_raw) + 1023u) & ~1023u, sums_s = ring_s + S * 2 * C::kBlock;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x % split);
  const int unit0 = (int)(blockIdx.x / split), stride = (int)(gridDim.x / split);   // unit: (row tile, token tile), token tiles fastest
  const int g0 = (int)((int64_t)a.G * rank / split), g1 = (int)((int64_t)a.G * (rank + 1) / split);
  // chunks of four tokens that this CTA adds up: rank, rank + split, ..
  const int chunks = SPLIT ? (min(a.T - unit0 % token_tiles * NT, NT) + 3) / 4 : 0;
  const int mine = rank < chunks ? (chunks - 1 - rank) / split + 1 : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&done[i], 2);                      // both MMA warps
      mbar_init(&freed[i], NW);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sc_full[i], 1);
      mbar_init(&sc_empty[i], NW);
    }
    mbar_init(&sums_in, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (mine > 0) mbar_expect_tx(smem_u32(&sums_in), (uint32_t)(mine * split) * 2048u, 1u);
  }
  if constexpr (SPLIT) cluster_arrive();
  if (warp == NW + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(C::kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  if constexpr (SPLIT) cluster_wait();                   // the others' barriers are ready
  grid_dep_sync();          // codes and scales may come from the kernel directly ahead
  grid_dep_trigger();

  if (warp == NW) {
    bool ok = true;
    int i = 0, s = 0;
    uint32_t par = 1;                              // of the stage's next `freed` phase (the first pass waits for none)
    const uint32_t on = lane == 0 ? 1u : 0u, full_s = smem_u32(&full[0]);
    for (int u = unit0; ok && u < n_units; u += stride) {
      const int row0 = u / token_tiles * 128, tok0 = u % token_tiles * NT;
      for (int g = g0; g < g1; g += 2, ++i) {
        if ((a.hook & 2u) && i == 1) ok = false;   // test hook: the waits on the second stage run out
        if (ok && i >= S) ok = mbar_wait(smem_u32(&freed[s]), par, &gave_up, a.polls, a.status);
        if (!ok) break;
        const uint32_t bar = full_s + 8 * s, dst = ring_s + s * 2 * C::kBlock, second = g + 1 < g1 ? on : 0u;
        mbar_expect_tx(bar, g + 1 < g1 ? 2 * C::kBlock : C::kBlock, on);
        tma_load_2d(dst, &a.mw, g * kBlockK, row0, bar, on);
        tma_load_2d(dst + 16384, &a.ma, g * kBlockK, tok0, bar, on);
        tma_load_2d(dst + C::kBlock, &a.mw, (g + 1) * kBlockK, row0, bar, second);
        tma_load_2d(dst + C::kBlock + 16384, &a.ma, (g + 1) * kBlockK, tok0, bar, second);
        if (++s == S) {
          s = 0;
          par ^= 1u;
        }
      }
    }
    if (!ok)                                       // leave nothing in flight
      for (int j = i < S ? 0 : i - S; j < i; ++j)
        for (int n = 0; n < 200 && !mbar_look<true>(smem_u32(&full[j % S]), (j / S) & 1); ++n) {
        }
  } else if (warp == NW + 1 || warp == NW + 2) {
    bool ok = true;
    int s = 0;
    uint32_t par = 0;                              // of the stage's next `full` phase
    const int k = warp - NW - 1;                   // which of the two blocks
    const uint32_t on = lane == 0 ? 1u : 0u, full_s = smem_u32(&full[0]), done_s = smem_u32(&done[0]);
    for (int u = unit0; ok && u < n_units; u += stride)
      for (int g = g0; g < g1; g += 2) {
        ok = mbar_wait(full_s + 8 * s, par, &gave_up, a.polls, a.status);
        if (!ok) break;
        tc_fence_after();
        const uint32_t w_s = ring_s + (s * 2 + k) * C::kBlock;
        if (g + k < g1)
          mma_block<false>(tmem + (s * 2 + k) * NT, swizzled_lo(w_s), swizzled_lo(w_s + 16384), kSwizzledHi, e4m3_idesc(128, NT), done_s + 8 * s, on);
        else
          mma_commit(done_s + 8 * s, on);
        if (++s == S) {
          s = 0;
          par ^= 1u;
        }
      }
  } else if (warp == NW + 3) {
    bool ok = true;
    int run = 0;
    for (int u = unit0; ok && u < n_units; u += stride) {
      const float* sw = a.sw + (int64_t)(u / token_tiles) * a.G;
      for (int g = g0; g < g1; g += kScaleRun, ++run) {
        const float w = g + (lane & 7) < g1 ? sw[g + (lane & 7)] : 1.f;
        if (run >= 2) ok = mbar_wait(smem_u32(&sc_empty[run & 1]), ((run >> 1) - 1) & 1, &gave_up, a.polls, a.status);
        if (!ok) break;
        const bool any = load_products<NT>(a.sa, (int64_t)(u % token_tiles) * NT, a.T, a.G, g, g1, w, scales[run & 1][0], powers[run & 1][0], lane);
        if (lane == 0) extreme_run[run & 1] = any;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sc_full[run & 1]);
      }
    }
  } else {
    const int col = (warp >> 2) * QC, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + col;
    bool ok = true, extreme = false;
    int s = 0, run = 0;
    uint32_t par = 0;                              // of the stage's next `done` phase
    uint64_t acc[QC / 2];                          // pairs of tokens: a packed multiply-add does two
    for (int u = unit0; u < n_units; u += stride) {
#pragma unroll
      for (int j = 0; j < QC / 2; ++j) acc[j] = 0;
      int in_run = 0;
#pragma unroll 1
      for (int g = g0; ok && g < g1; g += 2) {
        if (in_run == 0) {
          ok = mbar_wait(smem_u32(&sc_full[run & 1]), (run >> 1) & 1, &gave_up, a.polls, a.status);
          extreme = extreme_run[run & 1] != 0;
        }
        if (ok) ok = mbar_wait(smem_u32(&done[s]), par, &gave_up, a.polls, a.status);
        if (!ok) break;
        tc_fence_after();
        const bool two = g + 1 < g1;
        float v[2][QC];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int c = 0; c < QC; c += 16)
            if (k == 0 || two) tmem_ld16(lane_base + (s * 2 + k) * NT + c, v[k] + c);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int c = 0; c < QC; c += 16) tmem_wait16(v[k] + c);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&freed[s]);
        if (extreme) {                               // rare; kept this small: with the scales loaded and split here 4 % on 256 x 4096 x 4096
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < QC; j += 4) {
              const float4 m = *reinterpret_cast<const float4*>(&powers[run & 1][in_run + k][col + j]);
              v[k][j] *= m.x;
              v[k][j + 1] *= m.y;
              v[k][j + 2] *= m.z;
              v[k][j + 3] *= m.w;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (k == 1 && !two) break;
          const ulonglong2* cs = reinterpret_cast<const ulonglong2*>(scales[run & 1][in_run + k] + col);
#pragma unroll
          for (int j = 0; j < QC / 4; ++j) {
            const ulonglong2 f = cs[j];
            acc[2 * j] = fma2(pack2(v[k][4 * j], v[k][4 * j + 1]), f.x, acc[2 * j]);
            acc[2 * j + 1] = fma2(pack2(v[k][4 * j + 2], v[k][4 * j + 3]), f.y, acc[2 * j + 1]);
          }
        }
        in_run += 2;
        if (in_run == kScaleRun || g + 2 >= g1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&sc_empty[run & 1]);
          in_run = 0;
          ++run;
        }
        if (++s == S) {
          s = 0;
          par ^= 1u;
        }
      }
      const int64_t n = (int64_t)(u / token_tiles) * 128 + row;
      const int t0 = u % token_tiles * NT;
      if constexpr (!SPLIT) {
        if (ok && n < a.N) {
#pragma unroll
          for (int j = 0; j < QC; ++j)
            if (t0 + col + j < a.T)
              store1(a.out, (int64_t)(t0 + col + j) * a.ld_out + n, a.out_type, j & 1 ? hi_of(acc[j / 2]) : lo_of(acc[j / 2]));
        }
        __syncwarp();
        if (!ok) break;
        continue;
      }
      // [owner's chunk][rank][row] of four tokens.  Whoever gave up on a wait sends all the same, so the wait for the
      // others' sums outlasts any of theirs; a CTA that has received what is its own is sent nothing more and may leave.
#pragma unroll
      for (int k = 0; k < QC / 4; ++k) {
        const int c = col / 4 + k;
        if (c < chunks) {
          const int lc = c / split, owner = c - lc * split;
          send4(map_rank(sums_s + ((lc * split + rank) * 128 + row) * 16, owner), lo_of(acc[2 * k]), hi_of(acc[2 * k]), lo_of(acc[2 * k + 1]),
                hi_of(acc[2 * k + 1]), map_rank(smem_u32(&sums_in), owner));
        }
      }
      __syncwarp();
      volatile int no_matter = 0;
      if (mine > 0 && mbar_wait<true>(smem_u32(&sums_in), 0, &no_matter, 8 * a.polls, a.status) && n < a.N) {
        const float4* sums = reinterpret_cast<const float4*>(smem_raw + (sums_s - smem_u32(smem_raw))) + row;
        for (int lc = warp >> 2; lc < mine; lc += NW / 4) {
          float4 x = sums[lc * split * 128];
          for (int r = 1; r < split; ++r) {
            const float4 y = sums[(lc * split + r) * 128];
            x.x += y.x;
            x.y += y.y;
            x.z += y.z;
            x.w += y.w;
          }
          const int t = t0 + (lc * split + rank) * 4;
          const float o[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (t + j < a.T) store1(a.out, (int64_t)(t + j) * a.ld_out + n, a.out_type, o[j]);
        }
      }
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  __syncwarp();
  if (warp == NW + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::kCols));
}

// ---- many rows: pairs of CTAs --------------------------------------------------------------------
// D[256 tokens, BN weight rows] by two CTAs of a cluster on one tile (cta_group::2): each holds 128 of the token rows and
// half of the weight rows in its shared memory, and the accumulators of its own 128 tokens.  A block of 128 columns gets
// a fresh accumulator (512 / BN of them in turn); its sums leave tensor memory in one pass, are scaled and stay in
// registers until the tile is complete, so the epilogue warps work all the time, next to the MMAs.
//   warps 0-7   tensor memory -> registers, scales, output: warps 0-3 the first half of the columns, 4-7 the second;
//               thread = token row
//   warp 8      copies (both CTAs; a stage = 128 token rows and BN / 2 weight rows of one block, all counted on the
//               first CTA's barrier)
//   warps 9,10  MMAs (first CTA only), even and odd blocks; warp 9 owns tensor memory
//   warp 11     scales, eight blocks at a time, into shared memory
// The last four warps hand most of their registers to the first eight, whose sums fill 128 each.
// Persistent: a pair takes every n_pairs-th tile, token tiles fastest, so that the pairs at work share weight rows in L2.
// 4096 x 14336 x 4096: 222 to 231 us from GPU to GPU = 2.1 to 2.2 PFLOP/s (power capped in a loop: 265).  When it took 220,
// the MMAs alone were 153 of them and the epilogue alone 182: a block's 64 packed multiply-adds per warp (320 cycles of the
// FMA pipe) come behind the wait for its accumulator, of which two fill tensor memory.  Sixteen epilogue warps (240) and
// accumulators handed over in halves (222 to 249) were no faster.
constexpr int kPairThreads = 384;
template <int BN>
struct PairCfg {
  static constexpr int kStage = 16384 + BN / 2 * 128;
  static constexpr int kStages = BN == 256 ? 4 : 6;   // 128 KB in flight: what the latency of L2 times its rate asks for
  static_assert(kStages % 2 == 0, "a stage belongs to one MMA warp, see linear_few_kernel");
  static constexpr int kSmem = kStages * kStage + 65536 + 1024;   // and two boxes of output for each of eight warps
  static constexpr int kAcc = 512 / BN;           // accumulators in tensor memory (an even number, for the same reason)
};
// copy into this CTA's shared memory, counted on a barrier of the pair (shared::cluster address)
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst_s, const CUtensorMap* map, int x, int y, uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(dst_s),
      "l"(map), "r"(x), "r"(y), "r"(bar), "r"(on)
      : "memory");
}
// (nothing in memory is handed over with it, only tensor memory, which the tcgen05 fences order: a release at cluster
// scope would make the warp wait for its outstanding loads and stores first)
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait32(float* v) {
  tmem_wait16(v);
  tmem_wait16(v + 16);
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int x, int y, uint32_t src_s) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src_s) : "memory");
}

// A warp's 32 rows x COLS outputs, thread = row, by way of boxes of 32 rows x 128 bytes in shared memory (128-byte
// swizzle: 16-byte piece c of row r lies at c ^ (r mod 8)).  With a tensor map of the output the boxes leave by
// asynchronous copies, while the next tile is being summed; a box is written again once its copy has read it.  Without
// one (rows that are no multiple of 16 bytes long and apart) the lanes store element by element, contiguous along a row.
// (Stored straight from registers, 32 rows apart in every instruction, a tile's output took 10000 cycles.)
// One box: `words` are the row's 128 bytes.
__device__ __forceinline__ void store_box(uint32_t box_s, const char* box, const uint32_t* words, const LinearArgs& a, int64_t m0, int n, int size, int lane) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box_s + lane * 128 + ((c ^ (lane & 7)) << 4)), "r"(words[c * 4]),
                 "r"(words[c * 4 + 1]), "r"(words[c * 4 + 2]), "r"(words[c * 4 + 3])
                 : "memory");
  if (a.tma_out) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      if (m0 < a.T && n < a.N) tma_store_2d(&a.mo, n, (int)m0, box_s);   // rows and columns past the end are left out
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  } else {
    __syncwarp();
    for (int r = 0; r < 32 && m0 + r < a.T; ++r)
      for (int e = lane; e * size < 128 && n + e < a.N; e += 32) {
        const int byte = e * size;
        const char* from = box + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15);
        const int64_t at = (m0 + r) * a.ld_out + n + e;
        if (size == 4) static_cast<uint32_t*>(a.out)[at] = *reinterpret_cast<const uint32_t*>(from);
        else static_cast<uint16_t*>(a.out)[at] = *reinterpret_cast<const uint16_t*>(from);
      }
    __syncwarp();
  }
}
template <int COLS>
__device__ __forceinline__ void store_tile(uint32_t box_s, const char* box, const uint64_t* acc, const LinearArgs& a, int64_t m0, int n0, int lane) {
  uint32_t words[32];
  auto boxes_read = [&] {                                     // by the copies so far
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
  };
  boxes_read();
  if (a.out_type == PW_F32) {
#pragma unroll
    for (int p = 0; p < COLS / 32; ++p) {
      if (p == 2) boxes_read();
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        words[2 * j] = (uint32_t)acc[p * 16 + j];
        words[2 * j + 1] = (uint32_t)(acc[p * 16 + j] >> 32);
      }
      store_box(box_s + (p & 1) * 4096, box + (p & 1) * 4096, words, a, m0, n0 + p * 32, 4, lane);
    }
  } else {
    const bool half = a.out_type == PW_F16;
#pragma unroll
    for (int p = 0; p < COLS / 64; ++p) {
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const float lo = __uint_as_float((uint32_t)acc[p * 32 + j]), hi = __uint_as_float((uint32_t)(acc[p * 32 + j] >> 32));
        words[j] = half ? pack_half(lo, hi) : pack_bf(lo, hi);
      }
      store_box(box_s + p * 4096, box + p * 4096, words, a, m0, n0 + p * 64, 2, lane);
    }
  }
}

template <int BN>
__global__ void __launch_bounds__(kPairThreads, 1) linear_pair_kernel(const __grid_constant__ LinearArgs a, int token_tiles, int n_tiles) {
  using C = PairCfg<BN>;
  constexpr int S = C::kStages, A = C::kAcc, HC = BN / 2;
  static_assert(A <= S, "a stage's barrier stands for its accumulator too");
  extern __shared__ char smem_raw[];
  __shared__ unsigned long long full[S], done[S], acc_empty[A], sc_full[2], sc_empty[2];
  __shared__ uint32_t tmem_base;
  __shared__ volatile int gave_up;
  __shared__ alignas(16) float scales[2][kScaleRun][128 + 4];    // read four at a time
  __shared__ float w_scales[2][2][kScaleRun];
  __shared__ int extreme_run[2];                                 // whether split_factor may have anything to do for them
  const uint32_t ring_s = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = blockIdx.x & 1;           // cluster of two along x
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&done[i], 1);
    }
    for (int i = 0; i < A; ++i) mbar_init(&acc_empty[i], 16);   // the epilogue warps of both CTAs
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sc_full[i], 1);
      mbar_init(&sc_empty[i], 8);
    }
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();                                 // the other CTA's barriers and tensor memory are ready too
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  grid_dep_sync();          // codes and scales may come from the kernel directly ahead
  grid_dep_trigger();

  // 384 threads of 168 registers: four warps at 40 leave eight 232 each
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 8) {
      bool ok = true;
      int item = 0, s = 0;
      uint32_t par = 1;                             // of the stage's next `done` phase (the first pass waits for none)
      const uint32_t on = lane == 0 ? 1u : 0u, lead_on = rank == 0 ? on : 0u;
      const uint32_t full_s = smem_u32(&full[0]), lead_s = map_rank(full_s, 0);
      for (int t = pair; ok && t < n_tiles; t += n_pairs) {
        const int m0 = (t % token_tiles) * 256 + (int)rank * 128, n0 = (t / token_tiles) * BN + (int)rank * HC;
        for (int g = 0; g < a.G; ++g, ++item) {
          if ((a.hook & 2u) && item == 1) ok = false;   // test hook: the waits on the second stage run out
          if (ok && item >= S) ok = mbar_wait(smem_u32(&done[s]), par, &gave_up, a.polls, a.status);
          if (!ok) break;
          const uint32_t dst = ring_s + s * C::kStage;
          mbar_expect_tx(full_s + 8 * s, 2 * C::kStage, lead_on);
          tma_load_2d_pair(dst, &a.ma, g * kBlockK, m0, lead_s + 8 * s, on);
          tma_load_2d_pair(dst + 16384, &a.mw, g * kBlockK, n0, lead_s + 8 * s, on);
          if (++s == S) {
            s = 0;
            par ^= 1u;
          }
        }
      }
      // leave nothing behind: every stage handed back (its arrival crosses to the other CTA), or at least every copy landed
      for (int j = item < S ? 0 : item - S; ok && j < item; ++j)
        ok = mbar_wait(smem_u32(&done[j % S]), (j / S) & 1, &gave_up, a.polls, a.status);
      if (!ok && rank == 0)
        for (int j = item < S ? 0 : item - S; j < item; ++j)
          for (int n = 0; n < 200 && !mbar_look<true>(smem_u32(&full[j % S]), (j / S) & 1); ++n) {
          }
    } else if (warp == 9 || warp == 10) {
      // two warps issue, blocks in turn: every block has an accumulator of its own, so their order does not matter
      bool ok = rank == 0;
      const uint32_t on = lane == 0 ? 1u : 0u;
      const int my_tiles = pair < n_tiles ? (n_tiles - 1 - pair) / n_pairs + 1 : 0;
      const int64_t items = (int64_t)my_tiles * a.G;
      for (int64_t it = warp - 9; ok && it < items; it += 2) {
        const int item = (int)it, s = item % S, b = item % A;
        ok = mbar_wait(smem_u32(&full[s]), (item / S) & 1, &gave_up, a.polls, a.status);   // the accumulator comes last
        if (ok && item >= A) ok = mbar_wait(smem_u32(&acc_empty[b]), (item / A - 1) & 1, &gave_up, a.polls, a.status);
        if (!ok) break;
        tc_fence_after();
        const uint32_t x_s = ring_s + s * C::kStage;
        mma_block<true>(tmem + b * BN, swizzled_lo(x_s), swizzled_lo(x_s + 16384), kSwizzledHi, e4m3_idesc(256, BN), smem_u32(&done[s]), on);
      }
    } else if (warp == 11) {
      bool ok = true;
      int run = 0;
      for (int t = pair; ok && t < n_tiles; t += n_pairs) {
        const int64_t m0 = (int64_t)(t % token_tiles) * 256 + rank * 128;
        const int wb = (t / token_tiles) * BN / 128 + (lane >> 3);       // lanes 0-7, 8-15: the tile's weight blocks
        for (int g = 0; g < a.G; g += kScaleRun, ++run) {
          const float w = lane < 16 && (int64_t)wb * 128 < a.N && g + (lane & 7) < a.G ? a.sw[(int64_t)wb * a.G + g + (lane & 7)] : 0.f;
          if (run >= 2) ok = mbar_wait(smem_u32(&sc_empty[run & 1]), ((run >> 1) - 1) & 1, &gave_up, a.polls, a.status);
          if (!ok) break;
          if (lane < 16) w_scales[run & 1][lane >> 3][lane & 7] = w;
          const uint32_t w_least = __reduce_min_sync(0xffffffffu, 2 * __float_as_uint(w) - 1), w_most = __reduce_max_sync(0xffffffffu, 2 * __float_as_uint(w));
          float* dst = scales[run & 1][0];
          load_scales<128>(a.sa, m0, a.T, a.G, g, a.G, 0.f, lane, [&](int at, float v) { dst[at] = v; });
          __syncwarp();
          const bool any = w_most && products_leave<128>(dst, __uint_as_float((w_least >> 1) + 1), __uint_as_float(w_most >> 1), lane);
          if (lane == 0) extreme_run[run & 1] = any;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sc_full[run & 1]);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int row = (warp & 3) * 32 + lane, col = (warp >> 2) * HC;
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + col;
    const uint32_t box_s = ring_s + S * C::kStage + warp * 8192;
    const char* box = smem_raw + (box_s - smem_u32(smem_raw));
    // The loads run one step of 32 columns ahead of the multiply-adds, over the blocks' ends too: the last step of a
    // block is multiplied while the first of the next one is on its way.
    constexpr int Q = HC / 32;
    static_assert(Q % 2 == 0, "a block begins in the first buffer");
    bool ok = true, extreme = false;
    int s = 0, b = 0, run = 0, in_run = 0;
    uint32_t par = 0;                               // of the stage's next `done` phase
    float v[2][32];
    // waits for the next block's accumulator (b, s) and its scales, starts its first load
    auto begin = [&](bool new_run) {
      if (new_run) {
        ok = mbar_wait(smem_u32(&sc_full[run & 1]), (run >> 1) & 1, &gave_up, a.polls, a.status);
        extreme = extreme_run[run & 1] != 0;
      }
      if (ok) ok = mbar_wait(smem_u32(&done[s]), par, &gave_up, a.polls, a.status);
      if (!ok) return;
      tc_fence_after();
      tmem_ld32(lane_base + b * BN, v[0]);
    };
    if (pair < n_tiles) begin(true);
    for (int t = pair; ok && t < n_tiles; t += n_pairs) {
      uint64_t acc[HC / 2];                         // pairs of columns: a packed multiply-add does two
#pragma unroll
      for (int j = 0; j < HC / 2; ++j) acc[j] = 0;
      // The blocks of a run of scales: a loop of each kind.  (4096 x 14336 x 4096: 226 us without the rare kind, 231 so; with
      // the test for every block a tenth more, inside a block a third.)
      auto blocks = [&](auto kind, int first, int end) {
        constexpr bool kExtreme = decltype(kind)::value;
#pragma unroll 1
        for (int g = first; ok && g < end; ++g) {
          const float x = scales[run & 1][in_run][row], y = w_scales[run & 1][col / 128][in_run];
          const Factor fm = kExtreme ? split_factor(x, y) : Factor{x * y, 1.f};
          const uint64_t ff = pack2(fm.f, fm.f);
#pragma unroll
          for (int c = 0; c < Q; ++c) {
            tmem_wait32(v[c & 1]);
            if constexpr (kExtreme) {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[c & 1][j] *= fm.m;
            }
            if (c + 1 < Q) {
              tmem_ld32(lane_base + b * BN + (c + 1) * 32, v[(c + 1) & 1]);
            } else {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) {
                arrive_cluster(map_rank(smem_u32(&acc_empty[b]), 0));
                if (in_run == kScaleRun - 1 || g == a.G - 1) mbar_arrive(&sc_empty[run & 1]);
              }
              if (++in_run == kScaleRun || g == a.G - 1) {
                in_run = 0;
                ++run;
              }
              b = b + 1 == A ? 0 : b + 1;
              if (++s == S) {
                s = 0;
                par ^= 1u;
              }
              if (g + 1 < a.G || t + n_pairs < n_tiles) begin(in_run == 0);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[c * 16 + j] = fma2(pack2(v[c & 1][2 * j], v[c & 1][2 * j + 1]), ff, acc[c * 16 + j]);
          }
        }
      };
#pragma unroll 1
      for (int g = 0; ok && g < a.G; g += kScaleRun) {
        const int end = min(g + kScaleRun, a.G);
        if (extreme) blocks(std::true_type{}, g, end);
        else blocks(std::false_type{}, g, end);
      }
      // (after a wait that gave up the sums are not complete; what is stored is undefined then)
      store_tile<HC>(box_s, box, acc, a, (int64_t)(t % token_tiles) * 256 + rank * 128 + (warp & 3) * 32, (t / token_tiles) * BN + col, lane);
      __syncwarp();
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // the output is written, the boxes are read
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();                                 // nobody leaves while the other CTA may still arrive on its barriers
  tc_fence_after();
  __syncwarp();
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512));
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

// Map of the output: boxes of 32 rows x 128 bytes, swizzled.
static bool out_map(void* encode, void* base, int rows, int cols, int64_t stride, int type, CUtensorMap* m) {
  const int size = type_size(type);
  const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t pitch[1] = {(cuuint64_t)stride * size};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / size), 32}, step[2] = {1, 1};
  return reinterpret_cast<EncodeTiledFn>(encode)(m, size == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, base, dim, pitch,
                                                 box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                 CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Over how many CTAs of a cluster the blocks of a unit may be split.
constexpr int kSplits = 5;
constexpr int kSplit[kSplits] = {2, 3, 4, 5, 8};

static pw_status linear_setup(pw_ctx* ctx) {
  if (ctx->encode_tiled.load(std::memory_order_acquire)) return PW_OK;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  PW_CUDA_OK(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found));
  if (!fn || found != cudaDriverEntryPointSuccess) return PW_ERR_CUDA;
  PW_CUDA_OK((cudaFuncSetAttribute(linear_few_kernel<16, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<16, false>::kSmem)));
  PW_CUDA_OK((cudaFuncSetAttribute(linear_few_kernel<16, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<16, true>::kSmem)));
  PW_CUDA_OK((cudaFuncSetAttribute(linear_few_kernel<32, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<32, false>::kSmem)));
  PW_CUDA_OK((cudaFuncSetAttribute(linear_few_kernel<32, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<32, true>::kSmem)));
  PW_CUDA_OK((cudaFuncSetAttribute(linear_few_kernel<64, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<64, false>::kSmem)));
  PW_CUDA_OK((cudaFuncSetAttribute(linear_few_kernel<64, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<64, true>::kSmem)));
  PW_CUDA_OK(cudaFuncSetAttribute(linear_pair_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, PairCfg<128>::kSmem));
  PW_CUDA_OK(cudaFuncSetAttribute(linear_pair_kernel<256>, cudaFuncAttributeMaxDynamicSharedMemorySize, PairCfg<256>::kSmem));
  // how many clusters run at the same time, one CTA per SM: an SM left over in its group of SMs is of no use to a cluster
  // (16 of 8 CTAs did not fit on 148 SMs: 64 x 2048 x 2048 took 10.8 us, two rounds)
  for (int i = 0; i < kSplits; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kSplit[i];
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.gridDim = dim3(kSplit[i]);
    cfg.blockDim = dim3(FewCfg<64, true>::kThreads);
    cfg.dynamicSmemBytes = FewCfg<64, true>::kSmem;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    PW_CUDA_OK((cudaOccupancyMaxActiveClusters(&clusters, linear_few_kernel<64, true>, &cfg)));
    ctx->max_clusters[i].store(clusters, std::memory_order_relaxed);
  }
  ctx->encode_tiled.store(fn, std::memory_order_release);
  return PW_OK;
}

template <class... Args>
static cudaError_t launch_cluster(void (*kernel)(LinearArgs, Args...), unsigned ctas, unsigned cluster, int threads, size_t smem, cudaStream_t s,
                                  const LinearArgs& a, Args... args) {
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
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, args...);
}

// How a product is cut: the kernel (few: nt tokens per tile, or pair: bn weight rows per tile), the units of work and,
// for the few kernel, over how many CTAs of a cluster the blocks of a unit are split.
struct LinearPlan {
  int nt, bn, split;
  int64_t token_tiles, units;
  double us;                                       // estimate
};
static int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

static LinearPlan plan_few(int T, int N, int G, int nt, int sms, const int* max_clusters) {
  LinearPlan p{nt, 0, 1, tiles_of(T, nt), 0, 0.};
  p.units = p.token_tiles * tiles_of(N, 128);
  // few units: their blocks are split over a cluster, while all clusters run at the same time and two blocks are left for
  // every CTA
  for (int i = 0; i < kSplits; ++i)
    if (p.units <= max_clusters[i] && G >= kSplit[i] * 2) p.split = kSplit[i];
  const int64_t rounds = p.split > 1 ? 1 : tiles_of(p.units, sms), blocks = p.split > 1 ? tiles_of(G, p.split) : rounds * G;
  p.us = 1.5 * (rounds - 1) + (nt == 16 ? 3.3 + 0.26 * blocks : nt == 32 ? 3.8 + 0.30 * blocks : 4.4 + 0.32 * blocks);
  return p;
}
static LinearPlan plan_pair(int T, int N, int G, int bn, int sms) {
  LinearPlan p{0, bn, 1, tiles_of(T, 256), 0, 0.};
  p.units = p.token_tiles * tiles_of(N, bn);
  p.us = 4.6 + (bn == 128 ? 0.32 : 0.52) * tiles_of(p.units, sms / 2) * G;
  return p;
}
// The plan that finishes soonest by a model that is linear in the blocks of 128 columns a CTA (pair) goes through one
// after the other and in the units it does (301 x 64 x 2056: 16 tokens to a tile 4.7 us, 64 5.6; 3711 x 187 x 119: 16
// tokens, four units one after the other, 8.8, 64 tokens 4.9).  The times per block are measured (us, contraction 4096,
// tokens x weight rows, few 64 / pair 128 / pair 256; the pair kernel takes 2 to 5 % more since):  64 x 4096  7.6 / 14.1 /
// 18.3,  128 x 4096  9.6 / 14.4 / 18.9,  64 x 14336  14.6 / 26.2 / 20.9,  128 x 14336  27 / 27.6 / 22.7,
// 256 x 4096  11.7 / 14.7 / 19.1,  512 x 4096  26 / 16.4 / 20.0,  512 x 14336  80 / 48 / 38.
static LinearPlan plan_linear(int T, int N, int G, int sms, const int* max_clusters) {
  LinearPlan best = plan_few(T, N, G, 16, sms, max_clusters);
  for (int nt = 32; nt <= 64 && T > nt / 2; nt *= 2) {
    const LinearPlan p = plan_few(T, N, G, nt, sms, max_clusters);
    if (p.us < best.us) best = p;
  }
  for (int bn = 128; bn <= 256; bn *= 2) {
    const LinearPlan p = plan_pair(T, N, G, bn, sms);
    if (p.us < best.us) best = p;
  }
  return best;
}

template <int NT>
static cudaError_t launch_few(const LinearPlan& p, const LinearArgs& a, int sms, cudaStream_t s) {
  const int64_t ctas = p.split > 1 || p.units < sms ? p.units * p.split : sms;
  return p.split > 1 ? launch_cluster(linear_few_kernel<NT, true>, (unsigned)ctas, p.split, FewCfg<NT, true>::kThreads, FewCfg<NT, true>::kSmem, s, a,
                                      (int)p.token_tiles, (int)p.units, p.split)
                     : launch_cluster(linear_few_kernel<NT, false>, (unsigned)ctas, 1, FewCfg<NT, false>::kThreads, FewCfg<NT, false>::kSmem, s, a,
                                      (int)p.token_tiles, (int)p.units, 1);
}
template <int BN>
static cudaError_t launch_pair(const LinearPlan& p, const LinearArgs& a, int sms, cudaStream_t s) {
  const int64_t pairs = p.units < sms / 2 ? p.units : sms / 2;
  return launch_cluster(linear_pair_kernel<BN>, (unsigned)pairs * 2, 2, kPairThreads, PairCfg<BN>::kSmem, s, a, (int)p.token_tiles, (int)p.units);
}

}  // namespace pw

using namespace pw;

extern "C" pw_status pw_scaled_linear(pw_ctx* ctx, int T, int N, int K, const void* a_codes, int64_t a_stride,
                                      const float* a_scales, const void* w_codes, int64_t w_stride, const float* w_scales,
                                      void* out, int out_type, int64_t out_stride, pw_stream stream) {
  if (!ctx || T < 0 || N < 1 || K < 1 || !type_ok(out_type)) return PW_ERR_INVALID_ARG;
  if (T > 1 << 30 || N > 1 << 30 || K > 1 << 30) return PW_ERR_SHAPE;
  if (T == 0) return PW_OK;
  if (!a_codes || !a_scales || !w_codes || !w_scales || !out) return PW_ERR_INVALID_ARG;
  if ((T > 1 && (a_stride < K || out_stride < N)) || (N > 1 && w_stride < K)) return PW_ERR_SHAPE;
  const void* ptrs[5] = {a_codes, a_scales, w_codes, w_scales, out};
  for (const void* p : ptrs)
    if (!is_aligned(p, 16)) return PW_ERR_ALIGN;
  if ((T > 1 && a_stride % 16) || (N > 1 && w_stride % 16)) return PW_ERR_ALIGN;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  const pw_status st = linear_setup(ctx);
  if (st != PW_OK) return st;
  LinearArgs a{};
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
  void* const encode = ctx->encode_tiled.load(std::memory_order_acquire);
  int max_clusters[kSplits];
  for (int i = 0; i < kSplits; ++i) max_clusters[i] = ctx->max_clusters[i].load(std::memory_order_relaxed);
  const LinearPlan p = plan_linear(T, N, a.G, ctx->num_sms, max_clusters);
  if (p.units > 0x7fffffff) return PW_ERR_SHAPE;
  // a single row's stride is never used: give the map one that it accepts
  const int64_t pitch = ((int64_t)K + 15) / 16 * 16, out_pitch = T > 1 ? out_stride : N;
  if (!codes_map(encode, a_codes, T, K, T > 1 ? a_stride : pitch, p.bn ? 128 : p.nt, &a.ma) ||
      !codes_map(encode, w_codes, N, K, N > 1 ? w_stride : pitch, p.bn ? p.bn / 2 : 128, &a.mw))
    return PW_ERR_CUDA;
  // the copies of output boxes are cut at a row's end in units of 16 bytes only
  const int size = type_size(out_type);
  if (p.bn) a.tma_out = out_pitch * size % 16 == 0 && (int64_t)N * size % 16 == 0 && out_map(encode, out, T, N, out_pitch, out_type, &a.mo);
  PW_CUDA_OK(p.bn == 256   ? launch_pair<256>(p, a, ctx->num_sms, stream)
             : p.bn == 128 ? launch_pair<128>(p, a, ctx->num_sms, stream)
             : p.nt == 16  ? launch_few<16>(p, a, ctx->num_sms, stream)
             : p.nt == 32  ? launch_few<32>(p, a, ctx->num_sms, stream)
                           : launch_few<64>(p, a, ctx->num_sms, stream));
  ctx->launches++;
  return PW_OK;
}
