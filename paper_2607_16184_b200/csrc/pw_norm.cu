// Residual addition + root-mean-square norm (with the scaled 8-bit copy of its result), and the quantizer of the
// scaled 8-bit format.
//
//   s = x + r        r' = round(s)        y = s * w / sqrt(mean(s^2) + eps)
//   per block: top = max |y|, scale = top / 448, code = e4m3(y * (1 / scale))
//
// Both read every input element once and write every output element once; nothing else leaves the registers, so
// HBM bounds them at large sizes and the launch and one round trip to memory at small ones.  Measured in a graph of calls
// one behind the other: norm of 4096 x 4096 fp32 with residual, fp16 output and codes 29.2 us, quantizer of 14336 x 4096
// fp16 27.7 us (both 97 % of the copy bandwidth; launched call by call 31.0 and 29.6, 91 %); one row of 4096 2.0 us, where
// the emptiest launch takes 1.9.
//
// A code is rounded from y times the reciprocal of its scale, two fp32 roundings instead of one division's: 1.7 us less
// for the quantizer's case above.  A value that lies within them of the middle between two codes may get the other one.
#include "pw_scaled.cuh"

namespace pw {

struct NormArgs {
  const void* x;
  const void* r;
  const void* w;
  void* r_out;
  void* y;
  uint8_t* q;
  float* q_scales;
  int64_t x_stride, r_stride, r_out_stride, y_stride, q_stride;
  int H, w_type, y_type;
  float eps;
};

__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// One CTA per row; the row stays in registers between the sum and the output.  Elements a thread holds:
//   VEC   eight consecutive ones (16- and 32-byte accesses), half a warp = one group of 128;
//   else  every 32nd of 256 consecutive ones of its warp, so that single-element accesses are contiguous over the
//         lanes whatever the row's alignment is; entries 0..3 and 4..7 of a thread belong to one group each.
// The loads of x, r and (for short rows) w are all issued before the first use; a thread of a long row has no registers
// to keep w in across the sum and reads it afterwards.  TR = void: no residual.
template <class TX, class TR, bool VEC, int VPT>
__global__ void __launch_bounds__(1024) add_rmsnorm_kernel(const NormArgs a) {
  grid_dep_sync();      // the row may come from the kernel directly ahead
  grid_dep_trigger();
  constexpr bool kRes = !std::is_void<TR>::value;
  using R = typename std::conditional<kRes, TR, float>::type;
  __shared__ float part[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
  const int64_t row = blockIdx.x;
  const TX* x = static_cast<const TX*>(a.x) + row * a.x_stride;
  const R* r = static_cast<const R*>(a.r) + (kRes ? row * a.r_stride : 0);
  const int H = a.H;
  float z[VPT][8];
  auto at = [&](int v, int j) { return VEC ? (v * (int)blockDim.x + tid) * 8 + j : ((v * n_warps + warp) * 8 + j) * 32 + lane; };
  auto left = [&](int v, int j) { return H - at(v, 0) > j * 32; };   // !VEC: whether the row has entry j
  // the weights (the same row for every CTA: an L2 hit)
  constexpr bool kEarly = VPT <= 2;
  auto weights = [&](int v, float* w) {
    if constexpr (VEC) {
      if (at(v, 0) >= H) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 0.f;
      } else if (a.w_type == PW_F32) {
        Raw8<float> t;
        t.load(static_cast<const float*>(a.w) + at(v, 0));
        t.get(w);
      } else if (a.w_type == PW_F16) {
        Raw8<__half> t;
        t.load(static_cast<const __half*>(a.w) + at(v, 0));
        t.get(w);
      } else {
        Raw8<__nv_bfloat16> t;
        t.load(static_cast<const __nv_bfloat16*>(a.w) + at(v, 0));
        t.get(w);
      }
    } else {
      auto every = [&](auto* p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = left(v, j) ? to_f32(p[j * 32]) : 0.f;
      };
      if (a.w_type == PW_F32) every(static_cast<const float*>(a.w) + at(v, 0));
      else if (a.w_type == PW_F16) every(static_cast<const __half*>(a.w) + at(v, 0));
      else every(static_cast<const __nv_bfloat16*>(a.w) + at(v, 0));
    }
  };
  float early[kEarly ? VPT : 1][8];
  if constexpr (VEC) {
    Raw8<TX> rx[VPT];
    Raw8<R> rr[VPT];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      rx[v].zero();
      if (at(v, 0) < H) rx[v].load(x + at(v, 0));
    }
    if constexpr (kRes) {
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        rr[v].zero();
        if (at(v, 0) < H) rr[v].load(r + at(v, 0));
      }
    }
    if constexpr (kEarly) {
#pragma unroll
      for (int v = 0; v < VPT; ++v) weights(v, early[v]);
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      rx[v].get(z[v]);
      if constexpr (kRes) {
        float b[8];
        rr[v].get(b);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[v][j] = __fadd_rn(z[v][j], b[j]);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) z[v][j] = left(v, j) ? to_f32((x + at(v, 0))[j * 32]) : 0.f;
      if constexpr (kRes) {
        float b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = left(v, j) ? to_f32((r + at(v, 0))[j * 32]) : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) z[v][j] = __fadd_rn(z[v][j], b[j]);
      }
    }
  }
  // sum of squares in 32 bits, in a fixed order: thread, warp, warps
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < VPT; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(z[v][j], z[v][j], ss);
  ss = warp_add(ss);
  if (lane == 0) part[warp] = ss;
  if (a.r_out) {
    const int type = std::is_same<R, float>::value ? PW_F32 : std::is_same<R, __half>::value ? PW_F16 : PW_BF16;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      if constexpr (VEC) {
        if (at(v, 0) < H) store8(a.r_out, row * a.r_out_stride + at(v, 0), type, z[v]);
      } else {
        R* out = static_cast<R*>(a.r_out) + row * a.r_out_stride + at(v, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (left(v, j)) out[j * 32] = from_f32<R>(z[v][j]);
      }
    }
  }
  __syncthreads();
  ss = warp_add(lane < n_warps ? part[lane] : 0.f);
  const float inv = __frcp_rn(__fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)H), a.eps)));
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    float w[8];
    if constexpr (VEC && kEarly) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = early[v][j];
    } else {
      weights(v, w);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) z[v][j] = __fmul_rn(__fmul_rn(z[v][j], inv), w[j]);
  }
  if (a.y) {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      if constexpr (VEC) {
        if (at(v, 0) < H) store8(a.y, row * a.y_stride + at(v, 0), a.y_type, z[v]);
      } else {
        auto every = [&](auto* p) {
          using Y = std::remove_pointer_t<decltype(p)>;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (left(v, j)) p[j * 32] = from_f32<Y>(z[v][j]);
        };
        if (a.y_type == PW_F32) every(static_cast<float*>(a.y) + row * a.y_stride + at(v, 0));
        else if (a.y_type == PW_F16) every(static_cast<__half*>(a.y) + row * a.y_stride + at(v, 0));
        else every(static_cast<__nv_bfloat16*>(a.y) + row * a.y_stride + at(v, 0));
      }
    }
  }
  if (!a.q) return;
  // codes of the unrounded values
  const int G = (H + kGroup - 1) / kGroup;
  uint8_t* q = a.q + row * a.q_stride;
  float* qs = a.q_scales + row * G;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if constexpr (VEC) {
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = abs_max(top, z[v][j]);
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float scale = block_scale(top), rinv = __frcp_rn(scale);
      const int c = at(v, 0);
      if (c >= H) continue;
      if ((lane & 15) == 0) qs[c / kGroup] = scale;
      uint2 o;
      o.x = pack_e4m3(z[v][0] * rinv, z[v][1] * rinv) | (pack_e4m3(z[v][2] * rinv, z[v][3] * rinv) << 16);
      o.y = pack_e4m3(z[v][4] * rinv, z[v][5] * rinv) | (pack_e4m3(z[v][6] * rinv, z[v][7] * rinv) << 16);
      *reinterpret_cast<uint2*>(q + c) = o;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = abs_max(top, z[v][4 * h + j]);
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float scale = block_scale(top), rinv = __frcp_rn(scale);
        const int c = at(v, 4 * h);
        if (lane == 0 && c < H) qs[c / kGroup] = scale;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (left(v, 4 * h + j)) (q + at(v, 0))[(4 * h + j) * 32] = (uint8_t)pack_e4m3(z[v][4 * h + j] * rinv, 0.f);
      }
    }
  }
}

template <class TX, class TR>
static pw_status launch_norm(const NormArgs& a, bool vec, int T, int num_sms, cudaStream_t s) {
  // Threads.  With a row per SM at most, as many as there are vectors: more of them hide more latency (14 rows x 9728 fp32
  // with codes 5.0 -> 3.7 us).  With more rows one vector each up to 4096 columns, then CTAs of up to 512 threads, several
  // on an SM, before larger ones: rows of 12672 bf16 take 36 us as 416 threads of four vectors and 45 us as 800 of two
  // (2048 rows; HBM 32).  Above 16384 columns only 1024 threads keep a thread's share in its registers (1024 rows x 24576:
  // 40 us, 53 us as 512 threads of up to eight; HBM 31).  Single-element accesses take up to 1024 threads from 8192 columns
  // on (478 rows x 12671, with codes: 23 us, 33 us as 512): they are bound by their instructions, 64 bytes of a row each.
  // Above 16384 columns those threads hold four vectors in the 64 registers that 1024 of them leave, and spill 228 to 244
  // bytes each: part of the 71 us of 1024 rows x 24575 (24576, in vectors: 40).
  const int n8 = (a.H + 7) / 8;
  const int vpt = n8 <= (T <= num_sms ? 1024 : 512) ? 1 : n8 <= (T > num_sms && vec ? 1024 : 2048) ? 2 : 4;
  const int threads = ((n8 + vpt - 1) / vpt + 31) / 32 * 32;
  void (*k)(NormArgs);
  if (vec) k = vpt == 1 ? add_rmsnorm_kernel<TX, TR, true, 1> : vpt == 2 ? add_rmsnorm_kernel<TX, TR, true, 2> : add_rmsnorm_kernel<TX, TR, true, 4>;
  else k = vpt == 1 ? add_rmsnorm_kernel<TX, TR, false, 1> : vpt == 2 ? add_rmsnorm_kernel<TX, TR, false, 2> : add_rmsnorm_kernel<TX, TR, false, 4>;
  PW_CUDA_OK(launch_dependent(k, dim3(T), dim3(threads), 0, s, a));
  return PW_OK;
}
template <class TX>
static pw_status launch_norm_r(const NormArgs& a, int r_type, bool vec, int T, int num_sms, cudaStream_t s) {
  if (!a.r) return launch_norm<TX, void>(a, vec, T, num_sms, s);
  if (r_type == PW_F32) return launch_norm<TX, float>(a, vec, T, num_sms, s);
  if (r_type == PW_F16) return launch_norm<TX, __half>(a, vec, T, num_sms, s);
  return launch_norm<TX, __nv_bfloat16>(a, vec, T, num_sms, s);
}

// ---- quantizer ---------------------------------------------------------------------------------

// Four codes at column c of a row of codes (it starts on a 16-byte boundary; nothing is written behind its end).
__device__ __forceinline__ void store_four(uint8_t* q, int c, int cols, const float* z, float rinv) {
  const uint32_t o = pack_e4m3(z[0] * rinv, z[1] * rinv) | (pack_e4m3(z[2] * rinv, z[3] * rinv) << 16);
  if (c + 4 <= cols) {
    *reinterpret_cast<uint32_t*>(q + c) = o;
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (c + k < cols) q[c + k] = (uint8_t)(o >> (8 * k));
  }
}

struct QuantArgs {
  const void* x;
  uint8_t* q;
  float* scales;
  int64_t x_stride, q_stride;
  int rows, cols;
};

// Blocks of one row: a warp takes 1024 columns of a row (U pieces of two groups), all loaded before the first is used.
template <class TX, bool VEC>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantArgs a, uint32_t units, uint32_t per_row) {
  grid_dep_sync();
  grid_dep_trigger();
  constexpr int U = 4;
  const int lane = threadIdx.x & 31;
  const int G = (a.cols + kGroup - 1) / kGroup;
  for (uint32_t unit = blockIdx.x * 8 + (threadIdx.x >> 5); unit < units; unit += gridDim.x * 8) {
    const uint32_t row = unit / per_row;
    const int c0 = (int)(unit - row * per_row) * 256 * U;
    const TX* x = static_cast<const TX*>(a.x) + row * a.x_stride;
    uint8_t* q = a.q + row * a.q_stride;
    float* qs = a.scales + (int64_t)row * G;
    if constexpr (VEC) {
      Raw8<TX> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * 256 + lane * 8;
        raw[u].zero();
        if (c < a.cols) raw[u].load(x + c);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float z[8];
        raw[u].get(z);
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = abs_max(top, z[j]);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float scale = block_scale(top), rinv = __frcp_rn(scale);
        const int c = c0 + u * 256 + lane * 8;
        if (c >= a.cols) continue;
        if ((lane & 15) == 0) qs[c / kGroup] = scale;
        uint2 o;
        o.x = pack_e4m3(z[0] * rinv, z[1] * rinv) | (pack_e4m3(z[2] * rinv, z[3] * rinv) << 16);
        o.y = pack_e4m3(z[4] * rinv, z[5] * rinv) | (pack_e4m3(z[6] * rinv, z[7] * rinv) << 16);
        *reinterpret_cast<uint2*>(q + c) = o;
      }
    } else {
      constexpr int N = U * 2;                     // groups
      const int left = a.cols - c0;
      x += c0;
      TX raw[N][4];
#pragma unroll
      for (int h = 0; h < N; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[h][j] = h * kGroup + lane * 4 + j < left ? x[h * kGroup + lane * 4 + j] : (TX)0.f;
#pragma unroll
      for (int h = 0; h < N; ++h) {
        float z[4], top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = to_f32(raw[h][j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) top = abs_max(top, z[j]);
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float scale = block_scale(top), rinv = __frcp_rn(scale);
        const int c = c0 + h * kGroup;
        if (lane == 0 && c < a.cols) qs[c / kGroup] = scale;
        store_four(q, c + lane * 4, a.cols, z, rinv);
      }
    }
  }
}

// Blocks of 128 x 128: a CTA per block, 64 elements of it per thread, all loaded before the maximum is taken.
//   VEC   half a warp per row, eight columns per lane, eight passes of 16 rows;
//   else  a warp per row, two passes over the rows, the second from L1 or L2 (14336 x 4095 bf16: 61 us; all 64 elements
//         of a thread kept in registers, two CTAs on an SM, 80 us).
template <class TX, bool VEC>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const QuantArgs a) {
  grid_dep_sync();
  grid_dep_trigger();
  __shared__ float part[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = (a.cols + kGroup - 1) / kGroup;
  const int64_t rb = blockIdx.x / G;
  const int g = (int)(blockIdx.x - rb * G);
  const int64_t r0 = rb * kTileRows;
  const int c0 = g * kGroup;
  const TX* x = static_cast<const TX*>(a.x);
  // (the elements are kept as they were loaded and converted twice: fewer registers, twice as many CTAs on an SM)
  float top = 0.f;
  auto scale_of_block = [&](float m) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) part[warp] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, part[i]);
    const float scale = block_scale(m);
    if (tid == 0) a.scales[rb * G + g] = scale;
    return __frcp_rn(scale);
  };
  if constexpr (VEC) {
    Raw8<TX> raw[8];
    const int c = c0 + (lane & 15) * 8;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t r = r0 + p * 16 + (tid >> 4);
      raw[p].zero();
      if (r < a.rows && c < a.cols) raw[p].load(x + r * a.x_stride + c);
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      float z[8];
      raw[p].get(z);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = abs_max(top, z[j]);
    }
    const float rinv = scale_of_block(top);
#pragma unroll
    for (int p = 0; p < 8; ++p) raw[p].forget();
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t r = r0 + p * 16 + (tid >> 4);
      if (r >= a.rows || c >= a.cols) continue;
      float z[8];
      raw[p].get(z);
      uint2 o;
      o.x = pack_e4m3(z[0] * rinv, z[1] * rinv) | (pack_e4m3(z[2] * rinv, z[3] * rinv) << 16);
      o.y = pack_e4m3(z[4] * rinv, z[5] * rinv) | (pack_e4m3(z[6] * rinv, z[7] * rinv) << 16);
      *reinterpret_cast<uint2*>(a.q + r * a.q_stride + c) = o;
    }
  } else {
    const int n = (int)(a.rows - r0 < kTileRows ? a.rows - r0 : kTileRows);
    const TX* block = x + r0 * a.x_stride + c0;
    const int cols = a.cols - c0;
#pragma unroll 4
    for (int r = warp; r < n; r += 8) {
      const TX* row = block + r * a.x_stride;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = abs_max(top, j * 32 + lane < cols ? to_f32(row[j * 32 + lane]) : 0.f);
    }
    const float rinv = scale_of_block(top);
#pragma unroll 4
    for (int r = warp; r < n; r += 8) {
      const TX* row = block + r * a.x_stride;
      float z[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] = lane * 4 + j < cols ? to_f32(row[lane * 4 + j]) : 0.f;
      store_four(a.q + (r0 + r) * a.q_stride + c0, lane * 4, cols, z, rinv);
    }
  }
}

template <class TX>
static pw_status launch_quant(const QuantArgs& a, int block_rows, bool vec, int num_sms, cudaStream_t s) {
  const int64_t G = (a.cols + kGroup - 1) / kGroup;
  if (block_rows == 1) {
    const uint32_t per_row = (uint32_t)((G + 7) / 8);
    const int64_t units = (int64_t)a.rows * per_row, ctas = (units + 7) / 8, cap = (int64_t)num_sms * 64;
    if (units > 0x7fffffff) return PW_ERR_SHAPE;
    PW_CUDA_OK(launch_dependent(vec ? quantize_rows_kernel<TX, true> : quantize_rows_kernel<TX, false>,
                                dim3((unsigned)(ctas < cap ? ctas : cap)), dim3(256), 0, s, a, (uint32_t)units, per_row));
  } else {
    const int64_t ctas = ((int64_t)a.rows + kTileRows - 1) / kTileRows * G;
    if (ctas > 0x7fffffff) return PW_ERR_SHAPE;
    PW_CUDA_OK(launch_dependent(vec ? quantize_blocks_kernel<TX, true> : quantize_blocks_kernel<TX, false>,
                                dim3((unsigned)ctas), dim3(256), 0, s, a));
  }
  return PW_OK;
}

constexpr int kMaxNormWidth = 32768;            // 1024 threads x four vectors of eight

}  // namespace pw

using namespace pw;

extern "C" pw_status pw_add_rmsnorm(pw_ctx* ctx, int T, int H, const void* x, int x_type, int64_t x_stride,
                                    const void* residual, int residual_type, int64_t residual_stride, const void* weight,
                                    int weight_type, float eps, void* residual_out, int64_t residual_out_stride, void* y,
                                    int y_type, int64_t y_stride, void* q, int64_t q_stride, float* q_scales,
                                    pw_stream stream) {
  if (!ctx || T < 0 || H < 1 || !(eps >= 0.f)) return PW_ERR_INVALID_ARG;
  if (H > kMaxNormWidth) return PW_ERR_SHAPE;
  if (!type_ok(x_type) || !type_ok(weight_type) || (residual && !type_ok(residual_type)) || (y && !type_ok(y_type)))
    return PW_ERR_INVALID_ARG;
  if (T == 0) return PW_OK;
  if (!x || !weight || (residual_out && !residual) || (!y && !q) || (!q != !q_scales)) return PW_ERR_INVALID_ARG;
  if (T > 1 && ((x_stride < H) || (residual && residual_stride < H) || (residual_out && residual_out_stride < H) ||
                (y && y_stride < H) || (q && q_stride < H)))
    return PW_ERR_SHAPE;
  const void* ptrs[7] = {x, residual, weight, residual_out, y, q, q_scales};
  for (const void* p : ptrs)
    if (!is_aligned(p, 16)) return PW_ERR_ALIGN;
  if (q && T > 1 && q_stride % 16) return PW_ERR_ALIGN;       // (a single row's stride is never used)
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  NormArgs a{};
  a.x = x;
  a.r = residual;
  a.w = weight;
  a.r_out = residual_out;
  a.y = y;
  a.q = static_cast<uint8_t*>(q);
  a.q_scales = q_scales;
  a.x_stride = x_stride;
  a.r_stride = residual_stride;
  a.r_out_stride = residual_out_stride;
  a.y_stride = y_stride;
  a.q_stride = q_stride;
  a.H = H;
  a.w_type = weight_type;
  a.y_type = y_type;
  a.eps = eps;
  // 16-byte accesses where every row of every tensor starts on a 16-byte boundary and holds whole vectors
  auto rows16 = [&](const void* p, int type, int64_t stride) { return !p || (stride * type_size(type)) % 16 == 0; };
  const bool vec = H % 8 == 0 && rows16(x, x_type, x_stride) && rows16(residual, residual_type, residual_stride) &&
                   rows16(residual_out, residual_type, residual_out_stride) && rows16(y, y_type, y_stride);
  const pw_status st = x_type == PW_F32   ? launch_norm_r<float>(a, residual_type, vec, T, ctx->num_sms, stream)
                       : x_type == PW_F16 ? launch_norm_r<__half>(a, residual_type, vec, T, ctx->num_sms, stream)
                                          : launch_norm_r<__nv_bfloat16>(a, residual_type, vec, T, ctx->num_sms, stream);
  if (st == PW_OK) ctx->launches++;
  return st;
}

extern "C" pw_status pw_quantize_scaled(pw_ctx* ctx, const void* x, int x_type, int rows, int cols, int64_t x_stride,
                                        int block_rows, void* q, int64_t q_stride, float* scales, pw_stream stream) {
  if (!ctx || rows < 0 || cols < 1 || !type_ok(x_type) || (block_rows != 1 && block_rows != kTileRows))
    return PW_ERR_INVALID_ARG;
  if (cols > 1 << 30) return PW_ERR_SHAPE;
  if (rows == 0) return PW_OK;
  if (!x || !q || !scales) return PW_ERR_INVALID_ARG;
  if (rows > 1 && (x_stride < cols || q_stride < cols)) return PW_ERR_SHAPE;
  if (!is_aligned(x, 16) || !is_aligned(q, 16) || !is_aligned(scales, 16) || (rows > 1 && q_stride % 16)) return PW_ERR_ALIGN;
  const pw_status ds = check_device(ctx);
  if (ds != PW_OK) return ds;
  QuantArgs a{x, static_cast<uint8_t*>(q), scales, x_stride, q_stride, rows, cols};
  const bool vec = cols % 8 == 0 && (x_stride * type_size(x_type)) % 16 == 0;
  const pw_status st = x_type == PW_F32   ? launch_quant<float>(a, block_rows, vec, ctx->num_sms, stream)
                       : x_type == PW_F16 ? launch_quant<__half>(a, block_rows, vec, ctx->num_sms, stream)
                                          : launch_quant<__nv_bfloat16>(a, block_rows, vec, ctx->num_sms, stream);
  if (st == PW_OK) ctx->launches++;
  return st;
}
