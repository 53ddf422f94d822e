// Rows of weight pages against the operand rows of up to eight tokens: the inner loop of the calls for few tokens.
//
// A unit of work is 32 rows of a block.  Every warp streams a part of the block's columns ("steps") through a ring of its
// own in shared memory with 16-byte asynchronous copies and multiplies it on the spot; nothing is shared between warps
// before their sums meet at the end of a unit.  With so few tokens a weight is used at most eight times, so what counts is
// that the copies never pause: a warp waits for the step it asked for STAGES steps ago, multiplies it, asks for the next and
// goes on, without a barrier.
//
// The product runs on mma.sync m16n8k16 (two of them, 16 weight rows x 8 tokens each), not on tcgen05: a decoded weight goes
// from a register straight into the instruction, where the larger one wants 128 rows and its operand written to tensor
// memory first (the layer's kernels for batches, which do that, read a 4-bit page at 53 % of the copy bandwidth).
//
// A group of 128 columns of a row contributes
//     sum x * (code * scale + zero) = scale * sum x * code + zero * sum x
// and the codes themselves are the operands: a field of a code word is cut out with one logic instruction and is, in
// place, an fp16 number -- a subnormal, field << p reads field * 2^(p - 24) for every p with the field below bit 10.  The
// tensor core multiplies subnormals exactly, but lines up what it adds by their nominal exponents: leading zeros of a
// subnormal are bits that the sum does not have (a field at bits 0 .. 3: results off by 1.5e-6 of their norm, at bits 4 .. 7
// by 1e-7).  So narrow fields are moved up, by a multiplication, which is not the pipe that the logic instructions keep busy.
// The power of two goes into the scale, which is applied with the zero-point once per group, in fp32.  A pair of weights
// costs two instructions, where turning it into fp16(code * scale + zero) costs three; weights are not rounded to fp16 on
// this path.  A 4-bit step of a warp is about 265 instructions (112 to cut the codes out, 16 matrix instructions, 32 for
// scales and zero-points, 17 copies and loads), half of them for the pipe that starts one every other cycle: an SM then
// does a 2 KB step of each of its 16 warps in 1530 cycles, 22 bytes a cycle, where its share of the HBM rate is 24; steps
// of 8 and 16 bits keep up with that rate.
//
// Steps: 32 columns of a 16-bit block, 64 of an 8-bit one, a group of 128 otherwise, so that a step is 1 to 2 KB of
// codes.  Lane (g, t) = (lane / 4, lane % 4) multiplies part t of the step's columns, rows 4g .. 4g + 3 (as rows g and
// g + 8 of the two products), so that the scales of its rows are one 8-byte load.  The copies are cut the other way, a
// row's 16 bytes per lane: an instruction then takes 512 bytes in one piece, where one that follows the lanes of the
// product takes four pieces 2 KB apart (streaming alone, 71 MB out of the L2 cache: 7.6 us against 18.9).  Rows are
// exchanged inside a unit so that the loads of the product meet 32 banks (write_at).
//
// Operand rows are kept in pieces of 16 bytes.  A group's 128 columns are eight stretches of 16, as pairs W0 .. W7; piece
// 2s + h of stretch s holds W(2h), W(2h + 4), W(2h + 1), W(2h + 5): pairs next to one another are the two halves of an
// MMA's operand for every format (a field and the one at the same place eight columns on), so they lie in neighbouring
// registers.  Piece e of row c is the (e ^ (e >> 2) ^ 4 (c mod 2))-th of its 256 bytes: the four lanes of a row take
// pieces 4t + i, 2t + i or t (4-bit, 8-bit, 16-bit steps), two rows at a time, and meet 32 banks in all three.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "pw_layout.cuh"
#include "pw_ptx.cuh"

namespace pw {

enum : int { kFmt16 = 0, kFmt8, kFmt4, kFmt3, kFmt2, kFmtP4, kFmtP3, kFmtP2 };
// -1: not a format
__host__ __device__ inline int stream_format(int bits, bool planes) {
  if (planes) return bits == 4 ? kFmtP4 : bits == 3 ? kFmtP3 : bits == 2 ? kFmtP2 : -1;
  return bits == 16 ? kFmt16 : bits == 8 ? kFmt8 : bits == 4 ? kFmt4 : bits == 3 ? kFmt3 : bits == 2 ? kFmt2 : -1;
}
// log2 of the steps of a group
__host__ __device__ constexpr int step_shift(int fmt) { return fmt == kFmt16 ? 2 : fmt == kFmt8 ? 1 : 0; }
// bytes from one tile (of the TOP buffer, for planes) to the next, and of the scales inside it
__host__ __device__ constexpr uint32_t stream_tile_bytes(int fmt) {
  return fmt >= kFmtP4 ? (uint32_t)kPlaneTopTile : fmt == kFmt16 ? 32768u : fmt == kFmt8 ? 16896u : fmt == kFmt4 ? 8704u : fmt == kFmt3 ? 6656u : 4608u;
}
__host__ __device__ constexpr uint32_t stream_scale_offset(int fmt) {
  return fmt >= kFmtP4 ? (uint32_t)kPlaneTopCodes + 512u * (uint32_t)(kFmtP2 - fmt) : stream_tile_bytes(fmt) - 512u;
}

// the same for a format that is known at run time only: one load instead of a chain of selections
__constant__ uint32_t kTileBytes[8] = {32768, 16896, 8704, 6656, 4608, 5632, 5632, 5632};
__constant__ uint32_t kScaleOffset[8] = {32256, 16384, 8192, 6144, 4096, 5120, 4608, 4096};
constexpr int kSmemLimit = 232448;                // 227 KB
constexpr int kStreamWarps = 16;
constexpr int kStreamThreads = kStreamWarps * 32;
constexpr int kUnitRows = 32;
constexpr int kUnitCols = 8;                      // tokens of a unit
constexpr int kStepCodes = 2048;                  // bytes of a slot: codes, scales and zero-points
constexpr int kStepMeta = 128;
constexpr int kSlotBytes = kStepCodes + kStepMeta;
// Operand rows that are streamed with the codes have slots of 256 bytes a row, two rows at least (every lane's 16 bytes),
// in a place of their own.

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// Where the 16 bytes of unit u of row `row` lie in a slot, and with 16-byte (u < 4), 8-byte (u < 2) or 4-byte loads of the
// product's lanes: the loads take rows 4g + j, j fixed, and what makes them meet different banks goes into bits 0, 1 of the
// row.
//     512 * u + 16 * (row ^ (F <= kFmt4 ? u : u < 2 ? ((row >> 3) & 1) ^ (2 * u) : (row >> 3) & 3))
// Slots start at multiples of 64, so what is exchanged is two bits of an address: one instruction from one row or unit to
// the next.  The writing lane's place in unit u, row = lane:
template <int F, int U>
__device__ __forceinline__ uint32_t write_at(uint32_t slot, uint32_t lane) {
  const uint32_t row = slot + 16 * lane;
  if constexpr (F <= kFmt4) return (row ^ (16 * U)) + 512 * U;
  else if constexpr (U < 2) return (row ^ (lane << 1 & 16) ^ (32 * U)) + 512 * U;
  else return (row ^ (lane << 1 & 48)) + 512 * U;
}
__host__ __device__ constexpr uint32_t piece_at(uint32_t e, uint32_t row) { return e ^ (e >> 2) ^ ((row & 1) << 2); }

// What a warp has still to ask for of one block.  The pointers are the lane's own, of the next step.
struct Feed {
  const char* codes;
  const char* bit1;                               // planes
  const char* bit0;
  const char* meta;                               // lanes 0 .. 7: 16 bytes of the scales, of the zero-points
  const char* x;                                  // streamed operand: the lane's bytes of its first row
  uint32_t x_step;                                // bytes between the rows that a lane copies
  int fmt, left, sub;                             // sub: step inside the group
  int copies;                                     // operand rows that this lane copies from
};

// Sets `f` up for the codes of steps lo .. hi of rows 32 * slice .. of a block of `groups` groups.
__device__ __forceinline__ void feed_codes(Feed& f, int lane, const char* codes, const char* bit1, const char* bit0, int fmt, int groups, int slice,
                                           int lo, int hi) {
  const int ls = step_shift(fmt), sl = slice & 3;
  const size_t tile = (size_t)(slice >> 2) * groups + (lo >> ls);
  f.fmt = fmt;
  f.left = hi - lo;
  f.sub = lo & ((1 << ls) - 1);
  const char* at = codes + tile * kTileBytes[fmt];
  f.meta = at + kScaleOffset[fmt] + 64 * sl + (lane >> 2) * 256 + (lane & 3) * 16;
  const uint32_t row = (uint32_t)(32 * sl + lane) * 16;
  f.codes = at + f.sub * 8192 + row;
  if (fmt >= kFmtP4) {
    f.bit1 = bit1 + tile * kPlaneBitTile + row;
    f.bit0 = bit0 + tile * kPlaneBitTile + row;
  }
}
// ... and for operand rows that are streamed with them: `cols` rows of pieces, `pitch` bytes apart, row c in the order of
// row c.  A lane copies bytes of row lane >> (4 - ls), and of the rows 2 << ls further on.
__device__ __forceinline__ void feed_operand(Feed& f, int lane, const char* x, uint32_t pitch, int cols, int lo) {
  const int ls = step_shift(f.fmt);
  const int c = lane >> (4 - ls);
  f.copies = (cols - c + (2 << ls) - 1) >> (ls + 1);
  f.x = x + (size_t)c * pitch + (size_t)(lo >> ls) * 256 + (lane & ((16 >> ls) - 1)) * 16;
  f.x_step = pitch << (ls + 1);
}

// Asks for a step in format F and moves on; `left` is the caller's.  XC: the most operand rows that are streamed with it, 0:
// the operand is staged.
template <int F, int XC>
__device__ __forceinline__ void ask(Feed& f, uint32_t slot, uint32_t xslot, int lane) {
  constexpr int ls = step_shift(F);
  if constexpr (XC > 0) {
    // the step's part of a group's pieces: all, the half `sub`, or the quarter `sub` (quarters of odd rows are exchanged)
    const char* src = f.x;
    if constexpr (ls == 1) src += f.sub * 128;
    if constexpr (ls == 2) src += (f.sub ^ ((lane >> 2) & 1)) * 64;
    const uint32_t dst = xslot + lane * 16;
#pragma unroll
    for (int j = 0; j < (XC >> (ls + 1) > 0 ? XC >> (ls + 1) : 1); ++j)
      if (j < f.copies) cp16(dst + j * 512, src + j * f.x_step);
    f.x += ls == 0 || f.sub == (1 << ls) - 1 ? 256 : 0;
  }
  constexpr uint32_t tile = stream_tile_bytes(F);
  constexpr int units = F <= kFmt4 ? 4 : F == kFmt3 ? 3 : 2;
  cp16(write_at<F, 0>(slot, lane), f.codes);
  cp16(write_at<F, 1>(slot, lane), f.codes + 2048);
  if constexpr (units > 2) cp16(write_at<F, 2>(slot, lane), f.codes + 4096);
  if constexpr (units > 3) cp16(write_at<F, 3>(slot, lane), f.codes + 6144);
  if (F != kFmt16 && lane < 8) cp16(slot + kStepCodes + lane * 16, f.meta);
  if constexpr (F == kFmtP4 || F == kFmtP3) {
    cp16(write_at<F, 2>(slot, lane), f.bit1);
    f.bit1 += kPlaneBitTile;
  }
  if constexpr (F == kFmtP4) {
    cp16(write_at<F, 3>(slot, lane), f.bit0);
    f.bit0 += kPlaneBitTile;
  }
  if constexpr (F == kFmt16) {
    f.codes += 8192;                            // (a tile of 16 bits has nothing behind its codes)
  } else if constexpr (F == kFmt8) {
    f.codes += f.sub ? tile - 8192u : 8192u;
    f.meta += f.sub ? tile : 0u;
  } else {
    f.codes += tile;
    f.meta += tile;
  }
  if constexpr (ls > 0) f.sub = (f.sub + 1) & ((1 << ls) - 1);
}
template <int XC>
__device__ __forceinline__ void ask_any(Feed& f, uint32_t slot, uint32_t xslot, int lane) {
  f.left--;
  switch (f.fmt) {
    case kFmt16: ask<kFmt16, XC>(f, slot, xslot, lane); break;
    case kFmt8: ask<kFmt8, XC>(f, slot, xslot, lane); break;
    case kFmt4: ask<kFmt4, XC>(f, slot, xslot, lane); break;
    case kFmt3: ask<kFmt3, XC>(f, slot, xslot, lane); break;
    case kFmt2: ask<kFmt2, XC>(f, slot, xslot, lane); break;
    case kFmtP4: ask<kFmtP4, XC>(f, slot, xslot, lane); break;
    case kFmtP3: ask<kFmtP3, XC>(f, slot, xslot, lane); break;
    default: ask<kFmtP2, XC>(f, slot, xslot, lane); break;
  }
}

// Asks the L2 cache for n bytes, a multiple of 16 at a multiple of 16.
__device__ __forceinline__ void prefetch_bytes(const char* p, uint32_t n) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(n) : "memory");
}

// Asks the L2 cache for the feed's first steps, at most STAGES: a lane per line of a step.
template <int STAGES>
__device__ __forceinline__ void prefetch_steps(const Feed& f, int lane) {
  const int ls = step_shift(f.fmt), units = f.fmt <= kFmt4 ? 4 : f.fmt == kFmt3 ? 3 : 2;
  const int bits = f.fmt == kFmtP4 ? 2 : f.fmt == kFmtP3 ? 1 : 0;   // planes of single bits
  // lanes 0 .. 15: units of 512 bytes, four lines each; 16 .. 23: the planes'; 24, 25: scales and zero-points
  const char* line = f.codes - 16 * lane + 2048 * (lane >> 2) + 128 * (lane & 3);
  bool on = lane < 4 * units;
  if (lane >= 16 && lane < 16 + 4 * bits) {
    line = (lane < 20 ? f.bit1 : f.bit0) - 16 * lane + 128 * (lane & 3);
    on = true;
  } else if (lane >= 24 && lane < 26 && f.fmt != kFmt16) {
    line = f.meta - (lane >> 2) * 256 - (lane & 3) * 16 + (lane - 24) * 256;
    on = true;
  }
  const bool plane = lane >= 16 && lane < 24, meta = lane >= 24;
  const uint32_t tile = plane ? (uint32_t)kPlaneBitTile : kTileBytes[f.fmt];
  const int steps = min(STAGES, f.left);
#pragma unroll
  for (int i = 0; i < STAGES; ++i) {
    const int q = f.sub + i;
    const char* at = line + (uint32_t)(q >> ls) * tile;
    if (!plane && !meta) at += ((q & ((1 << ls) - 1)) - f.sub) * 8192;
    if (on && i < steps) asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
  }
}

// ---- staged operand ------------------------------------------------------------------------------
// Two neighbouring pieces (a stretch of 16 columns) of columns as they lie in memory.
__device__ __forceinline__ void make_pieces(const uint4& lo, const uint4& hi, uint4 (&piece)[2]) {
  piece[0] = make_uint4(lo.x, hi.x, lo.y, hi.y);
  piece[1] = make_uint4(lo.z, hi.z, lo.w, hi.w);
}
__device__ __forceinline__ float sum_halves(const uint4& v) {
  const float2 a = __half22float2(u32_as_h2(v.x)), b = __half22float2(u32_as_h2(v.y)), c = __half22float2(u32_as_h2(v.z)), d = __half22float2(u32_as_h2(v.w));
  return ((a.x + a.y) + (b.x + b.y)) + ((c.x + c.y) + (d.x + d.y));
}
// Groups g0 .. g0 + groups of `rows` operand rows (fp16, `pitch` bytes apart, k_bytes of a row count, zeros behind them) ->
// pieces [group][room][256 bytes] and the sums of the first half, the second half and the whole of every group,
// [group][3][room].  By `threads` threads (whole warps), with AHEAD stretches of each in flight.
template <int AHEAD>
__device__ __forceinline__ void stage_operand(const char* x, size_t pitch, int rows, int room, int g0, int groups, int k_bytes, char* pieces, float* sums,
                                              int thread, int threads) {
  const int n = rows * groups * 8;
  const uint32_t per_row = ((1u << 20) + rows - 1) / rows;   // (i / rows for i below 2^16: there is no room for more)
#pragma unroll 1
  for (int base = thread & ~31; base < n; base += AHEAD * threads) {
    uint4 v[AHEAD][2];
    int place[AHEAD];                            // group, row
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = base + a * threads + (thread & 31), s = i & 7, rg = i >> 3, g = (int)(rg * per_row >> 20), c = rg - g * rows;
      place[a] = g << 8 | c;
      v[a][0] = v[a][1] = make_uint4(0, 0, 0, 0);
      if (i < n) {
        const int k = (g0 + g) * 256 + s * 32;
        const char* src = x + (size_t)c * pitch + k;
        if (k + 32 <= k_bytes) {
          v[a][0] = reinterpret_cast<const uint4*>(src)[0];
          v[a][1] = reinterpret_cast<const uint4*>(src)[1];
        } else if (k < k_bytes) {
          // (one way only for the last, short stretch: it is met once in a row)
          uint32_t w[8] = {};
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (k + 4 * j < k_bytes) w[j] = reinterpret_cast<const uint16_t*>(src)[2 * j];
            if (k + 4 * j + 2 < k_bytes) w[j] |= (uint32_t) reinterpret_cast<const uint16_t*>(src)[2 * j + 1] << 16;
          }
          v[a][0] = make_uint4(w[0], w[1], w[2], w[3]);
          v[a][1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
      }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (base + a * threads >= n) break;         // (the same for a whole warp)
      const int i = base + a * threads + (thread & 31), s = i & 7, g = place[a] >> 8, c = place[a] & 255;
      if (i < n) {
        uint4 piece[2];
        make_pieces(v[a][0], v[a][1], piece);
        char* row = pieces + (size_t)(g * room + c) * 256;
        *reinterpret_cast<uint4*>(row + piece_at(2 * s, c) * 16) = piece[0];
        *reinterpret_cast<uint4*>(row + piece_at(2 * s + 1, c) * 16) = piece[1];
      }
      float part = sum_halves(v[a][0]) + sum_halves(v[a][1]);
      part += __shfl_xor_sync(0xffffffffu, part, 1);
      part += __shfl_xor_sync(0xffffffffu, part, 2);
      const float whole = part + __shfl_xor_sync(0xffffffffu, part, 4);
      if (i < n && (s & 3) == 0) {
        sums[(g * 3 + (s >> 2)) * room + c] = part;
        if (s == 0) sums[(g * 3 + 2) * room + c] = whole;
      }
    }
  }
}

// The operand of a block's steps, as a lane reads it.
struct Operand {
  uint32_t x;                                     // staged: this lane's row of group 0; streamed: the row's place in a slot
  uint32_t sum0, sum1;                            // staged, with sums: those of group 0, tokens 2t and 2t + 1
  int room;                                       // staged: rows there is room for
  uint32_t flip;                                  // 4 for an odd row (see piece_at; not in a streamed quarter of a group)
  int step;                                       // next step of the block
};

// ---- the product of a step -----------------------------------------------------------------------
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Constant operands in registers that the compiler takes for unknown values: constants it writes anew in front of every
// instruction, which was a sixth of a 4-bit step's instructions.
struct Fixed {
  float zero[4];
  uint32_t up[3];                                 // 16 (4 bits); 64, 16, 4: a multiplication is not for the pipe of the shifts
  __device__ __forceinline__ Fixed() {
    asm volatile("mov.b32 %0, 64;" : "=r"(up[0]));
    asm volatile("mov.b32 %0, 16;" : "=r"(up[1]));
    asm volatile("mov.b32 %0, 4;" : "=r"(up[2]));
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("mov.b32 %0, 0f00000000;" : "=f"(zero[i]));
  }
};
__device__ __forceinline__ void mma16_first(const Fixed& k, float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(k.zero[0]), "f"(k.zero[1]), "f"(k.zero[2]), "f"(k.zero[3]));
}
constexpr uint32_t kOnes = 0x3c003c00u;           // two fp16 ones

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t moved_by(uint32_t x, int s) { return s >= 0 ? x >> s : x << -s; }

// tot[h]: rows 4g + 2h (0, 1) and 4g + 2h + 1 (2, 3), tokens 2t (0, 2) and 2t + 1 (1, 3).
struct Scales {
  float s[4], z[4];
};
template <int F>
__device__ __forceinline__ void load_scales(uint32_t slot, uint32_t g, Scales& m) {
  constexpr float up = F == kFmt8 ? 16777216.0f : F == kFmt4 ? 1048576.0f : 262144.0f;   // 2^24 over the place of a code
  const uint2 s = lds8(slot + 8 * g + kStepCodes), z = lds8(slot + 8 * g + kStepCodes + 64);
  const float2 s0 = __half22float2(u32_as_h2(s.x)), s1 = __half22float2(u32_as_h2(s.y));
  const float2 z0 = __half22float2(u32_as_h2(z.x)), z1 = __half22float2(u32_as_h2(z.y));
  m.s[0] = s0.x * up, m.s[1] = s0.y * up, m.s[2] = s1.x * up, m.s[3] = s1.y * up;
  m.z[0] = z0.x, m.z[1] = z0.y, m.z[2] = z1.x, m.z[3] = z1.y;
}
// acc: the products of the codes, over what load_scales puts on the scales
__device__ __forceinline__ void apply_scales(const Scales& m, int h, const float (&acc)[4], float sum0, float sum1, float (&tot)[4]) {
  tot[0] = fmaf(m.s[2 * h], acc[0], fmaf(m.z[2 * h], sum0, tot[0]));
  tot[1] = fmaf(m.s[2 * h], acc[1], fmaf(m.z[2 * h], sum1, tot[1]));
  tot[2] = fmaf(m.s[2 * h + 1], acc[2], fmaf(m.z[2 * h + 1], sum0, tot[2]));
  tot[3] = fmaf(m.s[2 * h + 1], acc[3], fmaf(m.z[2 * h + 1], sum1, tot[3]));
}

// The codes of one row's stretch of 16 columns as operands: pair(j, p) = pair j of its first (p = 0) and second eight
// columns, as integers at bit 0 (8 bits), 4 (4 bits) or 6.
template <int F>
struct Codes {
  static constexpr int up = F == kFmtP4 ? 2 : F == kFmtP3 ? 1 : 0;   // planes: bits below the leading two
  static constexpr bool third = F == kFmt3;

  uint32_t w[4];                                  // 8 bits: the words of a stretch; 4 bits: the two; else top codes and low bits
  // stretch s of the step for this lane (8 bits: the only one)
  __device__ __forceinline__ void take(const uint4& wide, const uint2& lead, uint32_t h1, uint32_t h0, int s) {
    if constexpr (F == kFmt8) {
      w[0] = wide.x, w[1] = wide.y, w[2] = wide.z, w[3] = wide.w;
    } else if constexpr (F == kFmt4) {
      w[0] = word_of(wide, 2 * s), w[1] = word_of(wide, 2 * s + 1);
    } else {
      const uint32_t l = s ? lead.y : lead.x;
      w[0] = l << up;
      w[1] = l >> (8 - up);
      if constexpr (third) {                      // the third bit stands above the two: at 2j + 2
        w[2] = moved_by(h1, 8 * s - 2);
        w[3] = moved_by(h1, 8 * s - 1);
      } else if constexpr (up == 1) {
        w[2] = moved_by(h1, 8 * s);
        w[3] = moved_by(h1, 8 * s + 1);
      } else if constexpr (up == 2) {
        w[2] = and_or(moved_by(h1, 8 * s - 1), 0x00aa00aau, (h0 >> (8 * s)) & 0x00550055u);
        w[3] = and_or(moved_by(h1, 8 * s), 0x00aa00aau, (h0 >> (8 * s + 1)) & 0x00550055u);
      }
    }
  }
  __device__ __forceinline__ uint32_t pair(const Fixed& k, int j, int p) const {
    if constexpr (F == kFmt8) {
      return __byte_perm(w[2 * p + (j >> 1)], 0, j & 1 ? 0x4342 : 0x4140);
    } else if constexpr (F == kFmt4) {
      const uint32_t byte = j & 2 ? w[p] >> 8 : w[p];
      return (j & 1 ? byte : byte * k.up[1]) & 0x00f000f0u;
    } else {
      constexpr uint32_t one = 0x00010001u;
      uint32_t v = w[p] & ((3u << (2 * j + up)) * one);
      if constexpr (third || up) v = and_or(w[2 + p], (third ? 4u << (2 * j) : up == 2 ? 3u << (2 * j) : 1u << (2 * j)) * one, v);
      return j == 3 ? v : v * k.up[j];
    }
  }
};

// One step in format F out of a slot.  xrow: this lane's operand row, with the step's pieces at at0 ^ 16 i.  SUMS:
// the operands' sums are at at_sum0 and at_sum1, else they are made here, by a row of ones on the same fragments.
template <int F, bool SUMS>
__device__ __forceinline__ void multiply_step(const Fixed& k, uint32_t slot, int lane, uint32_t xrow, uint32_t at0, uint32_t at_sum0, uint32_t at_sum1,
                                              float (&tot)[2][4]) {
  const uint32_t g = (uint32_t)lane >> 2, t = (uint32_t)lane & 3;
  if constexpr (F == kFmt16) {
    // columns of the lane: pairs 2b, 2b + 1 (b = t mod 2) of both halves of stretch t / 2
    const uint32_t at = slot + 1024 * (t >> 1) + 8 * (t & 1) + 64 * g + 32 * (t >> 1);   // unit 2 (t / 2), row 4g
    const uint4 x = lds16(xrow + at0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t r0 = at ^ (32 * h), r1 = r0 ^ 16;
      const uint2 a0 = lds8(r0), b0 = lds8(r1), a1 = lds8(r1 + 512), b1 = lds8(r0 + 512);
      mma16(tot[h], a0.x, b0.x, a1.x, b1.x, x.x, x.y);
      mma16(tot[h], a0.y, b0.y, a1.y, b1.y, x.z, x.w);
    }
  } else {
    using C = Codes<F>;
    constexpr int S = F == kFmt8 ? 1 : 2;         // stretches of a lane
    uint4 x[2 * S];
#pragma unroll
    for (int i = 0; i < 2 * S; ++i) x[i] = lds16((xrow + at0) ^ (16 * i));
    float sum0, sum1;
    if constexpr (SUMS) {
      sum0 = __uint_as_float(lds4(at_sum0)), sum1 = __uint_as_float(lds4(at_sum1));
    } else {
      float ones[4];
#pragma unroll
      for (int i = 0; i < 2 * S; ++i) {
        if (i == 0) mma16_first(k, ones, kOnes, kOnes, kOnes, kOnes, x[i].x, x[i].y);
        else mma16(ones, kOnes, kOnes, kOnes, kOnes, x[i].x, x[i].y);
        mma16(ones, kOnes, kOnes, kOnes, kOnes, x[i].z, x[i].w);
      }
      sum0 = ones[0], sum1 = ones[1];
    }
    Scales m;
    load_scales<F>(slot, g, m);
    // row 4g of the lane's unit, of its part of a leading unit, of its part of units 2 and 3
    const uint32_t wide_at = slot + 64 * g + 528 * t;
    const uint32_t lead_at = slot + 64 * g + 16 * ((g >> 1 & 1) ^ (t & 2)) + 512 * (t >> 1) + 8 * (t & 1);
    const uint32_t low_at = slot + 64 * g + 16 * (g >> 1 & 3) + 4 * t;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 wide[2];
      uint2 lead[2];
      uint32_t h1[2], h0[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t row = 16 * (2 * h + r);
        wide[r] = make_uint4(0, 0, 0, 0), lead[r] = make_uint2(0, 0), h1[r] = h0[r] = 0;
        if constexpr (F <= kFmt4) wide[r] = lds16(wide_at ^ row);
        else lead[r] = lds8(lead_at ^ row);
        if constexpr (C::third || C::up) h1[r] = lds4((low_at ^ row) + 1024);
        if constexpr (C::up == 2) h0[r] = lds4((low_at ^ row) + 1536);
      }
      float acc[4];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        C c[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) c[r].take(wide[r], lead[r], h1[r], h0[r], s);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4& xs = x[2 * s + (j >> 1)];
          const uint32_t b0 = j & 1 ? xs.z : xs.x, b1 = j & 1 ? xs.w : xs.y;
          if (s == 0 && j == 0) mma16_first(k, acc, c[0].pair(k, j, 0), c[1].pair(k, j, 0), c[0].pair(k, j, 1), c[1].pair(k, j, 1), b0, b1);
          else mma16(acc, c[0].pair(k, j, 0), c[1].pair(k, j, 0), c[0].pair(k, j, 1), c[1].pair(k, j, 1), b0, b1);
        }
      }
      apply_scales(m, h, acc, sum0, sum1, tot[h]);
    }
  }
}

// ---- a warp's walk over its steps ----------------------------------------------------------------
struct Ring {
  uint32_t base, slot;                            // shared memory: the warp's slots, the next step's
  uint32_t x;                                     // the next step's slot of the streamed operand
  int lane;
};
template <int XC, int STAGES>
__device__ __forceinline__ void ring_on(Ring& r) {
  cp_commit();
  const bool last = r.slot == r.base + (STAGES - 1) * kSlotBytes;
  r.slot = last ? r.base : r.slot + kSlotBytes;
  if constexpr (XC > 0) r.x += last ? -(STAGES - 1) * 256 * XC : 256 * XC;
}
// Multiplies steps of a block in format F, at most n, and asks for the next step of the feed after each while that is in
// the same format.  Returns with n = 0, or having multiplied a step without having asked (true).
template <int F, int XC, int STAGES>
__device__ __forceinline__ bool walk_format(const Fixed& k, int& n, Feed& f, Ring& r, Operand& o, float (&tot)[2][4]) {
  constexpr int ls = step_shift(F);
  const uint32_t t = (uint32_t)r.lane & 3;
  // The lane's pieces of a step: e = 4t + i, 8q + 2t + i or 4q + t, q the step inside its group, in the order of piece_at:
  // at0 ^ (what q adds) ^ i.  A streamed row is the part of its step.
  const uint32_t at0 = 16 * ((ls == 0 ? 5 * t : ls == 1 ? (2 * t) ^ (t >> 1) : t) ^ o.flip);
  constexpr uint32_t of_q = 16 * (ls == 1 ? (XC ? 2 : 10) : XC ? 1 : 5);
  const uint32_t x_group = (uint32_t)o.room * 256, sum_part = (uint32_t)o.room * 4, sum_group = 3 * sum_part, grp = (uint32_t)o.step >> ls;
  uint32_t x = o.x, sum0 = o.sum0, sum1 = o.sum1;
  if constexpr (XC == 0) x += grp * x_group, sum0 += grp * sum_group, sum1 += grp * sum_group;
  int asks = f.fmt == F ? min(n, f.left) : 0;
  f.left -= asks;
  bool due = false;
#pragma unroll 1
  do {
    cp_wait<STAGES - 1>();
    __syncwarp();                                 // what the other lanes have copied
    const uint32_t q = ls ? (uint32_t)o.step & ((1 << ls) - 1) : 0;
    const uint32_t part = ls == 1 ? q * sum_part : 2 * sum_part;
    multiply_step<F, XC == 0>(k, r.slot, r.lane, XC ? x + r.x : x, ls ? at0 ^ (of_q * q) : at0, sum0 + part, sum1 + part, tot);
    if (XC == 0 && (ls == 0 || q == (1 << ls) - 1)) {
      x += x_group;
      sum0 += sum_group;
      sum1 += sum_group;
    }
    o.step++;
    __syncwarp();                                 // every lane has read the slot
    --n;
    due = asks == 0;
    if (due) break;
    --asks;
    ask<F, XC>(f, r.slot, r.x, r.lane);
    ring_on<XC, STAGES>(r);
  } while (n);
  return due;
}
// Multiplies the next n steps, all of one block in format `fmt` (F, if that is not kAnyFormat: all blocks are), and asks for
// as many.  ask_next(): asks for the feed's next step, of the next block if need be, into the ring's next slot, or for
// nothing if there is none.
constexpr int kAnyFormat = -1;
template <int F, int XC, int STAGES, class AskNext>
__device__ __forceinline__ void walk(const Fixed& k, int fmt, int n, Feed& f, Ring& r, Operand& o, float (&tot)[2][4], AskNext ask_next) {
  while (n) {
    bool due;
    if constexpr (F != kAnyFormat) {
      due = walk_format<F, XC, STAGES>(k, n, f, r, o, tot);
    } else {
      switch (fmt) {
        case kFmt16: due = walk_format<kFmt16, XC, STAGES>(k, n, f, r, o, tot); break;
        case kFmt8: due = walk_format<kFmt8, XC, STAGES>(k, n, f, r, o, tot); break;
        case kFmt4: due = walk_format<kFmt4, XC, STAGES>(k, n, f, r, o, tot); break;
        case kFmt3: due = walk_format<kFmt3, XC, STAGES>(k, n, f, r, o, tot); break;
        case kFmtP4: due = walk_format<kFmtP4, XC, STAGES>(k, n, f, r, o, tot); break;
        case kFmtP3: due = walk_format<kFmtP3, XC, STAGES>(k, n, f, r, o, tot); break;
        case kFmt2: due = walk_format<kFmt2, XC, STAGES>(k, n, f, r, o, tot); break;
        default: due = walk_format<kFmtP2, XC, STAGES>(k, n, f, r, o, tot); break;
      }
    }
    if (due) {
      ask_next();
      ring_on<XC, STAGES>(r);
    }
  }
}

// ---- sums of the warps ---------------------------------------------------------------------------
// A warp's 32 x 8 sums in shared memory: [token][kSumPitch], so that neither the stores of a fragment nor the loads of
// 32 rows meet in a bank.
constexpr int kSumPitch = 36;
constexpr int kSumFloats = kUnitCols * kSumPitch;
__device__ __forceinline__ void put_sums(float* mine, int lane, const float (&tot)[2][4]) {
  const int g = lane >> 2, t = lane & 3;
  *reinterpret_cast<float4*>(mine + 2 * t * kSumPitch + 4 * g) = make_float4(tot[0][0], tot[0][2], tot[1][0], tot[1][2]);
  *reinterpret_cast<float4*>(mine + (2 * t + 1) * kSumPitch + 4 * g) = make_float4(tot[0][1], tot[0][3], tot[1][1], tot[1][3]);
}

}  // namespace pw
