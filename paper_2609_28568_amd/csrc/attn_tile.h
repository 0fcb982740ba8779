// Tiles of the attention kernels: rows of one head in LDS, the fragments read
// from them, and the register orders of a 32x32 accumulator.
#pragma once

#include "common.h"
#include "lds_dma.h"

namespace {

constexpr int TILE = 64;    // rows per LDS tile (keys or queries)
typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef LDS_AS v4f32 lds_v4f32_t;
constexpr int BQ = 128;     // rows owned by one workgroup (4 waves x 32)
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float RESCALE_SLACK = 8.0f;

// 2^x with the bare hardware instruction: softmax arguments are at most
// RESCALE_SLACK (forward) or 0 (backward), and results below 2^-126 are
// negligible against the row maximum's term of at least 1
DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

DEV int bitrev3(int x) { return ((x & 1) << 2) | (x & 2) | ((x >> 2) & 1); }
DEV int bitrev4(int x) { return ((x & 1) << 3) | ((x & 2) << 1) | ((x >> 1) & 2) | ((x >> 3) & 1); }

// Physical 16-byte unit of (row, chunk) in a [64][HD] tile. The XOR keeps
// both access patterns free of bank conflicts: 32 lanes reading 16 bytes of
// 32 consecutive rows at one chunk, and 32 lanes of transposed reads covering
// 4 consecutive rows x 4 chunks.
template <int HD>
DEV int unit(int row, int c) {
  constexpr int U = HD / 8;
  int f = 0;
  if constexpr (U == 16) f = bitrev4(row & 15);
  else if constexpr (U == 8) f = bitrev3((row >> 1) & 7);
  else if constexpr (U == 4) f = (row >> 2) & 3;
  return row * U + (c ^ f);
}

// Loads rows [r0, r0+64) of one head's slice (row stride ld elements) of a
// buffer into an LDS tile. Instruction i of the tile goes to bytes
// [1024 i, 1024 i + 1024); waves take instructions in turn. A lane's byte
// offset within the tile's rows is the same for every tile, so it is
// computed once; a tile adds only its (scalar) starting offset.
template <int HD>
struct RowLoader {
  static constexpr int U = HD / 8, UNITS = TILE * U, INSTR = (UNITS + 63) / 64, PER = (INSTR + 3) / 4;
  uint32_t rel[PER];

  DEV void init(int ld, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int u = (wave + 4 * i) * 64 + lane;
      const int row = u / U, p = u % U;
      const int c = unit<HD>(row, p) - row * U;   // the XOR is its own inverse
      rel[i] = ((uint32_t)row * (uint32_t)ld + (uint32_t)(c * 8)) * 2u;
    }
  }

  // off: byte offset in the buffer of row r0 of the head's slice
  DEV void issue(v4i32 rs, uint32_t off, lds_char_t* dst, int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int ins = wave + 4 * i;
      if (ins < INSTR && (UNITS % 64 == 0 || ins * 64 + lane < UNITS))
        dma16(rs, off + rel[i], lds_addr(dst + ins * 1024));
    }
  }
};

// The same load with the lane offsets recomputed per tile (for kernels whose
// registers are at the limit). src: row 0 of the head's slice.
template <int HD>
DEV void issue_rows(v4i32 rs, const bf16_t* base_of_buffer, const bf16_t* src, int r0, int ld, lds_char_t* dst,
                    int wave, int lane) {
  constexpr int U = HD / 8, UNITS = TILE * U, INSTR = (UNITS + 63) / 64;
  const uint32_t src_off = (uint32_t)((src - base_of_buffer) * 2);
  for (int ins = wave; ins < INSTR; ins += 4) {
    const int u = ins * 64 + lane;
    const int row = u / U, p = u % U;
    const int c = unit<HD>(row, p) - row * U;   // the XOR is its own inverse
    const uint32_t off = src_off + ((uint32_t)(r0 + row) * (uint32_t)ld + (uint32_t)(c * 8)) * 2u;
    if (UNITS % 64 == 0 || u < UNITS) dma16(rs, off, lds_addr(dst + ins * 1024));
  }
}

// 8 contraction values of tile row (row) at chunk c (a natural-layout operand).
template <int HD>
DEV bf16x8 read_row(const lds_char_t* t, int row, int c) {
  return lds_read16(t + unit<HD>(row, c) * 16);
}

// Transposed operand from a [64][HD] tile: lane gets column n = d0 +
// lane%32 at tile rows kb + {0..3} (slots 0..3) and kb + 8 + {0..3} (slots
// 4..7), where kb = rbase + 4*(lane/32) -- the register order of a 32x32
// accumulator over rows rbase..rbase+15.
template <int HD>
DEV bf16x8 read_tr(const lds_char_t* t, int d0, int rbase, int lane) {
  const int s = lane & 15, h = (lane >> 4) & 1, g = lane >> 5;
  // for hd 16 the upper 16 output rows of the 32-row MFMA tile are never
  // stored; their columns are folded back into the tile
  const int n = (d0 + 16 * h + 4 * (s & 3)) & (HD < 32 ? HD - 1 : 0x7fffffff);
  const int kb = rbase + 4 * g + (s >> 2);
  const int c = n >> 3, sub = (n & 7) * 2;
  const uint2 a = lds_read_tr(t + unit<HD>(kb, c) * 16 + sub);
  const uint2 b = lds_read_tr(t + unit<HD>(kb + 8, c) * 16 + sub);
  return as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
}

// Registers 8h..8h+7 of a 32x32 fp32 accumulator as a bf16 operand.
DEV bf16x8 acc_slots(const floatx16& x, int h) {
  return as_bf16x8(make_uint4(pack2(x[8 * h + 0], x[8 * h + 1]), pack2(x[8 * h + 2], x[8 * h + 3]),
                              pack2(x[8 * h + 4], x[8 * h + 5]), pack2(x[8 * h + 6], x[8 * h + 7])));
}

// accumulator register r of lane group g sits at row 8*(r/4) + 4g + r%4
DEV int acc_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

DEV void zero(floatx16& x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 0.0f;
}

template <int HD>
struct Shape {
  static constexpr int KS = HD / 16;                 // k-steps over the head dim
  static constexpr int DT = HD < 32 ? 1 : HD / 32;   // 32-row tiles over the head dim
  static constexpr int TB = TILE * HD * 2;           // bytes of one tile
  static constexpr int TBA = (TB + 1023) / 1024 * 1024;
};

// Row loads for an eight-wave workgroup: instruction i of the 64-row tile
// goes to bytes [1024 i, 1024 i + 1024), waves taking instructions in turn.
// off: byte offset in the buffer of row 0 of the head's slice.
template <int HD>
DEV void issue_rows8(v4i32 rs, uint32_t off, int r0, int ld, lds_char_t* dst, int wave, int lane) {
  constexpr int U = HD / 8, INSTR = TILE * U / 64;
  static_assert(INSTR % 8 == 0, "tile must split evenly over 8 waves");
#pragma unroll
  for (int i = 0; i < INSTR / 8; ++i) {
    const int ins = wave + 8 * i;
    const int u = ins * 64 + lane;
    const int row = u / U, p = u % U;
    const int c = unit<HD>(row, p) - row * U;   // the XOR is its own inverse
    dma16(rs, off + ((uint32_t)(r0 + row) * (uint32_t)ld + (uint32_t)(c * 8)) * 2u, lds_addr(dst + ins * 1024));
  }
}

}  // namespace
