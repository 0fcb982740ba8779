// Operand tiles of the MFMA products: from global memory straight into LDS
// and from there into fragments. 16-bit elements, whatever they hold (bf16, or
// the fp16 halves of a split fp32 value).
#pragma once

#include "lds_dma.h"

namespace {

DEV int bitrev3(int x) { return ((x & 1) << 2) | (x & 2) | ((x >> 2) & 1); }

// Physical 16-byte unit of logical (row, chunk) in a contraction-contiguous
// tile [R][BK]. 32 lanes read 32 consecutive rows at one chunk; the XOR
// spreads them over all 64 banks.
template <int BK>
DEV int unit_n(int row, int c) {
  if constexpr (BK == 32) return row * 4 + (c ^ ((row >> 2) & 3));
  else return row * 8 + (c ^ bitrev3((row >> 1) & 7));
}
// ... in a contraction-strided tile [BK][R]: R/8 units per k-row. A
// transposed fragment read touches 4 consecutive k-rows x 4 units per
// 32 lanes; the chunk XOR spreads those 16 units over all 64 banks:
// 4*(k%4) when a row is a multiple of 16 units (256 B), 4*((k/2)%2) for
// 192-wide tiles (24 units, so consecutive rows already sit 8 units apart).
// Both stay inside aligned groups of 8 or 16 units, hence inside the row.
template <int R>
DEV int unit_t(int k, int c) {
  if constexpr ((R / 8) % 16 == 0) return k * (R / 8) + (c ^ ((k & 3) << 2));
  else return k * (R / 8) + (c ^ (((k >> 1) & 1) << 2));
}

// Issue the direct-to-LDS loads of one operand tile (R rows of the operand,
// BK contraction steps starting at k0) into the stage at `dst`. Wave w of NW
// issues instructions w, w+NW, ...; each instruction moves 64 units (1 KB),
// unit u of the tile going to byte 16*u.
// With PAIRS (a contraction-contiguous operand only), tile row r reads
// operand row r0 + 32 (r / 64) + r % 32, plus alt for the odd 32-row groups:
// 32 rows of one block of the operand, then the same 32 rows of the block
// alt rows further on, and so on.
template <int R, int BK, bool TR, int NW, bool PAIRS = false>
DEV void issue_tile(v4i32 rs, int ld, int r0, int k0, lds_char_t* dst, int wave, int lane, int alt = 0) {
  static_assert(!PAIRS || (!TR && R % 64 == 0), "paired rows: contraction-contiguous tiles of whole 64-row pairs");
  constexpr int UNITS = R * BK / 8;
  constexpr int INSTR = UNITS / 64;
  static_assert(UNITS % (64 * NW) == 0, "tile must split evenly over the waves");
#pragma unroll
  for (int i = 0; i < INSTR / NW; ++i) {
    const int ins = wave + NW * i;
    const int u = ins * 64 + lane;   // physical unit written by this lane
    uint32_t off;
    if constexpr (!TR) {
      constexpr int U = BK / 8;
      const int row = u / U, p = u % U;
      const int c = unit_n<BK>(row, p) - row * U;   // the XOR is its own inverse
      const int grow = PAIRS ? r0 + 32 * (row >> 6) + (row & 31) + ((row >> 5) & 1) * alt : r0 + row;
      off = ((uint32_t)grow * (uint32_t)ld + (uint32_t)(k0 + c * 8)) * 2u;
    } else {
      const int k = u / (R / 8), p = u % (R / 8);
      const int c = unit_t<R>(k, p) - k * (R / 8);
      off = ((uint32_t)(k0 + k) * (uint32_t)ld + (uint32_t)(r0 + c * 8)) * 2u;
    }
    dma16(rs, off, lds_addr(dst + ins * 1024));
  }
}

// MFMA fragment: 8 consecutive k (k-step s, lane group lane/32) of row
// row_base + lane%32 of the tile.
template <int R, int BK, bool TR>
DEV bf16x8 read_frag(const lds_char_t* stage, int row_base, int s, int lane) {
  if constexpr (!TR) {
    const int row = row_base + (lane & 31), c = 2 * s + (lane >> 5);
    return lds_read16(stage + unit_n<BK>(row, c) * 16);
  } else {
    // lane t of each 16-lane group names k-row kb + t/4 and columns
    // n + 4*(t%4)..+3; it receives column n + t at k-rows kb..kb+3
    const int t = lane & 15, h = (lane >> 4) & 1, g = lane >> 5;
    const int n = row_base + 16 * h + 4 * (t & 3);
    const int kb = 16 * s + 8 * g + (t >> 2);
    const int c = n >> 3, sub = (n & 7) * 2;   // byte offset 0 or 8 in the unit
    const uint2 a = lds_read_tr(stage + unit_t<R>(kb, c) * 16 + sub);
    const uint2 b = lds_read_tr(stage + unit_t<R>(kb + 4, c) * 16 + sub);
    return as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
  }
}

}  // namespace
