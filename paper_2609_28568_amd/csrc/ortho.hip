// Orthogonalised updates: Newton-Schulz products that push every singular
// value of a matrix towards 1, for many matrices at once.
//
//   X0 = G / |G|_F (0 for G = 0; a G taller than wide is transposed),
//   A = X X^T,  P = a I + b A + c A^2,  X <- P X     (each iteration)
//
// with a, b, c = 3.4445, -4.7750, 2.0315: a quintic on the singular values
// that keeps [0, 1.2023] in itself and multiplies small ones by a, so X and A
// stay below 1.5 and P, with its a on the diagonal, below 3.5.
//
// Precision: small singular values are multiplied by a^5 = 485, and rounding
// errors with them, so bf16 products would leave a per cent. Every operand is
// held as two fp16 numbers instead, hi = fp16(v s) and lo = fp16(v s - hi)
// with s = 2^13 (|v| < 3.5, so v s < 28673 of fp16's 65504): 22 bits of v from
// about 2^-15 up, and below that what reaches down to 2^-37, fp16's smallest
// number over s, where 1 is the norm of the matrix. A product is three MFMAs into
// fp32 accumulators: hi hi + hi lo + lo hi. The dropped lo lo is 2^-22 of the
// product at most. That is a third of the fp16 rate, which is five times the
// card's fp32 one.
//
// Matrices that fit the LDS of a CU go through all iterations in one workgroup
// (ortho_small_kernel). For the others, one product kernel for the three
// products; A and A^2 are symmetric, so only the tiles on and below the diagonal
// are computed, and written twice. All matrices of all shapes of one call go
// through each product in one launch: workgroup b finds its group, matrix and
// tile.
//
// What bounds it: 48 matrices of 768 x 768 take 1.60-1.68 ms on different
// cards, their products 800 (A), 745 (P), 780 (X) and, with the fp32 result
// stored, 700 TFLOP/s of MFMA work, at the MFMA unit's power limit for numbers of
// this kind (the library's batched fp16 products of the same sizes: 815 and 706),
// plus 28 and 50 us for the norms and the halves.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/gpt2.h"
#include "common.h"
#include "kernels.h"
#include "lds_dma.h"
#include "tile.h"

namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float v4f32_t __attribute__((ext_vector_type(4)));
typedef LDS_AS v4f32_t lds_v4f32_t;
typedef LDS_AS float lds_f32_t;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float SPLIT = 8192.0f;   // s
constexpr int SMALL_LDS = 156 * 1024;   // of a matrix that stays in LDS, see ortho_small_kernel
constexpr int PAD = 64;            // stored matrices are padded to multiples of this, with zeros

struct Params {
  OrthoGroup g[ORTHO_GROUPS];
  int ngroups;
  _Float16* w;             // planes
  double* parts;           // sums of squares, ORTHO_PARTS per matrix
  const float* norm_coef;  // update: [1] is the clip coefficient
  float momentum, lr, weight_decay, scale;
  int nesterov;
  int src, dst;            // X buffers of this product
};

// Stored matrices are cut into panels of 32 columns, each all its rows of 64
// bytes one after another, so that a tile's 32 contraction steps are one
// contiguous run (or, for the right operand of APPLY, runs of 2 KB): read from
// plain rows, half a cache line of each, the same tiles took twice as long.
DEV size_t panel_at(int row, int col, int rows) { return ((size_t)(col >> 5) * rows + row) * 32 + (col & 31); }

// The matrix and the item within it that global item b falls to, with n(g)
// items per matrix of group g.
template <class N>
DEV const OrthoGroup& locate(const Params& p, int& b, int& mat, N n) {
  int k = 0;
  for (; k + 1 < p.ngroups; ++k) {
    const int t = n(p.g[k]) * p.g[k].count;
    if (b < t) break;
    b -= t;
  }
  const int per = n(p.g[k]);
  mat = b / per;
  b -= mat * per;
  return p.g[k];
}

// first matrix of the group among all
DEV int first_matrix(const Params& p, const OrthoGroup& g) {
  int f = 0;
  for (int k = 0; &p.g[k] != &g; ++k) f += p.g[k].count;
  return f;
}

DEV float update_of(float g, float m_new, float mu, int nesterov) { return nesterov ? fmaf(mu, m_new, g) : m_new; }

// Multiplication by s / sqrt(sum), whatever the range of the sum: a power of
// two, which brings subnormal numbers up whole, and a factor in [0.5, 1) in
// fp32. 0 for no sum (a matrix of zeros).
struct Scale {
  float f;
  int e;
  DEV explicit Scale(double sum) {
    const double inv = sum == 0.0 ? 0.0 : (double)SPLIT / sqrt(sum);
    f = (float)__builtin_amdgcn_frexp_mant(inv);
    e = __builtin_amdgcn_frexp_exp(inv);
  }
  DEV float operator()(float v) const { return __builtin_amdgcn_ldexpf(v, e) * f; }
};

// Sum of squares of each matrix in fp64, ORTHO_PARTS partial sums. With
// UPDATE the momentum is advanced here, m = mu m + coef g, and the matrix is
// the update made of both.
template <bool UPDATE>
__global__ __launch_bounds__(256) void ortho_norm_kernel(Params p) {
  __shared__ double sh[4];
  int b = blockIdx.x, mat;
  const OrthoGroup& g = locate(p, b, mat, [](const OrthoGroup&) { return ORTHO_PARTS; });
  const float* x = g.x + (size_t)mat * g.stride;
  float* mo = UPDATE ? g.mom + (size_t)mat * g.stride : nullptr;
  const float coef = UPDATE ? p.norm_coef[1] : 1.0f;
  const uint32_t cols = (uint32_t)g.cols, n = (uint32_t)g.rows * cols;
  double s = 0.0;
  auto one = [&](float gv, float& mv) {
    if constexpr (UPDATE) {
      gv *= coef;
      mv = fmaf(p.momentum, mv, gv);
      gv = update_of(gv, mv, p.momentum, p.nesterov);
    }
    s += (double)gv * (double)gv;
  };
  if (g.vec) {
    constexpr int FLIGHT = 4;
    for (uint32_t i0 = (b * 256u + threadIdx.x) * 4u; i0 < n; i0 += ORTHO_PARTS * 1024u * FLIGHT) {
      float4 v[FLIGHT], m4[FLIGHT];
      size_t at[FLIGHT];
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        const uint32_t i = min(i0 + ORTHO_PARTS * 1024u * k, n - 4);
        at[k] = (size_t)(i / cols) * g.ld + i % cols;
        v[k] = *reinterpret_cast<const float4*>(x + at[k]);
        if constexpr (UPDATE) m4[k] = *reinterpret_cast<const float4*>(mo + at[k]);
      }
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        if (i0 + ORTHO_PARTS * 1024u * k >= n) break;
        one(v[k].x, m4[k].x); one(v[k].y, m4[k].y); one(v[k].z, m4[k].z); one(v[k].w, m4[k].w);
        if constexpr (UPDATE) *reinterpret_cast<float4*>(mo + at[k]) = m4[k];
      }
    }
  } else {
    for (uint32_t i = b * 256u + threadIdx.x; i < n; i += ORTHO_PARTS * 256u) {
      const size_t at = (size_t)(i / cols) * g.ld + i % cols;
      float mv = UPDATE ? mo[at] : 0.0f;
      one(x[at], mv);
      if constexpr (UPDATE) mo[at] = mv;
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    p.parts[(size_t)(first_matrix(p, g) + mat) * ORTHO_PARTS + b] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// The normalised matrix as hi and lo planes [mp][np], padding zero, in 64 x 64
// tiles through LDS, so that a tall matrix is transposed on the way.
template <bool UPDATE>
__global__ __launch_bounds__(256) void ortho_split_kernel(Params p) {
  __shared__ float sh[64][65];
  int b = blockIdx.x, mat;
  const OrthoGroup& g = locate(p, b, mat, [](const OrthoGroup& q) { return (q.mp / PAD) * (q.np / PAD); });
  const int m0 = b / (g.np / PAD) * PAD, n0 = b % (g.np / PAD) * PAD;
  const int tid = threadIdx.x, lane = tid & 63;
  double s = lane < ORTHO_PARTS ? p.parts[(size_t)(first_matrix(p, g) + mat) * ORTHO_PARTS + lane] : 0.0;
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  const Scale inv(s);
  const float coef = UPDATE ? p.norm_coef[1] : 1.0f;
  const float* x = g.x + (size_t)mat * g.stride;
  const float* mo = UPDATE ? g.mom + (size_t)mat * g.stride : nullptr;
  // source tile: rows r0.., columns c0.. of the matrix as it is stored
  const int r0 = g.tall ? n0 : m0, c0 = g.tall ? m0 : n0;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int r = (tid >> 6) + 4 * k, c = lane;
    float v = 0.0f;
    if (r0 + r < g.rows && c0 + c < g.cols) {
      const size_t at = (size_t)(r0 + r) * g.ld + c0 + c;
      v = x[at];
      if constexpr (UPDATE) v = update_of(v * coef, mo[at], p.momentum, p.nesterov);
      v = inv(v);
    }
    if (g.tall) sh[c][r] = v;
    else sh[r][c] = v;
  }
  __syncthreads();
  _Float16* hi = p.w + g.x_off[0] + (size_t)mat * 2 * g.mp * g.np;
  _Float16* lo = hi + (size_t)g.mp * g.np;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int r = tid >> 2, c = 32 * q + 8 * (tid & 3);   // a panel's 64 rows in one run
    const size_t at = panel_at(m0 + r, n0 + c, g.mp);
    half8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = sh[r][c + e];
      h[e] = (_Float16)v;
      l[e] = (_Float16)(v - (float)h[e]);
    }
    *reinterpret_cast<half8*>(hi + at) = h;
    *reinterpret_cast<half8*>(lo + at) = l;
  }
}

// Tile of T rows from r0 on, contraction steps 32 kt.. (a panel of its own)
template <int T>
DEV void issue_panel(v4i32 rs, int rows, int r0, int kt, lds_char_t* dst, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int ins = wave + 4 * i, u = ins * 64 + lane, row = u >> 2;
    const int c = unit_n<32>(row, u & 3) - row * 4;   // the XOR is its own inverse
    dma16(rs, ((uint32_t)kt * (uint32_t)rows + (uint32_t)(r0 + row)) * 64u + (uint32_t)c * 16u,
          lds_addr(dst + ins * 1024));
  }
}
// Tile of T columns from c0 on, contraction steps 32 kt.. the rows
template <int T>
DEV void issue_across(v4i32 rs, int rows, int c0, int kt, lds_char_t* dst, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int ins = wave + 4 * i, u = ins * 64 + lane, k = u / (T / 8), p = u % (T / 8);
    const int c = unit_t<T>(k, p) - k * (T / 8);
    dma16(rs, ((uint32_t)((c0 >> 5) + (c >> 2)) * (uint32_t)rows + (uint32_t)(32 * kt + k)) * 64u + (uint32_t)(c & 3) * 16u,
          lds_addr(dst + ins * 1024));
  }
}

DEV half8 as_half8(bf16x8 v) { return __builtin_bit_cast(half8, v); }

enum Product { GRAM, POLY, APPLY, LAST, LAST_UPDATE };

template <int T>
DEV int product_tiles(const OrthoGroup& g, bool symmetric) {
  const int tm = (g.mp + T - 1) / T;
  return symmetric ? tm * (tm + 1) / 2 : tm * ((g.np + T - 1) / T);
}

// One T x T tile of one product, 2 x 2 waves, a ring of NS stages of the four
// planes' tiles, BK contraction steps each.
//   GRAM   A = X X^T          POLY  P = a I + b A + c A A
//   APPLY  X' = P X           LAST  the fp32 result, LAST_UPDATE the parameters'
template <int T, int NS, int PH>
__global__ __launch_bounds__(256, NS * T * 256 > 80 * 1024 ? 1 : 2) void ortho_product_kernel(Params p) {
  constexpr bool SYM = PH == GRAM || PH == POLY;
  constexpr bool B_T = !SYM;   // X as the right operand: its rows are the contraction
  constexpr int BK = 32;
  constexpr int PLANE = T * BK * 2, STAGE = 4 * PLANE, KSTEPS = BK / 16;
  constexpr int WT = T / 2, TT = WT / 32, LOADS = 4 * PLANE / 4096;
  static_assert(KSTEPS % 2 == 0, "fragment double buffer alternates per k-step");
  __shared__ __attribute__((aligned(1024))) char smem_raw[NS * STAGE];
  lds_char_t* smem = (lds_char_t*)smem_raw;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // every XCD takes a contiguous run of the tiles (blocks are dealt to them in turn)
  int b = blockIdx.x, mat;
  {
    const int tot = gridDim.x, x = b & 7;
    b = x * (tot >> 3) + min(x, tot & 7) + (b >> 3);
  }
  const OrthoGroup& g = locate(p, b, mat, [](const OrthoGroup& q) { return product_tiles<T>(q, SYM); });
  int ti, tj;
  if constexpr (SYM) {
    ti = (int)((sqrtf(8.0f * b + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > b) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= b) ++ti;
    tj = b - ti * (ti + 1) / 2;
  } else {
    const int tn = (g.np + T - 1) / T;
    ti = b / tn;
    tj = b - ti * tn;
  }
  const int m0 = ti * T, n0 = tj * T;
  const size_t xn = (size_t)g.mp * g.np, an = (size_t)g.mp * g.mp;
  const _Float16* X = p.w + g.x_off[p.src] + (size_t)mat * 2 * xn;
  _Float16* A = p.w + g.a_off + (size_t)mat * 2 * an;
  _Float16* P = p.w + g.p_off + (size_t)mat * 2 * an;
  const _Float16* L = PH == GRAM ? X : PH == POLY ? A : P;
  const _Float16* R = PH == POLY ? A : X;
  const size_t ln = PH == GRAM ? xn : an, rn = PH == POLY ? an : xn;
  const int K = PH == GRAM ? g.np : g.mp;
  v4i32 rl[2], rr[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    rl[h] = make_rsrc(L + h * ln, (uint32_t)(ln * 2));
    rr[h] = make_rsrc(R + h * rn, (uint32_t)(rn * 2));
  }
  // a stage's loads, in three parts
  auto issue = [&](int kt, int part) {
    lds_char_t* st = smem + kt % NS * STAGE;
    auto right = [&](int h) {
      if constexpr (SYM) issue_panel<T>(rr[h], g.mp, n0, kt, st + (2 + h) * PLANE, wave, lane);
      else issue_across<T>(rr[h], g.mp, n0, kt, st + (2 + h) * PLANE, wave, lane);
    };
    if (part == 0) issue_panel<T>(rl[0], g.mp, m0, kt, st, wave, lane);
    if (part == 0) right(0);
    if (part == 1) issue_panel<T>(rl[1], g.mp, m0, kt, st + PLANE, wave, lane);
    if (part == 2) right(1);
  };
  // The cross terms in sums of their own where the registers hold them (192
  // would take 288 for the sums alone), so that the large sums are rounded a
  // third as often. Against 64 bits, one sum and two: 28 x 2032 2.2e-6 and
  // 1.2e-6, 682 x 489 2.3e-6 and 1.4e-6, 1024 x 1024 3.0e-6 and 1.8e-6 (fp32
  // library products 1.1e-6, 2.1e-6, 2.5e-6), for at most a hundredth of the time.
  constexpr bool APART = T <= 128;
  floatx16 acc[TT][TT], low[APART ? TT : 1][APART ? TT : 1];
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        acc[i][j][r] = 0.0f;
        if constexpr (APART) low[i][j][r] = 0.0f;
      }
  half8 fl[2][2][TT], fr[2][2][TT];   // [buffer][hi, lo]
  constexpr int FRAGS = 4 * TT;
  // a k-step's fragments, in three parts, the hi ones first
  auto load = [&](int b, int kt, int s, int part) {
    const lds_char_t* st = smem + kt % NS * STAGE;
#pragma unroll
    for (int f = FRAGS * part / 3; f < FRAGS * (part + 1) / 3; ++f) {
      const int h = f / (2 * TT), i = f % TT;
      if (f / TT % 2 == 0) fl[b][h][i] = as_half8(read_frag<T, BK, false>(st + h * PLANE, wm * WT + 32 * i, s, lane));
      else fr[b][h][i] = as_half8(read_frag<T, BK, B_T>(st + (2 + h) * PLANE, wn * WT + 32 * i, s, lane));
    }
  };
  // hi hi, then the two cross terms
  auto mma = [&](int b, int part) {
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
      for (int j = 0; j < TT; ++j) {
        floatx16& sum = APART && part > 0 ? low[APART ? i : 0][APART ? j : 0] : acc[i][j];
        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[b][part == 1][j], fl[b][part == 2][i], sum, 0, 0, 0);
      }
  };
  // One k-step's MFMAs on fragment buffer b, with the reads of the next step's
  // fragments and the loads of a later stage dealt out between them: issued in
  // one go, the reads hold the wave until LDS has taken them, and the MFMA
  // unit idles meanwhile.
  auto step = [&](int b, bool more, int kt_read, int s_read, bool fetch, int kt_fetch) {
#pragma unroll
    for (int part = 0; part < 3; ++part) {
      if (fetch) issue(kt_fetch, part);
      if (more) load(b ^ 1, kt_read, s_read, part);
      mma(b, part);
#pragma unroll
      for (int k = 0; k < TT * TT; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // an LDS read
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // an MFMA
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // The last k-step of a stage reads from the next: before it every wave has
  // waited for its own loads of that stage and its own reads of this one, whose
  // place the barrier then frees.
  const int nk = K / BK;
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < nk)
#pragma unroll
      for (int part = 0; part < 3; ++part) issue(s, part);
  wait_tiles<NS - 1, LOADS>(min(NS, nk) - 1);
  block_barrier();
#pragma unroll
  for (int part = 0; part < 3; ++part) load(0, 0, 0, part);
  for (int kt = 0; kt + 1 < nk; ++kt) {
#pragma unroll
    for (int s = 0; s + 1 < KSTEPS; ++s) step(s & 1, true, kt, s + 1, false, 0);
    wait_tiles<NS - 2, LOADS>(min(NS - 2, nk - 2 - kt));
    __builtin_amdgcn_s_waitcnt(0xC07F);
    block_barrier();
    step(1, true, kt + 1, 0, kt + NS < nk, kt + NS);
  }
#pragma unroll
  for (int s = 0; s + 1 < KSTEPS; ++s) step(s & 1, true, nk - 1, s + 1, false, 0);
  step(1, false, 0, 0, false, 0);
  if constexpr (APART) {
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
      for (int j = 0; j < TT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] += low[i][j][r];
  }

  // Blocks of 32 x 32 go through LDS, so that every store is one contiguous
  // run: from the accumulators, where lane l holds row l%32 and, in registers
  // 4q..4q+3, columns 8q + 4(l/32) + 0..3, to row l/4 (and 16 further on),
  // columns 8(l%4)..+7, which a panel holds as they stand; and read across, the
  // same of the transposed block.
  __syncthreads();   // the stages are free
  constexpr int LD = 36;
  lds_f32_t* blk = (lds_f32_t*)smem_raw + wave * 32 * LD;
  const int br = lane >> 2, bc = 8 * (lane & 3);
  auto rows_of = [&](float* v, int u) {   // row br + 16 u of the block
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const v4f32_t x = *reinterpret_cast<const lds_v4f32_t*>(blk + (br + 16 * u) * LD + bc + e);
      v[e] = x.x; v[e + 1] = x.y; v[e + 2] = x.z; v[e + 3] = x.w;
    }
  };
  auto cols_of = [&](float* v, int u) {   // row br + 16 u of the transposed block
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = blk[(bc + e) * LD + br + 16 * u];
  };
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) {
      const int mb = m0 + wm * WT + 32 * i, nb = n0 + wn * WT + 32 * j;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<lds_v4f32_t*>(blk + (lane & 31) * LD + 8 * q + 4 * (lane >> 5)) =
            v4f32_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]} * (1.0f / SPLIT);
      if constexpr (PH == GRAM || PH == POLY || PH == APPLY) {
        if (mb >= g.mp || nb >= (SYM ? g.mp : g.np)) continue;   // whole blocks lie outside
        _Float16* D = PH == GRAM ? A : PH == POLY ? P : p.w + g.x_off[p.dst] + (size_t)mat * 2 * xn;
        const size_t dn = SYM ? an : xn;
        auto put = [&](size_t at, const float* v) {
          half8 h, l;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
          }
          *reinterpret_cast<half8*>(D + at) = h;
          *reinterpret_cast<half8*>(D + dn + at) = l;
        };
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float v[8];
          rows_of(v, u);
          const int m = mb + br + 16 * u, n = nb + bc;
          const size_t at = panel_at(m, n, g.mp);
          if constexpr (PH == POLY) {
            const half8 h = *reinterpret_cast<const half8*>(A + at), l = *reinterpret_cast<const half8*>(A + an + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = fmaf(NS_C, v[e], NS_B * ((float)h[e] + (float)l[e]));
              if (m == n + e) v[e] += NS_A * SPLIT;
            }
            if (ti != tj)   // for the transposed block
#pragma unroll
              for (int e = 0; e < 8; e += 4)
                *reinterpret_cast<lds_v4f32_t*>(blk + (br + 16 * u) * LD + bc + e) =
                    v4f32_t{v[e], v[e + 1], v[e + 2], v[e + 3]};
          }
          put(at, v);
        }
        if constexpr (SYM)
          if (ti != tj)   // the tile above the diagonal
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              float v[8];
              cols_of(v, u);
              put(panel_at(nb + br + 16 * u, mb + bc, g.mp), v);
            }
      } else {
        // rows and columns as the matrix is stored
        const int rb = g.tall ? nb : mb, cb = g.tall ? mb : nb;
        float* y = g.y + (size_t)mat * g.stride;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float v[8];
          if (g.tall) cols_of(v, u);
          else rows_of(v, u);
          const int r = rb + br + 16 * u, c = cb + bc;
          if (r >= g.rows) continue;
          const size_t at = (size_t)r * g.ld + c;
          auto out = [&](float o, float w) {
#pragma clang fp contract(off)
            o *= 1.0f / SPLIT;
            return PH == LAST_UPDATE ? fmaf(-p.lr, fmaf(p.weight_decay, w, g.scale * o), w) : o;
          };
          if (g.vec && c + 8 <= g.cols) {
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
              float4* dst = reinterpret_cast<float4*>(y + at + e);
              const float4 w = PH == LAST_UPDATE ? *dst : make_float4(0, 0, 0, 0);
              const float4 o = make_float4(out(v[e], w.x), out(v[e + 1], w.y), out(v[e + 2], w.z), out(v[e + 3], w.w));
              *dst = o;
              if constexpr (PH == LAST_UPDATE)
                *reinterpret_cast<uint2*>(g.p_bf16 + (size_t)mat * g.stride + at + e) =
                    make_uint2(pack2(o.x, o.y), pack2(o.z, o.w));
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (c + e >= g.cols) break;
              const float o = out(v[e], PH == LAST_UPDATE ? y[at + e] : 0.0f);
              y[at + e] = o;
              if constexpr (PH == LAST_UPDATE) g.p_bf16[(size_t)mat * g.stride + at + e] = f2bf(o);
            }
          }
        }
      }
    }
}

// A whole small matrix in one workgroup: all iterations with X, and the Gram
// matrix that P then replaces, in LDS, rows of 16-bit halves `xs` (`as`) bytes
// apart, hi plane then lo. 8 waves: the tiles of A and P are dealt to them, with
// few tiles A's contraction too (partial sums through LDS); of X each wave
// takes blocks of 32 columns, which only depend on themselves, so they are
// updated in place. 112 matrices of 16 x 1024: 42 us, two of 64 x 256: 35, where
// 17 launches of the products took 193 and 78; an iteration is 5 us (A 1.5, P
// 1.3, X 2), the loads and the end 10.
struct SmallShape {
  int mp, np, xs, as, split;   // padded sides; row strides; waves that share a tile of A
  int a_at, red_at, bytes;     // LDS offsets of A and of the partial sums
};
__host__ __device__ inline SmallShape small_shape(int m, int n) {
  SmallShape z;
  z.mp = (m + 31) / 32 * 32;
  z.np = (n + 31) / 32 * 32;
  // 16 bytes more than the row: 32 rows read at one column then spread over the banks
  z.xs = 2 * z.np + 16;
  z.as = 2 * z.mp + 16;
  z.split = z.mp == 32 ? 4 : z.mp == 64 ? 2 : 1;
  z.a_at = 2 * z.mp * z.xs;
  z.red_at = z.a_at + 2 * z.mp * z.as;
  const int tm = z.mp / 32, tiles = tm * (tm + 1) / 2;
  z.bytes = z.red_at + (z.split > 1 ? z.split * tiles * 4096 : 0);
  return z;
}
// Whether a matrix goes this way: the whole of it fits the LDS.
inline bool is_small(const OrthoGroup& g) {
  const int m = g.rows < g.cols ? g.rows : g.cols, n = g.rows < g.cols ? g.cols : g.rows;
  return m <= 128 && n <= 4096 && small_shape(m, n).bytes <= SMALL_LDS;
}

// The iterations of a matrix of TM blocks of 32 rows, in LDS from `smem` on.
template <int TM, bool UPDATE>
DEV void small_iterations(const Params& p, const OrthoGroup& g, int mat, const SmallShape& z, lds_char_t* smem,
                          int iterations, int tid) {
  constexpr int MP = 32 * TM, TRI = TM * (TM + 1) / 2, AS = 2 * MP + 16, AP = MP * AS;
  constexpr int SPLITS = TM == 1 ? 4 : TM == 2 ? 2 : 1;
  constexpr int CB = TM == 1 ? 4 : 1;   // column blocks of X in hand
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = g.tall ? g.cols : g.rows, n = g.tall ? g.rows : g.cols;
  const int xs = z.xs, xp = MP * xs;
  lds_char_t* X = smem;
  lds_char_t* A = smem + z.a_at;
  lds_char_t* red = smem + z.red_at;
  const int lr = lane & 31, lk = 8 * (lane >> 5), lg = 4 * (lane >> 5);
  // 8 contraction steps along a row, and down a column (rows k0 + 8 (lane/32)
  // + 0..7, column c0 + lane%32), of a plane
  auto along = [&](const lds_char_t* t, int stride, int row0, int k0) {
    return as_half8(lds_read16(t + (row0 + lr) * stride + (k0 + lk) * 2));
  };
  const lds_char_t* xd = X + (lk + ((lane & 15) >> 2)) * xs + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  auto down = [&](int plane, int c0, int k0) {
    const lds_char_t* t = xd + plane + k0 * xs + c0 * 2;
    const uint2 lo = lds_read_tr(t), hi = lds_read_tr(t + 4 * xs);
    return as_half8(as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y)));
  };
  auto mfma = [](half8 nn, half8 mm, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(nn, mm, c, 0, 0, 0); };
  // 4 consecutive columns of a row, split, to both planes
  auto put = [&](lds_char_t* t, int plane, const float* v) {
    half4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[e] = (_Float16)v[e];
      l[e] = (_Float16)(v[e] - (float)h[e]);
    }
    *reinterpret_cast<LDS_AS half4*>(t) = h;
    *reinterpret_cast<LDS_AS half4*>(t + plane) = l;
  };
  // ... of A, on both sides of the diagonal
  auto put_a = [&](int ti, int tj, int row, int col, const float* v) {
    put(A + row * AS + col * 2, AP, v);
    if (ti != tj)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        LDS_AS _Float16* d = (LDS_AS _Float16*)(A + (col + e) * AS) + row;
        const _Float16 h = (_Float16)v[e];
        d[0] = h;
        *(LDS_AS _Float16*)((lds_char_t*)d + AP) = (_Float16)(v[e] - (float)h);
      }
  };
  auto tile_of = [](int t, int& ti, int& tj) {
    ti = 0;
#pragma unroll
    for (int k = 1; k < TM; ++k) ti += t >= k * (k + 1) / 2;
    tj = t - ti * (ti + 1) / 2;
  };

  for (int it = 0; it < iterations; ++it) {
    // A = X X^T, a sum for each of the three products: they need not wait for one another
    for (int u = wave; u < TRI * SPLITS; u += 8) {
      const int t = u / SPLITS, part = u % SPLITS;
      int ti, tj;
      tile_of(t, ti, tj);
      floatx16 acc, hl, lh;
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] = hl[r] = lh[r] = 0.0f;
      const int steps = z.np / 16, k1 = steps * (part + 1) / SPLITS;
#pragma unroll 4
      for (int k = steps * part / SPLITS; k < k1; ++k) {
        const half8 nh = along(X, xs, 32 * tj, 16 * k), nl = along(X + xp, xs, 32 * tj, 16 * k);
        const half8 mh = along(X, xs, 32 * ti, 16 * k), ml = along(X + xp, xs, 32 * ti, 16 * k);
        acc = mfma(nh, mh, acc);
        hl = mfma(nh, ml, hl);
        lh = mfma(nl, mh, lh);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (acc[4 * q + e] + (hl[4 * q + e] + lh[4 * q + e])) * (1.0f / SPLIT);
        if constexpr (SPLITS > 1)
          *reinterpret_cast<lds_v4f32_t*>(red + u * 4096 + (q * 64 + lane) * 16) = v4f32_t{v[0], v[1], v[2], v[3]};
        else put_a(ti, tj, 32 * ti + lr, 32 * tj + 8 * q + lg, v);
      }
    }
    __syncthreads();
    if constexpr (SPLITS > 1) {
      // the parts of each 4 columns added up in order
      for (int i = tid; i < TRI * 256; i += 512) {
        const int t = i >> 8, q = (i >> 6) & 3, l = i & 63;
        int ti, tj;
        tile_of(t, ti, tj);
        v4f32_t a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int part = 0; part < SPLITS; ++part)
          a += *reinterpret_cast<const lds_v4f32_t*>(red + (t * SPLITS + part) * 4096 + (q * 64 + l) * 16);
        const float v[4] = {a.x, a.y, a.z, a.w};
        put_a(ti, tj, 32 * ti + (l & 31), 32 * tj + 8 * q + 4 * (l >> 5), v);
      }
      __syncthreads();
    }
    // P = a I + b A + c A A, held in registers until everyone has read A
    constexpr int PT = (TM * TM + 7) / 8;
    floatx16 pacc[PT];
#pragma unroll
    for (int w = 0; w < PT; ++w) {
      const int t = wave + 8 * w, ti = t / TM, tj = t % TM;
      if (t >= TM * TM) break;
      floatx16 hl, lh;
#pragma unroll
      for (int r = 0; r < 16; ++r) pacc[w][r] = hl[r] = lh[r] = 0.0f;
#pragma unroll
      for (int k = 0; k < MP; k += 16) {
        const half8 nh = along(A, AS, 32 * tj, k), nl = along(A + AP, AS, 32 * tj, k);
        const half8 mh = along(A, AS, 32 * ti, k), ml = along(A + AP, AS, 32 * ti, k);
        pacc[w] = mfma(nh, mh, pacc[w]);
        hl = mfma(nh, ml, hl);
        lh = mfma(nl, mh, lh);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = 32 * ti + lr, col = 32 * tj + 8 * q + lg;
        const half4 h = *reinterpret_cast<const LDS_AS half4*>(A + row * AS + col * 2);
        const half4 l = *reinterpret_cast<const LDS_AS half4*>(A + AP + row * AS + col * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * q + e;
          float v = fmaf(NS_C, (pacc[w][r] + (hl[r] + lh[r])) * (1.0f / SPLIT), NS_B * ((float)h[e] + (float)l[e]));
          if (row == col + e) v += NS_A * SPLIT;
          pacc[w][r] = v;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < PT; ++w) {
      const int t = wave + 8 * w, ti = t / TM, tj = t % TM;
      if (t >= TM * TM) break;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {pacc[w][4 * q], pacc[w][4 * q + 1], pacc[w][4 * q + 2], pacc[w][4 * q + 3]};
        put(A + (32 * ti + lr) * AS + (32 * tj + 8 * q + lg) * 2, AP, v);
      }
    }
    __syncthreads();
    // X <- P X, CB blocks of 32 columns at a time; blocks past the last are the last again, by the same wave
    const bool last = it + 1 == iterations;
    const int blocks = z.np / 32;
    for (int c0 = wave; c0 < blocks; c0 += 8 * CB) {
      floatx16 acc[CB][TM];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[cb][i][r] = 0.0f;
#pragma unroll
      for (int k = 0; k < MP; k += 16) {
        half8 nh[CB], nl[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const int col = 32 * (c0 + 8 * cb < blocks ? c0 + 8 * cb : c0);
          nh[cb] = down(0, col, k);
          nl[cb] = down(xp, col, k);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const half8 mh = along(A, AS, 32 * i, k), ml = along(A + AP, AS, 32 * i, k);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) acc[cb][i] = mfma(nh[cb], mh, acc[cb][i]);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) acc[cb][i] = mfma(nl[cb], mh, acc[cb][i]);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) acc[cb][i] = mfma(nh[cb], ml, acc[cb][i]);
        }
      }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        if (c0 + 8 * cb >= blocks) break;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int row = 32 * i + lr, col = 32 * (c0 + 8 * cb) + 8 * q + lg;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[cb][i][4 * q + e] * (1.0f / SPLIT);
            if (!last) {
              put(X + row * xs + col * 2, xp, v);
              continue;
            }
            if (row >= m) continue;
            float* y = g.y + (size_t)mat * g.stride;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
              if (col + e >= n) break;
              const size_t at = g.tall ? (size_t)(col + e) * g.ld + row : (size_t)row * g.ld + col + e;
              float o = v[e] * (1.0f / SPLIT);
              if constexpr (UPDATE) {
                const float w = y[at];
                o = fmaf(-p.lr, fmaf(p.weight_decay, w, g.scale * o), w);
                g.p_bf16[(size_t)mat * g.stride + at] = f2bf(o);
              }
              y[at] = o;
            }
          }
      }
    }
    __syncthreads();
  }
}

template <bool UPDATE>
__global__ __launch_bounds__(512, 1) void ortho_small_kernel(Params p, int iterations) {
  __shared__ __attribute__((aligned(1024))) char smem_raw[SMALL_LDS];
  __shared__ double sums[8];
  lds_char_t* smem = (lds_char_t*)smem_raw;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int b = blockIdx.x, mat;
  const OrthoGroup& g = locate(p, b, mat, [](const OrthoGroup&) { return 1; });
  const SmallShape z = g.tall ? small_shape(g.cols, g.rows) : small_shape(g.rows, g.cols);
  const float* x = g.x + (size_t)mat * g.stride;
  float* mo = UPDATE ? g.mom + (size_t)mat * g.stride : nullptr;
  const float coef = UPDATE ? p.norm_coef[1] : 1.0f;
  const uint32_t cols = (uint32_t)g.cols, total = (uint32_t)g.rows * cols;

  // zeros where the padding is: rows, or with columns short all of both planes
  const int rows = g.tall ? g.cols : g.rows, plane = z.mp * z.xs;
  const int from = (g.tall ? g.rows : g.cols) == z.np ? rows * z.xs : 0;
  for (int i = from + 16 * tid; i < plane; i += 512 * 16) {
    *reinterpret_cast<lds_v4u32_t*>(smem + i) = v4u32{0, 0, 0, 0};
    *reinterpret_cast<lds_v4u32_t*>(smem + plane + i) = v4u32{0, 0, 0, 0};
  }
  // f(v, row, column, place) on every V elements of the matrix as it is stored
  // (of the update, with FIRST made anew and the momentum advanced), 8 loads of
  // a thread in flight: one by one they took 30 of 50 us
  auto each = [&](auto v_, auto first_, auto f) {
    constexpr int V = decltype(v_)::value, FLIGHT = 8;
    constexpr bool FIRST = decltype(first_)::value;
    using Vec = std::conditional_t<V == 4, float4, float>;
    const uint32_t units = total / V;
    for (uint32_t i0 = tid; i0 < units; i0 += 512 * FLIGHT) {
      Vec v[FLIGHT], mv[FLIGHT];
      uint32_t r[FLIGHT], c[FLIGHT];
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        const uint32_t i = min(i0 + 512u * k, units - 1) * V;
        r[k] = i / cols;
        c[k] = i - r[k] * cols;
        const size_t at = (size_t)r[k] * g.ld + c[k];
        v[k] = *reinterpret_cast<const Vec*>(x + at);
        if constexpr (UPDATE) mv[k] = *reinterpret_cast<const Vec*>(mo + at);
      }
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        if (i0 + 512u * k >= units) break;
        float* pv = reinterpret_cast<float*>(&v[k]);
        if constexpr (UPDATE) {
          float* pm = reinterpret_cast<float*>(&mv[k]);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            pv[e] *= coef;
            if (FIRST) pm[e] = fmaf(p.momentum, pm[e], pv[e]);
            pv[e] = update_of(pv[e], pm[e], p.momentum, p.nesterov);
          }
          if (FIRST) *reinterpret_cast<Vec*>(mo + (size_t)r[k] * g.ld + c[k]) = mv[k];
        }
        f(pv, r[k], c[k]);
      }
    }
  };
  using V1 = std::integral_constant<int, 1>;
  using V4 = std::integral_constant<int, 4>;
  double s = 0.0;
  auto square = [&](auto v_) {
    each(v_, std::true_type{}, [&](const float* v, uint32_t, uint32_t) {
#pragma unroll
      for (int e = 0; e < decltype(v_)::value; ++e) s += (double)v[e] * (double)v[e];
    });
  };
  if (g.vec) square(V4{});
  else square(V1{});
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) sums[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += sums[w];
  const Scale inv(s);
  auto store = [&](auto v_) {
    each(v_, std::false_type{}, [&](const float* v, uint32_t r, uint32_t c) {
      constexpr int V = decltype(v_)::value;
      _Float16 h[V], l[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float u = inv(v[e]);
        h[e] = (_Float16)u;
        l[e] = (_Float16)(u - (float)h[e]);
      }
      if (V == 4 && !g.tall) {
        LDS_AS half4* d = (LDS_AS half4*)(smem + r * z.xs + c * 2);
        *d = half4{h[0], h[V / 4], h[V / 2], h[V - 1]};
        *(LDS_AS half4*)((lds_char_t*)d + plane) = half4{l[0], l[V / 4], l[V / 2], l[V - 1]};
        return;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        LDS_AS _Float16* d = (LDS_AS _Float16*)(smem + (g.tall ? c + e : r) * z.xs) + (g.tall ? r : c + e);
        d[0] = h[e];
        *(LDS_AS _Float16*)((lds_char_t*)d + plane) = l[e];
      }
    });
  };
  if (g.vec) store(V4{});
  else store(V1{});
  __syncthreads();

  switch (z.mp / 32) {   // the same for the whole workgroup
    case 1: return small_iterations<1, UPDATE>(p, g, mat, z, smem, iterations, tid);
    case 2: return small_iterations<2, UPDATE>(p, g, mat, z, smem, iterations, tid);
    case 3: return small_iterations<3, UPDATE>(p, g, mat, z, smem, iterations, tid);
    default: return small_iterations<4, UPDATE>(p, g, mat, z, smem, iterations, tid);
  }
}

template <int PH>
hipError_t product(const Params& p, hipStream_t s) {
  constexpr bool SYM = PH == GRAM || PH == POLY;
  auto tiles = [&](int T) {
    long t = 0;
    for (int k = 0; k < p.ngroups; ++k) {
      const long tm = (p.g[k].mp + T - 1) / T, tn = (p.g[k].np + T - 1) / T;
      t += (SYM ? tm * (tm + 1) / 2 : tm * tn) * p.g[k].count;
    }
    return t;
  };
  const long t128 = tiles(128), t192 = tiles(192);
  int steps = 0;   // the longest contraction
  for (int k = 0; k < p.ngroups; ++k) steps = std::max(steps, PH == GRAM ? p.g[k].np : p.g[k].mp);
#define L(T, NS) hipLaunchKernelGGL((ortho_product_kernel<T, NS, PH>), dim3((unsigned)tiles(T)), dim3(256), 0, s, p)
  // Whole calls with one tile for every product (us; matrices, tiles of 128 in
  // the symmetric and the other products; 64, 128, 128 with three stages, 192):
  //   12 x 512 x 512 (120, 192)    263, 276, 272, 440
  //   16 x 512 x 512 (160, 256)    328, 289, 291, 458
  //   2048 x 2048 (136, 256)       874, 774, 739, 1221
  //   48 x 512 x 512 (480, 768)    705, 621, 688, 927
  //   4 x 1536 x 1536 (312, 576)   1247, 1115, 1342, 1125; 1031 with 192 for X only
  // Tiles of 64 while those of 128 leave half of the CUs idle; three stages for
  // long contractions of one workgroup a CU, whose loads nothing else covers
  // (A of 12 768 x 3072, 252 tiles: 99 -> 84); 192 where the busiest CU then
  // computes less: with tiles of 128 two workgroups share one.
  const long cost128 = ((t128 + 511) / 512 * 2 - (t128 % 512 > 0 && t128 % 512 <= 256)) * 128 * 128;
  const long cost192 = (t192 + 255) / 256 * 192 * 192;
  const bool few_long = t128 <= 256 && steps >= 2048;
  if (t128 < 144) L(64, 4);
  else if (t128 > 256 && cost192 < cost128) L(192, 2);
  else if constexpr (PH == LAST_UPDATE) L(128, 2);   // the steps' blocks of width 2048 have 1,024 tiles and more
  else if (few_long) L(128, 3);
  else L(128, 2);
#undef L
  return hipGetLastError();
}

long align128(long n) { return (n + 127) / 128 * 128; }

}  // namespace

// Offsets of every group's planes (fp16 elements), after the partial sums;
// returns the bytes in all, or 0 when a shape is out of range. Matrices that
// stay in LDS use neither; a nominal 256 bytes for each tile of one of them keep
// a size telling their shapes apart.
size_t ortho_layout(OrthoGroup* g, int ngroups) {
  long mats = 0, tiles = 0, large = 0, nominal = 0;
  for (int k = 0; k < ngroups; ++k) {
    OrthoGroup& q = g[k];
    if (q.rows < 1 || q.cols < 1 || q.count < 1) return 0;
    q.tall = q.rows > q.cols;
    const long m = q.tall ? q.cols : q.rows, n = q.tall ? q.rows : q.cols;
    const long mp = (m + PAD - 1) / PAD * PAD, np = (n + PAD - 1) / PAD * PAD;
    if (np > (1L << 30) || mp * np >= (1L << 31)) return 0;   // 32-bit byte offsets within a plane
    q.mp = (int)mp;
    q.np = (int)np;
    mats += q.count;
    tiles += mp * np / (PAD * PAD) * q.count;
    // launches of less than 2^32 threads
    if (mats * ORTHO_PARTS * 256 >= (1L << 32) || tiles * 256 >= (1L << 32)) return 0;
    if (is_small(q)) nominal += mp * np / (PAD * PAD) * 128;
    else large += q.count;
  }
  long o = align128(large * ORTHO_PARTS * (long)(sizeof(double) / 2)) + nominal;
  for (int k = 0; k < ngroups; ++k) {
    OrthoGroup& q = g[k];
    if (is_small(q)) continue;
    const long xn = align128((long)q.count * 2 * q.mp * q.np), an = align128((long)q.count * 2 * q.mp * q.mp);
    q.x_off[0] = o; o += xn;
    q.x_off[1] = o; o += xn;
    q.a_off = o; o += an;
    q.p_off = o; o += an;
  }
  return (size_t)o * 2;
}

double ortho_flops(const OrthoArgs& a) {
  double fl = 0.0;
  for (int k = 0; k < a.ngroups; ++k) {
    const double m = std::min(a.g[k].rows, a.g[k].cols), n = std::max(a.g[k].rows, a.g[k].cols);
    fl += a.iterations * a.g[k].count * (m * (m + 1) * n + m * m * (m + 1) + 2.0 * m * m * n);
  }
  return fl;
}

const char* muon_invalid(const gpt2_muon* how) {
  if (!how) return "the update's settings are NULL";
  if (!(how->momentum >= 0.0f && how->momentum < 1.0f)) return "momentum must be in [0, 1)";
  if (how->iterations < 1 || how->iterations > 32) return "iterations must be in 1..32";
  if (!(how->scale > 0.0f && std::isfinite(how->scale))) return "scale must be positive";
  return nullptr;
}

hipError_t launch_orthogonalise(const OrthoArgs& a, hipStream_t s) {
  if (a.ngroups < 1 || a.ngroups > ORTHO_GROUPS || a.iterations < 1) return hipErrorInvalidValue;
  OrthoGroup all[ORTHO_GROUPS];
  for (int k = 0; k < a.ngroups; ++k) all[k] = a.g[k];
  if (!ortho_layout(all, a.ngroups)) return hipErrorInvalidValue;
  Params p{}, small{};   // matrices that go through the products, and through LDS
  unsigned mats = 0, tiles = 0, smalls = 0;
  for (int k = 0; k < a.ngroups; ++k) {
    OrthoGroup& q = all[k];
    auto ok = [](const void* v) { return (reinterpret_cast<uintptr_t>(v) & 15) == 0; };
    q.vec = q.cols % 4 == 0 && q.ld % 4 == 0 && q.stride % 4 == 0 && ok(q.x) && ok(q.y) && ok(q.mom) && ok(q.p_bf16);
    if (is_small(q)) {
      small.g[small.ngroups++] = q;
      smalls += q.count;
      continue;
    }
    p.g[p.ngroups++] = q;
    mats += q.count;
    tiles += (q.mp / PAD) * (q.np / PAD) * q.count;
  }
  p.w = static_cast<_Float16*>(a.workspace);
  p.parts = static_cast<double*>(a.workspace);
  p.norm_coef = small.norm_coef = a.norm_coef;
  p.momentum = small.momentum = a.momentum;
  p.nesterov = small.nesterov = a.nesterov;
  p.lr = small.lr = a.lr;
  p.weight_decay = small.weight_decay = a.weight_decay;
  if (smalls) {
    if (a.update) hipLaunchKernelGGL(ortho_small_kernel<true>, dim3(smalls), dim3(512), 0, s, small, a.iterations);
    else hipLaunchKernelGGL(ortho_small_kernel<false>, dim3(smalls), dim3(512), 0, s, small, a.iterations);
  }
  if (!mats) return hipGetLastError();
  if (a.update) {
    hipLaunchKernelGGL((ortho_norm_kernel<true>), dim3(mats * ORTHO_PARTS), dim3(256), 0, s, p);
    hipLaunchKernelGGL((ortho_split_kernel<true>), dim3(tiles), dim3(256), 0, s, p);
  } else {
    hipLaunchKernelGGL((ortho_norm_kernel<false>), dim3(mats * ORTHO_PARTS), dim3(256), 0, s, p);
    hipLaunchKernelGGL((ortho_split_kernel<false>), dim3(tiles), dim3(256), 0, s, p);
  }
  hipError_t e = hipGetLastError();
  for (int it = 0; it < a.iterations && e == hipSuccess; ++it) {
    p.src = it & 1;
    p.dst = p.src ^ 1;
    e = product<GRAM>(p, s);
    if (e == hipSuccess) e = product<POLY>(p, s);
    if (e != hipSuccess) break;
    if (it + 1 < a.iterations) e = product<APPLY>(p, s);
    else e = a.update ? product<LAST_UPDATE>(p, s) : product<LAST>(p, s);
  }
  return e;
}
