// Orthogonalised updates: Newton-Schulz products that push every singular
// value of a matrix towards 1, for many matrices at once.
//
//   X0 = G / |G|_F (0 for G = 0; a G taller than wide is transposed),
//   A = X X^T,  P = a I + b A + c A^2,  X <- P X     (each iteration)
//
// with a, b, c = 3.4445, -4.7750, 2.0315: a quintic on the singular values
// that keeps [0, 1.2023] in itself and multiplies small ones by a, so all the
// values the iteration stores stay within a factor of 3 of 1 or below.
//
// Precision: small singular values are multiplied by a^5 = 485, and rounding
// errors with them, so bf16 products would leave a per cent. Every operand is
// held as two fp16 numbers instead, hi = fp16(v s) and lo = fp16(v s - hi)
// with s = 2^13 (|v| < 3, so v s < 65504; the rest of an fp32 significand down
// to 2^-37 absolute), and a product is three MFMAs into one fp32 accumulator:
// hi hi + hi lo + lo hi. The dropped lo lo is 2^-22 of the product at most.
// That is a third of the fp16 rate, five times the card's fp32 one.
//
// One product kernel for the three products; A and A^2 are symmetric, so only
// the tiles on and below the diagonal are computed, and written twice. All
// matrices of all shapes of one call go through each product in one launch:
// workgroup b finds its group, matrix and tile.
#include <algorithm>
#include <cmath>

#include "../../include/gpt2.h"
#include "common.h"
#include "kernels.h"
#include "lds_dma.h"
#include "tile.h"

namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float SPLIT = 8192.0f;   // s
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
    for (uint32_t i = (b * 256u + threadIdx.x) * 4u; i < n; i += ORTHO_PARTS * 1024u) {
      const size_t at = (size_t)(i / cols) * g.ld + i % cols;
      const float4 v = *reinterpret_cast<const float4*>(x + at);
      float4 m4 = UPDATE ? *reinterpret_cast<const float4*>(mo + at) : make_float4(0, 0, 0, 0);
      one(v.x, m4.x); one(v.y, m4.y); one(v.z, m4.z); one(v.w, m4.w);
      if constexpr (UPDATE) *reinterpret_cast<float4*>(mo + at) = m4;
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
  // in fp64, so that the square root of no sum and the scale of no matrix leave the range
  const double inv = s == 0.0 ? 0.0 : (double)SPLIT / sqrt(s);
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
      v = (float)((double)v * inv);
    }
    if (g.tall) sh[c][r] = v;
    else sh[r][c] = v;
  }
  __syncthreads();
  const int r = tid >> 2, c = 16 * (tid & 3);
  _Float16* hi = p.w + g.x_off[0] + (size_t)mat * 2 * g.mp * g.np + (size_t)(m0 + r) * g.np + n0 + c;
  _Float16* lo = hi + (size_t)g.mp * g.np;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    half8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = sh[r][c + 8 * q + e];
      h[e] = (_Float16)v;
      l[e] = (_Float16)(v - (float)h[e]);
    }
    *reinterpret_cast<half8*>(hi + 8 * q) = h;
    *reinterpret_cast<half8*>(lo + 8 * q) = l;
  }
}

DEV half8 as_half8(bf16x8 v) { return __builtin_bit_cast(half8, v); }

enum Product { GRAM, POLY, APPLY, LAST, LAST_UPDATE };

template <int T>
DEV int product_tiles(const OrthoGroup& g, bool symmetric) {
  const int tm = (g.mp + T - 1) / T;
  return symmetric ? tm * (tm + 1) / 2 : tm * ((g.np + T - 1) / T);
}

// One T x T tile of one product, 2 x 2 waves, double-buffered stages of the
// four planes' tiles, BK contraction steps each.
//   GRAM   A = X X^T          POLY  P = a I + b A + c A A
//   APPLY  X' = P X           LAST  the fp32 result, LAST_UPDATE the parameters'
template <int T, int BK, int PH>
__global__ __launch_bounds__(256, 2) void ortho_product_kernel(Params p) {
  constexpr bool SYM = PH == GRAM || PH == POLY;
  constexpr bool B_T = !SYM;   // X as the right operand: its rows are the contraction
  constexpr int PLANE = T * BK * 2, STAGE = 4 * PLANE, KSTEPS = BK / 16;
  constexpr int WT = T / 2, TT = WT / 32;
  __shared__ __attribute__((aligned(1024))) char smem_raw[2 * STAGE];
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
  const int lld = PH == GRAM ? g.np : g.mp, rld = PH == POLY ? g.mp : g.np;
  const int K = PH == GRAM ? g.np : g.mp;
  v4i32 rl[2], rr[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    rl[h] = make_rsrc(L + h * ln, (uint32_t)(ln * 2));
    rr[h] = make_rsrc(R + h * rn, (uint32_t)(rn * 2));
  }
  auto issue = [&](int kt) {
    lds_char_t* st = smem + (kt & 1) * STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      issue_tile<T, BK, false, 4>(rl[h], lld, m0, kt * BK, st + h * PLANE, wave, lane);
      issue_tile<T, BK, B_T, 4>(rr[h], rld, n0, kt * BK, st + (2 + h) * PLANE, wave, lane);
    }
  };
  floatx16 acc[TT][TT];
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  const int nk = K / BK;
  issue(0);
  for (int kt = 0; kt < nk; ++kt) {
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
    block_barrier();
    if (kt + 1 < nk) issue(kt + 1);
    const lds_char_t* st = smem + (kt & 1) * STAGE;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
      half8 fl[2][TT], fr[2][TT];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < TT; ++i) {
          fl[h][i] = as_half8(read_frag<T, BK, false>(st + h * PLANE, wm * WT + 32 * i, s, lane));
          fr[h][i] = as_half8(read_frag<T, BK, B_T>(st + (2 + h) * PLANE, wn * WT + 32 * i, s, lane));
        }
      // hi hi, then the two cross terms
#pragma unroll
      for (int t = 0; t < 3; ++t)
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
          for (int j = 0; j < TT; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[t == 1][j], fl[t == 2][i], acc[i][j], 0, 0, 0);
    }
  }

  // lane l holds row l%32 of the tile and, in registers 4q..4q+3, columns
  // 8q + 4(l/32) + 0..3
  const int gq = lane >> 5;
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    const int m = m0 + wm * WT + 32 * i + (lane & 31);
#pragma unroll
    for (int j = 0; j < TT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn * WT + 32 * j + 8 * q + 4 * gq;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e] * (1.0f / SPLIT);
        if constexpr (PH == GRAM || PH == POLY || PH == APPLY) {
          const int nld = SYM ? g.mp : g.np;
          if (m >= g.mp || n >= nld) continue;
          const size_t at = (size_t)m * nld + n;
          if constexpr (PH == POLY) {
            const half4 h = *reinterpret_cast<const half4*>(A + at), l = *reinterpret_cast<const half4*>(A + an + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = fmaf(NS_C, v[e], NS_B * ((float)h[e] + (float)l[e]));
              if (m == n + e) v[e] += NS_A * SPLIT;
            }
          }
          _Float16* D = PH == GRAM ? A : PH == POLY ? P : p.w + g.x_off[p.dst] + (size_t)mat * 2 * xn;
          const size_t dn = SYM ? an : xn;
          half4 h, l;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
          }
          *reinterpret_cast<half4*>(D + at) = h;
          *reinterpret_cast<half4*>(D + dn + at) = l;
          if constexpr (SYM) {
            if (ti != tj)   // the tile above the diagonal
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const size_t up = (size_t)(n + e) * nld + m;
                D[up] = h[e];
                D[dn + up] = l[e];
              }
          }
        } else {
          const int mt = g.tall ? g.cols : g.rows, ntrue = g.tall ? g.rows : g.cols;
          if (m >= mt) continue;
          float* y = g.y + (size_t)mat * g.stride;
          auto put = [&](size_t at, float o) {
#pragma clang fp contract(off)
            o *= 1.0f / SPLIT;
            if constexpr (PH == LAST_UPDATE) {
              const float w = y[at];
              o = fmaf(-p.lr, fmaf(p.weight_decay, w, g.scale * o), w);
              g.p_bf16[(size_t)mat * g.stride + at] = f2bf(o);
            }
            y[at] = o;
          };
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < ntrue) put(g.tall ? (size_t)(n + e) * g.ld + m : (size_t)m * g.ld + n + e, v[e]);
        }
      }
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
  const long big = tiles(128), small = tiles(64);
  if (small > 0x7fffffffL) return hipErrorInvalidValue;
  if (big >= 256) hipLaunchKernelGGL((ortho_product_kernel<128, 32, PH>), dim3((unsigned)big), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((ortho_product_kernel<64, 64, PH>), dim3((unsigned)small), dim3(256), 0, s, p);
  return hipGetLastError();
}

long align128(long n) { return (n + 127) / 128 * 128; }

}  // namespace

// Offsets of every group's planes (fp16 elements), after the partial sums;
// returns the bytes in all, or 0 when a shape is out of range.
size_t ortho_layout(OrthoGroup* g, int ngroups) {
  long mats = 0;
  for (int k = 0; k < ngroups; ++k) {
    OrthoGroup& q = g[k];
    if (q.rows < 1 || q.cols < 1 || q.count < 1) return 0;
    q.tall = q.rows > q.cols;
    const long m = q.tall ? q.cols : q.rows, n = q.tall ? q.rows : q.cols;
    const long mp = (m + PAD - 1) / PAD * PAD, np = (n + PAD - 1) / PAD * PAD;
    // 32-bit byte offsets within a plane, 32-bit tile and part counts
    if (np > (1L << 30) || mp * np >= (1L << 31) || mp * np / (PAD * PAD) * q.count >= (1L << 31)) return 0;
    q.mp = (int)mp;
    q.np = (int)np;
    mats += q.count;
  }
  if (mats * ORTHO_PARTS >= (1L << 31)) return 0;
  long o = align128(mats * ORTHO_PARTS * (long)(sizeof(double) / 2));
  for (int k = 0; k < ngroups; ++k) {
    OrthoGroup& q = g[k];
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
  Params p{};
  p.ngroups = a.ngroups;
  for (int k = 0; k < a.ngroups; ++k) p.g[k] = a.g[k];
  if (!ortho_layout(p.g, p.ngroups)) return hipErrorInvalidValue;
  unsigned mats = 0, tiles = 0;
  for (int k = 0; k < p.ngroups; ++k) {
    OrthoGroup& q = p.g[k];
    auto ok = [](const void* v) { return (reinterpret_cast<uintptr_t>(v) & 15) == 0; };
    q.vec = q.cols % 4 == 0 && q.ld % 4 == 0 && q.stride % 4 == 0 && ok(q.x) && ok(q.mom);
    mats += q.count;
    tiles += (q.mp / PAD) * (q.np / PAD) * q.count;
  }
  p.w = static_cast<_Float16*>(a.workspace);
  p.parts = static_cast<double*>(a.workspace);
  p.norm_coef = a.norm_coef;
  p.momentum = a.momentum;
  p.nesterov = a.nesterov;
  p.lr = a.lr;
  p.weight_decay = a.weight_decay;
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
