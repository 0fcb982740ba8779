// Attention over packed sequences that share one prefix. Rows of q|k|v are
// tokens: the prefix 0..P-1, then the sequences one after another. Token t sees
// token j <= t of the prefix, and of its own sequence:
//
//   j <= t and (j < P or first[t] <= j),   first[t] = first token of t's sequence
//
// or, from the key's side, j <= t < end[j], end[j] = the token after j's
// sequence (all tokens, for a key of the prefix). The prefix' keys are walked
// once for all sequences: a workgroup's 128 rows are any 128 consecutive rows,
// whatever sequences they belong to, so even sequences of one token fill its
// MFMA tiles, and every key tile it loads serves them all.
//
// Rows of the forward and dQ kernels are (token, query head of a group) pairs,
// token by token, so a group's heads share the loads of its key head too. The
// dK/dV kernel walks the tokens of one query head after another.
//
// Which workgroup walks what is laid down by the host once per layout, in items
// (prefix.cpp): rows and a range of tiles. Long walks are dealt to several
// workgroups where the items are few, with fp32 partial results joined by a
// second launch in a fixed order.
//
// Measured: 16 sequences of 256 over a prefix of 2048, 16 + 8 heads of 128:
// forward 115-130 us (700-790 TFLOP/s), dQ 170-194 (700-790), dK/dV 230-248 + 11
// (750); waves wait on their own chain of products, exponentials and products. 64
// single tokens after 8192: 17 + 5 us, 34 MB of keys and values and 10 MB of
// partial results.
//
// The tile arithmetic is attention.hip's: S^T = K Q^T with one row per lane,
// probabilities handed to the next MFMA from the accumulator registers, where they
// and the score gradients are rounded to bf16 (2^-8 of each at most): products of
// fp32 operands would run at an eighth of the rate. Sums, maxima and the
// log-sum-exp are fp32. Against 64 bits the output is 2.2e-3 and the gradients
// 2.4e-3 off, where rounding only the results leaves 1.7e-3.
#include <type_traits>

#include "attn_tile.h"
#include "common.h"
#include "kernels.h"

namespace {

typedef float float2_t __attribute__((ext_vector_type(2)));

// Item decoding: blocks run through the key/value heads of an item, then the
// next item, so that with 8 of them each keeps to one XCD's L2.
struct Where {
  PrefixItem it;
  int j;   // key/value head
};
DEV Where where(const PrefixArgs& a, const PrefixItem* items) {
  const int b = blockIdx.x;
  Where w;
  w.it = items[b / a.Hkv];
  w.j = b % a.Hkv;
  return w;
}

// One row (token, query head) of the forward and dQ kernels: the lane's own,
// rows past the end taken as the last one.
struct Row {
  int t, rq, h;      // token; its place among the tokens with queries; query head
  int first;         // first key of its own sequence it sees (none in the prefix)
  int t0, t1;        // tokens of the wave's first and last row
  int first0, first1;   // smallest and largest first key among the wave's rows in sequences
  bool on;
};
DEV Row row_of(const PrefixArgs& a, int row, int j, int lane) {
  const int G = a.H / a.Hkv, rows = a.nq * G;
  const int r = min(row + (lane & 31), rows - 1);
  Row o;
  o.on = row + (lane & 31) < rows;
  o.rq = r / G;
  o.h = j * G + r - o.rq * G;
  o.t = a.q0 + o.rq;
  o.first = a.first[o.t];
  o.t0 = __builtin_amdgcn_readfirstlane(o.t);
  o.t1 = __builtin_amdgcn_readlane(o.t, 31);
  o.first0 = o.t0 >= a.P ? __builtin_amdgcn_readfirstlane(o.first) : a.P;
  o.first1 = __builtin_amdgcn_readlane(o.first, 31);
  return o;
}

// What a wave's rows see of the tile of 64 keys at kv0.
enum Sight { NONE, SOME, ALL };
DEV Sight sight(const PrefixArgs& a, const Row& r, int kv0, bool own) {
  if (!own) return kv0 > r.t1 ? NONE : kv0 + TILE - 1 <= min(r.t0, a.P - 1) ? ALL : SOME;
  if (r.t1 < a.P || kv0 > r.t1 || kv0 + TILE - 1 < r.first0) return NONE;
  return r.t0 >= a.P && kv0 >= r.first1 && kv0 + TILE - 1 <= r.t0 ? ALL : SOME;
}

// Keys lo..hi of the segment that a lane's row sees.
DEV void seen(const PrefixArgs& a, const Row& r, bool own, int& lo, int& hi) {
  lo = own ? (r.t >= a.P ? r.first : r.t + 1) : 0;
  hi = own ? r.t : min(r.t, a.P - 1);
}

// Key and value tiles of an item's walk, double-buffered: tile f < it.npre is
// keys 64 f.. of the prefix, the others follow from it.own on.
template <int HD>
struct KeyWalk {
  using S = Shape<HD>;
  v4i32 rs;
  uint32_t koff, voff;
  int ld, npre, own;
  DEV void init(const PrefixArgs& a, const Where& w) {
    ld = (a.H + 2 * a.Hkv) * HD;
    rs = make_rsrc(a.qkv, (uint32_t)((size_t)a.N * ld * 2));
    koff = (uint32_t)((a.H + w.j) * HD * 2);
    voff = koff + (uint32_t)(a.Hkv * HD * 2);
    npre = w.it.npre;
    own = w.it.own;
  }
  DEV bool is_own(int f) const { return f >= npre; }
  DEV int key0(int f) const { return f < npre ? f * TILE : own + (f - npre) * TILE; }
  DEV void issue(int f, lds_char_t* st, int wave, int lane) const {
    constexpr int U = HD / 8, INSTR = TILE * U / 64;
    const uint32_t r0 = (uint32_t)key0(f);
#pragma unroll
    for (int i = 0; i < INSTR / 4; ++i) {
      const int ins = wave + 4 * i, u = ins * 64 + lane;
      const int row = u / U, c = unit<HD>(row, u % U) - row * U;   // the XOR is its own inverse
      const uint32_t off = ((r0 + (uint32_t)row) * (uint32_t)ld + (uint32_t)(c * 8)) * 2u;
      dma16(rs, koff + off, lds_addr(st + ins * 1024));
      dma16(rs, voff + off, lds_addr(st + S::TBA + ins * 1024));
    }
  }
};

DEV size_t part_at(const PrefixArgs& a, int slot, int j, size_t floats) {
  return ((size_t)slot * a.Hkv + j) * floats;
}
constexpr size_t fwd_part(int hd) { return (size_t)BQ * (hd + 2); }    // O [128][hd], max [128], sum [128]
constexpr size_t dq_part(int hd) { return (size_t)BQ * hd; }
constexpr size_t dkdv_part(int hd) { return (size_t)2 * BQ * hd; }     // dK, dV [128][hd]

// Where items are too few for two workgroups a CU, GR groups of four waves walk
// the item's tiles in turn and merge what they have at the end: a walk's time is
// one wave's chain of products and exponentials, tile after tile.
template <int HD, int GR>
__global__ __launch_bounds__(256 * GR, GR == 1 ? 2 : 1) void prefix_fwd_kernel(PrefixArgs a) {
  using S = Shape<HD>;
  constexpr int GROUP = 2 * 2 * S::TBA;   // 2 stages x (K, V)
  constexpr int KEEP = S::DT * 4096 + 512;   // a wave's O, maxima and sums
  static_assert(4 * (GR - 1) * KEEP <= GR * GROUP, "the groups' results fit their tiles' space");
  __shared__ __attribute__((aligned(1024))) char smem_raw[GR * GROUP];
  const int tid = threadIdx.x, lane = tid & 63, all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = all & 3, group = all >> 2;
  lds_char_t* smem = (lds_char_t*)smem_raw + group * GROUP;
  const int lq = lane & 31, g = lane >> 5;
  const Where w = where(a, a.items);
  KeyWalk<HD> keys;
  keys.init(a, w);
  auto stage = [&](int f) { return smem + (f - w.it.f0) / GR % 2 * 2 * S::TBA; };
  // under way while the rows are read
  if (w.it.f0 + group < w.it.f1) keys.issue(w.it.f0 + group, stage(w.it.f0 + group), wave, lane);
  const Row r = row_of(a, w.it.row + 32 * wave, w.j, lane);

  bf16x8 qf[S::KS];
  const bf16_t* q = a.qkv + (size_t)r.t * keys.ld + r.h * HD;
#pragma unroll
  for (int s = 0; s < S::KS; ++s) qf[s] = as_bf16x8(*reinterpret_cast<const uint4*>(q + 16 * s + 8 * g));
  floatx16 o[S::DT];
#pragma unroll
  for (int d = 0; d < S::DT; ++d) zero(o[d]);
  float m_run = -INFINITY, l_run = 0.0f;
  const float sc = LOG2E / sqrtf((float)HD);

  for (int f0 = w.it.f0; f0 < w.it.f1; f0 += GR) {
    const int f = f0 + group;
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
    block_barrier();
    if (f + GR < w.it.f1) keys.issue(f + GR, stage(f + GR), wave, lane);
    if (f >= w.it.f1) continue;
    const int kv0 = keys.key0(f);
    const bool own = keys.is_own(f);
    const Sight see = sight(a, r, kv0, own);
    if (see == NONE) continue;
    const lds_char_t* Ks = stage(f);
    const lds_char_t* Vs = Ks + S::TBA;

    floatx16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      zero(s[t]);
#pragma unroll
      for (int k = 0; k < S::KS; ++k) s[t] = mfma32(read_row<HD>(Ks, 32 * t + lq, 2 * k + g), qf[k], s[t]);
    }
    float mt = -INFINITY;
    auto mask_max = [&](auto masked) {
      int lo, hi;
      seen(a, r, own, lo, hi);
      lo -= kv0 + 4 * g;
      hi -= kv0 + 4 * g;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = s[t][e];
          const int k = 32 * t + acc_row(e, 0);
          if constexpr (decltype(masked)::value) x = k >= lo && k <= hi ? x : -INFINITY;
          s[t][e] = x;
          mt = fmaxf(mt, x);
        }
    };
    if (see == SOME) mask_max(std::true_type{});
    else mask_max(std::false_type{});
    mt = max32(mt) * sc;
    const bool grow = mt > m_run + RESCALE_SLACK;
    if (__ballot(grow) != 0) {
      const float alpha = grow ? fast_exp2(m_run - mt) : 1.0f;
      m_run = grow ? mt : m_run;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
    }
    // a row that has seen nothing yet (its keys come later) has no maximum
    const float shift = m_run == -INFINITY ? 0.0f : m_run;
    float rsum = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = fast_exp2(fmaf(s[t][e], sc, -shift));
        s[t][e] = p;
        rsum += p;
      }
    l_run += sum32(rsum);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const bf16x8 pf = acc_slots(s[t], hh);
#pragma unroll
        for (int d = 0; d < S::DT; ++d) o[d] = mfma32(read_tr<HD>(Vs, 32 * d, 32 * t + 16 * hh, lane), pf, o[d]);
      }
  }

  if constexpr (GR > 1) {
    // the other groups' results through LDS, joined in order
    __syncthreads();
    lds_char_t* keep = (lds_char_t*)smem_raw + ((group - 1) * 4 + wave) * KEEP + lane * 16;
    if (group > 0) {
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<lds_v4f32_t*>(keep + (d * 4 + c) * 1024) =
              v4f32{o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]};
      *reinterpret_cast<LDS_AS float2_t*>(keep + S::DT * 4096 - lane * 8) = float2_t{m_run, l_run};
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < GR - 1; ++k) {
      const lds_char_t* from = keep + (k + 1) * 4 * KEEP;
      const float2_t ml = *reinterpret_cast<const LDS_AS float2_t*>(from + S::DT * 4096 - lane * 8);
      const float m = fmaxf(m_run, ml.x);
      const float f0 = m_run == -INFINITY ? 0.0f : fast_exp2(m_run - m), f1 = ml.x == -INFINITY ? 0.0f : fast_exp2(ml.x - m);
      m_run = m;
      l_run = l_run * f0 + ml.y * f1;
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const v4f32 x = *reinterpret_cast<const lds_v4f32_t*>(from + (d * 4 + c) * 1024);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * c + e] = o[d][4 * c + e] * f0 + x[e] * f1;
        }
    }
  }
  if (!r.on) return;
  if (w.it.slot >= 0) {
    float* part = a.part + part_at(a, w.it.slot, w.j, fwd_part(HD));
    const int row = 32 * wave + lq;
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(part + (size_t)row * HD + 32 * d + 8 * c + 4 * g) =
            make_float4(o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]);
    if (g == 0) {
      part[(size_t)BQ * HD + row] = m_run;
      part[(size_t)BQ * HD + BQ + row] = l_run;
    }
    return;
  }
  const float inv = 1.0f / l_run;
  bf16_t* out = a.out + ((size_t)r.rq * a.H + r.h) * HD;
#pragma unroll
  for (int d = 0; d < S::DT; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<uint2*>(out + 32 * d + 8 * c + 4 * g) =
          make_uint2(pack2(o[d][4 * c] * inv, o[d][4 * c + 1] * inv),
                     pack2(o[d][4 * c + 2] * inv, o[d][4 * c + 3] * inv));
  if (g == 0) a.lse[(size_t)r.h * a.nq + r.rq] = (m_run + log2f(l_run)) * LN2;
}

// The parts of a row merged, a wave a row: lane k first holds part k's maximum
// and sum (the maximum's weight afterwards), then HD/8 lanes take the row's
// elements, 8 each, and the groups of them the parts in turn.
template <int HD>
__global__ __launch_bounds__(256) void prefix_fwd_join_kernel(PrefixArgs a) {
  constexpr int LANES = HD / 8, GROUPS = 64 / LANES;
  const int lane = threadIdx.x & 63;
  const int b = blockIdx.x, j = b % a.Hkv;
  const PrefixJoin jn = a.joins[b / a.Hkv];
  const int G = a.H / a.Hkv, row = blockIdx.y * 4 + (threadIdx.x >> 6), c = lane % LANES * 8;
  const int rr = jn.row + row;
  if (rr >= a.nq * G) return;
  const float* part0 = a.part + part_at(a, jn.slot, j, fwd_part(HD));
  const size_t step = (size_t)a.Hkv * fwd_part(HD);
  float m = -INFINITY;
  for (int k = lane; k < jn.parts; k += 64) m = fmaxf(m, part0[k * step + (size_t)BQ * HD + row]);
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.0f, o[8] = {};
  for (int k0 = 0; k0 < jn.parts; k0 += 64) {
    float wgt = 0.0f;
    if (k0 + lane < jn.parts) {
      const float* p = part0 + (k0 + lane) * step + (size_t)BQ * HD;
      wgt = fast_exp2(p[row] - m);
      l += wgt * p[BQ + row];
    }
    const int n = min(64, jn.parts - k0);
#pragma unroll 4
    for (int k = 0; k < n; k += GROUPS) {
      const int q = k + lane / LANES;
      const float f = __shfl(wgt, min(q, 63));
      if (q < n) {
        const float* p = part0 + (k0 + q) * step + (size_t)row * HD + c;
        const float4 x = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
        o[0] += f * x.x; o[1] += f * x.y; o[2] += f * x.z; o[3] += f * x.w;
        o[4] += f * y.x; o[5] += f * y.y; o[6] += f * y.z; o[7] += f * y.w;
      }
    }
  }
  l = wave_sum(l);
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int s = LANES; s < 64; s <<= 1) o[e] += __shfl_xor(o[e], s);
  if (lane >= LANES) return;
  const float inv = 1.0f / l;
  const int rq = rr / G, h = j * G + rr - rq * G;
  *reinterpret_cast<uint4*>(a.out + ((size_t)rq * a.H + h) * HD + c) =
      make_uint4(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv), pack2(o[4] * inv, o[5] * inv),
                 pack2(o[6] * inv, o[7] * inv));
  if (c == 0) a.lse[(size_t)h * a.nq + rq] = (m + log2f(l)) * LN2;
}

// ... a row's HD/8 lanes taking its parts one after another, where rows are
// many and parts few.
template <int HD>
__global__ __launch_bounds__(256) void prefix_fwd_join_few_kernel(PrefixArgs a) {
  constexpr int LANES = HD / 8, ROWS = 256 / LANES;
  const int b = blockIdx.x, j = b % a.Hkv;
  const PrefixJoin jn = a.joins[b / a.Hkv];
  const int G = a.H / a.Hkv, row = blockIdx.y * ROWS + threadIdx.x / LANES, c = threadIdx.x % LANES * 8;
  const int rr = jn.row + row;
  if (rr >= a.nq * G) return;
  const float* part0 = a.part + part_at(a, jn.slot, j, fwd_part(HD));
  const size_t step = (size_t)a.Hkv * fwd_part(HD);
  float m = -INFINITY;
#pragma unroll 4
  for (int k = 0; k < jn.parts; ++k) m = fmaxf(m, part0[k * step + (size_t)BQ * HD + row]);
  float l = 0.0f, o[8] = {};
#pragma unroll 4
  for (int k = 0; k < jn.parts; ++k) {
    const float* p = part0 + k * step;
    const float f = fast_exp2(p[(size_t)BQ * HD + row] - m);
    const float4 x = *reinterpret_cast<const float4*>(p + (size_t)row * HD + c);
    const float4 y = *reinterpret_cast<const float4*>(p + (size_t)row * HD + c + 4);
    l += f * p[(size_t)BQ * HD + BQ + row];
    o[0] += f * x.x; o[1] += f * x.y; o[2] += f * x.z; o[3] += f * x.w;
    o[4] += f * y.x; o[5] += f * y.y; o[6] += f * y.z; o[7] += f * y.w;
  }
  const float inv = 1.0f / l;
  const int rq = rr / G, h = j * G + rr - rq * G;
  *reinterpret_cast<uint4*>(a.out + ((size_t)rq * a.H + h) * HD + c) =
      make_uint4(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv), pack2(o[4] * inv, o[5] * inv),
                 pack2(o[6] * inv, o[7] * inv));
  if (c == 0) a.lse[(size_t)h * a.nq + rq] = (m + log2f(l)) * LN2;
}

// The zero gradient of queries that a prefix does not have.
template <int HD>
__global__ __launch_bounds__(256) void prefix_zero_kernel(PrefixArgs a) {
  const int lanes = a.H * (HD / 8);
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const int t = (int)(i / lanes), c = (int)(i - (long)t * lanes) * 8;
  if (t < a.q0) *reinterpret_cast<uint4*>(a.dqkv + (size_t)t * (a.H + 2 * a.Hkv) * HD + c) = make_uint4(0, 0, 0, 0);
}

// D = rowsum(dO * O) from the bf16 O is off by a rounding that all keys of the
// row share. Beside the roundings of dS, which average, that counts the more the
// fewer keys hold the row's weight, so rows of few keys take a first walk that
// sums D = sum_j P_j dP_j in fp32: gradients of 9 ragged answers with 64-wide
// heads are 2.4e-3 off instead of 2.6e-3, of rows of up to 70 keys 2.4e-3
// instead of 2.8e-3 (rounding exact ones 1.7e-3); dQ of the former takes 18 us
// instead of 14. Longer walks would pay two products more of five for a
// difference of a few per cent.
constexpr int EXACT_TILES = 8;

// That sum over the whole walk of the item's rows, tiles dealt out among the
// groups as below; the walk's first tiles are under way in the first stages.
template <int HD, int GR>
DEV float walk_d(const PrefixArgs& a, const KeyWalk<HD>& keys, const Row& r, int tiles, const bf16x8 (&qf)[HD / 16],
                 const bf16x8 (&df)[HD / 16], float sc, float lse2, lds_char_t* all_groups, int wave, int group,
                 int lane) {
  using S = Shape<HD>;
  constexpr int GROUP = 2 * 2 * S::TBA;
  lds_char_t* smem = all_groups + group * GROUP;
  const int lq = lane & 31, g = lane >> 5;
  float sum = 0.0f;
  for (int f0 = 0; f0 < tiles; f0 += GR) {
    const int f = f0 + group;
    lds_char_t* Ks = smem + f0 / GR % 2 * 2 * S::TBA;
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
    block_barrier();
    if (f + GR < tiles) keys.issue(f + GR, smem + (f0 / GR + 1) % 2 * 2 * S::TBA, wave, lane);
    if (f >= tiles) continue;
    const int kv0 = keys.key0(f);
    const bool own = keys.is_own(f);
    if (sight(a, r, kv0, own) == NONE) continue;
    int lo, hi;
    seen(a, r, own, lo, hi);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx16 p, dp;
      zero(p);
      zero(dp);
#pragma unroll
      for (int k = 0; k < S::KS; ++k) {
        p = mfma32(read_row<HD>(Ks, 32 * t + lq, 2 * k + g), qf[k], p);
        dp = mfma32(read_row<HD>(Ks + S::TBA, 32 * t + lq, 2 * k + g), df[k], dp);
      }
      const int k0 = kv0 + 32 * t + 4 * g;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = fast_exp2(p[e] * sc - lse2) * dp[e];
        sum += k0 + acc_row(e, 0) >= lo && k0 + acc_row(e, 0) <= hi ? x : 0.0f;
      }
    }
  }
  sum = sum32(sum);
  // the groups' sums, in order; the stages are free for the walk that follows
  __syncthreads();
  if constexpr (GR > 1) {
    LDS_AS float* part = (LDS_AS float*)all_groups;
    if (lane < 32) part[(group * 4 + wave) * 32 + lq] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < GR; ++k) sum += part[(k * 4 + wave) * 32 + lq];
    __syncthreads();
  }
  return sum;
}

// dQ of 128 rows, walking the forward's tiles: dS = P (dO V^T - D), dQ = dS K.
template <int HD, int GR>
__global__ __launch_bounds__(256 * GR, GR == 1 ? 2 : 1) void prefix_dq_kernel(PrefixArgs a) {
  using S = Shape<HD>;
  constexpr int GROUP = 2 * 2 * S::TBA, KEEP = S::DT * 4096;   // as the forward's
  static_assert(4 * (GR - 1) * KEEP <= GR * GROUP, "the groups' results fit their tiles' space");
  __shared__ __attribute__((aligned(1024))) char smem_raw[GR * GROUP];
  const int tid = threadIdx.x, lane = tid & 63, all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = all & 3, group = all >> 2;
  lds_char_t* smem = (lds_char_t*)smem_raw + group * GROUP;
  const int lq = lane & 31, g = lane >> 5;
  const Where w = where(a, a.items);
  KeyWalk<HD> keys;
  keys.init(a, w);
  auto stage = [&](int f) { return smem + (f - w.it.f0) / GR % 2 * 2 * S::TBA; };
  // under way while the rows are read
  const bool exact = w.it.tiles <= EXACT_TILES;
  const int from = exact ? 0 : w.it.f0, to = exact ? w.it.tiles : w.it.f1;
  if (from + group < to) keys.issue(from + group, smem, wave, lane);
  const Row r = row_of(a, w.it.row + 32 * wave, w.j, lane);

  bf16x8 qf[S::KS], df[S::KS];
  const bf16_t* q = a.qkv + (size_t)r.t * keys.ld + r.h * HD;
  const bf16_t* dout = a.dout + ((size_t)r.rq * a.H + r.h) * HD;
#pragma unroll
  for (int s = 0; s < S::KS; ++s) {
    qf[s] = as_bf16x8(*reinterpret_cast<const uint4*>(q + 16 * s + 8 * g));
    df[s] = as_bf16x8(*reinterpret_cast<const uint4*>(dout + 16 * s + 8 * g));
  }
  const size_t d_at = (size_t)r.h * a.nq + r.rq;
  const float lse2 = a.lse[d_at] * LOG2E;
  const float scale = 1.0f / sqrtf((float)HD);
  const float sc = scale * LOG2E;
  float dsum;
  if (exact) {
    dsum = walk_d<HD, GR>(a, keys, r, w.it.tiles, qf, df, sc, lse2, (lds_char_t*)smem_raw, wave, group, lane);
    if (w.it.f0 + group < w.it.f1) keys.issue(w.it.f0 + group, smem, wave, lane);
  } else {
    const bf16_t* out = a.out + ((size_t)r.rq * a.H + r.h) * HD;
    dsum = 0.0f;
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      const uint4 o = *reinterpret_cast<const uint4*>(out + 16 * s + 8 * g), d = __builtin_bit_cast(uint4, df[s]);
      dsum += lo_f(d.x) * lo_f(o.x) + hi_f(d.x) * hi_f(o.x) + lo_f(d.y) * lo_f(o.y) + hi_f(d.y) * hi_f(o.y);
      dsum += lo_f(d.z) * lo_f(o.z) + hi_f(d.z) * hi_f(o.z) + lo_f(d.w) * lo_f(o.w) + hi_f(d.w) * hi_f(o.w);
    }
    dsum = sum32(dsum);
  }
  if (w.it.f0 == 0 && group == 0 && r.on && g == 0) a.dsum[d_at] = dsum;   // for dK/dV
  floatx16 dq[S::DT];
#pragma unroll
  for (int d = 0; d < S::DT; ++d) zero(dq[d]);

  for (int f0 = w.it.f0; f0 < w.it.f1; f0 += GR) {
    const int f = f0 + group;
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
    block_barrier();
    if (f + GR < w.it.f1) keys.issue(f + GR, stage(f + GR), wave, lane);
    if (f >= w.it.f1) continue;
    const int kv0 = keys.key0(f);
    const bool own = keys.is_own(f);
    const Sight see = sight(a, r, kv0, own);
    if (see == NONE) continue;
    const lds_char_t* Ks = stage(f);
    const lds_char_t* Vs = Ks + S::TBA;

    floatx16 ds[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx16 p;
      zero(p);
      zero(ds[t]);
#pragma unroll
      for (int k = 0; k < S::KS; ++k) {
        p = mfma32(read_row<HD>(Ks, 32 * t + lq, 2 * k + g), qf[k], p);
        ds[t] = mfma32(read_row<HD>(Vs, 32 * t + lq, 2 * k + g), df[k], ds[t]);
      }
      auto probs = [&](auto masked) {
        int lo = 0, hi = 0;
        if constexpr (decltype(masked)::value) {
          seen(a, r, own, lo, hi);
          lo -= kv0 + 32 * t + 4 * g;
          hi -= kv0 + 32 * t + 4 * g;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = fast_exp2(p[e] * sc - lse2) * (ds[t][e] - dsum);
          // the product goes, not a factor: dO V of a key that is not seen may be infinite
          if constexpr (decltype(masked)::value) x = acc_row(e, 0) >= lo && acc_row(e, 0) <= hi ? x : 0.0f;
          ds[t][e] = x;
        }
      };
      if (see == SOME) probs(std::true_type{});
      else probs(std::false_type{});
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const bf16x8 sf = acc_slots(ds[t], hh);
#pragma unroll
        for (int d = 0; d < S::DT; ++d) dq[d] = mfma32(read_tr<HD>(Ks, 32 * d, 32 * t + 16 * hh, lane), sf, dq[d]);
      }
  }

  if constexpr (GR > 1) {
    __syncthreads();
    lds_char_t* keep = (lds_char_t*)smem_raw + ((group - 1) * 4 + wave) * KEEP + lane * 16;
    if (group > 0) {
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<lds_v4f32_t*>(keep + (d * 4 + c) * 1024) =
              v4f32{dq[d][4 * c], dq[d][4 * c + 1], dq[d][4 * c + 2], dq[d][4 * c + 3]};
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 1; k < GR; ++k)
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const v4f32 x = *reinterpret_cast<const lds_v4f32_t*>(keep + k * 4 * KEEP + (d * 4 + c) * 1024);
#pragma unroll
          for (int e = 0; e < 4; ++e) dq[d][4 * c + e] += x[e];
        }
  }
  if (!r.on) return;
  if (w.it.slot >= 0) {
    float* part = a.part + part_at(a, w.it.slot, w.j, dq_part(HD)) + (size_t)(32 * wave + lq) * HD;
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(part + 32 * d + 8 * c + 4 * g) =
            make_float4(dq[d][4 * c], dq[d][4 * c + 1], dq[d][4 * c + 2], dq[d][4 * c + 3]);
    return;
  }
  bf16_t* dst = a.dqkv + (size_t)r.t * keys.ld + r.h * HD;
#pragma unroll
  for (int d = 0; d < S::DT; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<uint2*>(dst + 32 * d + 8 * c + 4 * g) =
          make_uint2(pack2(dq[d][4 * c] * scale, dq[d][4 * c + 1] * scale),
                     pack2(dq[d][4 * c + 2] * scale, dq[d][4 * c + 3] * scale));
}

// The parts of 128 rows added up: dQ rows (token, head of the group), or dK and
// dV rows of a key/value head.
template <int HD, bool KEYS>
__global__ __launch_bounds__(256) void prefix_sum_join_kernel(PrefixArgs a) {
  constexpr int LANES = HD / 8, ROWS = 256 / LANES;
  constexpr size_t PART = KEYS ? dkdv_part(HD) : dq_part(HD);
  const int b = blockIdx.x, j = b % a.Hkv, ld = (a.H + 2 * a.Hkv) * HD;
  const PrefixJoin jn = (KEYS ? a.kjoins : a.joins)[b / a.Hkv];
  const int G = a.H / a.Hkv, c = threadIdx.x % LANES * 8;
  const int row = blockIdx.y * ROWS + threadIdx.x / LANES;   // dV's rows follow dK's
  const bool is_v = KEYS && row >= BQ;
  const int rr = jn.row + (is_v ? row - BQ : row);
  if (rr >= (KEYS ? (jn.row < a.P ? a.P : a.N) : a.nq * G)) return;
  float o[8] = {};
#pragma unroll 4
  for (int k = 0; k < jn.parts; ++k) {
    const float* part = a.part + part_at(a, jn.slot + k, j, PART) + (size_t)row * HD + c;
    const float4 x = *reinterpret_cast<const float4*>(part), y = *reinterpret_cast<const float4*>(part + 4);
    o[0] += x.x; o[1] += x.y; o[2] += x.z; o[3] += x.w;
    o[4] += y.x; o[5] += y.y; o[6] += y.z; o[7] += y.w;
  }
  const float f = is_v ? 1.0f : 1.0f / sqrtf((float)HD);
  const int rq = rr / G;
  const size_t at = KEYS ? (size_t)rr * ld + (a.H + j + (is_v ? a.Hkv : 0)) * HD
                         : (size_t)(a.q0 + rq) * ld + (j * G + rr - rq * G) * HD;
  *reinterpret_cast<uint4*>(a.dqkv + at + c) =
      make_uint4(pack2(o[0] * f, o[1] * f), pack2(o[2] * f, o[3] * f), pack2(o[4] * f, o[5] * f),
                 pack2(o[6] * f, o[7] * f));
}

// dK, dV of 128 keys with eight waves, as attention.hip's: wave w owns keys
// 32 (w % 4)..+31 and the query half w / 4 of every tile of 64 queries; the
// keys' rows stay in LDS. Query tile f of the walk is tile f % nt of the tokens
// it.t0..it.t1-1, head f / nt of the group.
template <int HD>
__global__ __launch_bounds__(512, 1) void prefix_dkdv_kernel(PrefixArgs a) {
  using S = Shape<HD>;
  constexpr int KVB = BQ * HD * 2;             // one 128-row block of K or V
  constexpr int STAGE = 2 * S::TBA + 1024;     // Q tile, dO tile, lse and D rows
  constexpr int SMEM_T = 2 * KVB + 2 * STAGE;
  constexpr int NACC = 2 * S::DT * 16;         // dK and dV registers per lane
  constexpr int SMEM = SMEM_T > 4 * NACC * 64 * 4 ? SMEM_T : 4 * NACC * 64 * 4;
  __shared__ __attribute__((aligned(1024))) char smem_raw[SMEM];
  lds_char_t* smem = (lds_char_t*)smem_raw;
  lds_char_t* Ks = smem;
  lds_char_t* Vs = smem + KVB;
  lds_char_t* stages = smem + 2 * KVB;
  const Where w = where(a, a.kitems);
  const int H = a.H, C = H * HD, Hkv = a.Hkv, ld = (H + 2 * Hkv) * HD, G = H / Hkv, j = w.j;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave & 3, th = wave >> 2;   // key group, query half
  const int lk = lane & 31, g = lane >> 5;
  const int k0 = w.it.row, kend = k0 < a.P ? a.P : a.N;
  const int kv0w = k0 + kw * 32, kv = kv0w + lk;
  // queries kv..end-1 see key kv
  const int end = a.end[min(kv, kend - 1)];
  const int end0 = __builtin_amdgcn_readfirstlane(end), end1 = __builtin_amdgcn_readlane(end, 31);
  const v4i32 rq = make_rsrc(a.qkv, (uint32_t)((size_t)a.N * ld * 2));
  const v4i32 rd = make_rsrc(a.dout, (uint32_t)((size_t)a.nq * C * 2));
  const v4i32 rl = make_rsrc(a.lse, (uint32_t)((size_t)H * a.nq * 4));
  const v4i32 rD = make_rsrc(a.dsum, (uint32_t)((size_t)H * a.nq * 4));

  floatx16 dk[S::DT], dv[S::DT];
#pragma unroll
  for (int d = 0; d < S::DT; ++d) {
    zero(dk[d]);
    zero(dv[d]);
  }
  const float scale = 1.0f / sqrtf((float)HD);
  const float sc = scale * LOG2E;
  const int nt = (w.it.t1 - w.it.t0 + TILE - 1) / TILE;
  auto issue = [&](int f) {
    lds_char_t* st = stages + ((f - w.it.f0) & 1) * STAGE;
    const int gi = f / nt, h = j * G + gi;
    const int t = w.it.t0 + (f - gi * nt) * TILE, rt = t - a.q0;
    issue_rows8<HD>(rq, (uint32_t)(h * HD) * 2u, t, ld, st, wave, lane);
    issue_rows8<HD>(rd, (uint32_t)(h * HD) * 2u, rt, C, st + S::TBA, wave, lane);
    // the tile's 64 log-sum-exp and D values (256 bytes each): 16 lanes
    if (wave == 0 && lane < 16) {
      const uint32_t off = ((uint32_t)h * (uint32_t)a.nq + (uint32_t)rt) * 4u + 16u * lane;
      dma16(rl, off, lds_addr(st + 2 * S::TBA));
      dma16(rD, off, lds_addr(st + 2 * S::TBA + 256));
    }
  };
  if (w.it.f0 < w.it.f1) {
    const uint32_t koff = (uint32_t)((H + j) * HD) * 2u, voff = koff + (uint32_t)(Hkv * HD) * 2u;
    issue_rows8<HD>(rq, koff, k0, ld, Ks, wave, lane);
    issue_rows8<HD>(rq, koff, k0 + TILE, ld, Ks + S::TB, wave, lane);
    issue_rows8<HD>(rq, voff, k0, ld, Vs, wave, lane);
    issue_rows8<HD>(rq, voff, k0 + TILE, ld, Vs + S::TB, wave, lane);
    issue(w.it.f0);
  }
  for (int f = w.it.f0; f < w.it.f1; ++f) {
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
    block_barrier();
    if (f + 1 < w.it.f1) issue(f + 1);
    const int qh0 = w.it.t0 + f % nt * TILE + 32 * th;   // this wave's first query
    if (qh0 + 31 < kv0w || qh0 >= end1) continue;   // none of its queries sees its keys
    const lds_char_t* Qs = stages + ((f - w.it.f0) & 1) * STAGE;
    const lds_char_t* Ds = Qs + S::TBA;
    const lds_char_t* lr = Qs + 2 * S::TBA;   // lse [64] then D [64], fp32
    const bool some = qh0 < kv0w + 31 || qh0 + 32 > end0 || kv0w + 32 > kend;

    floatx16 p, ds;
    zero(p);
    zero(ds);
#pragma unroll
    for (int k = 0; k < S::KS; ++k) {
      p = mfma32(read_row<HD>(Qs, 32 * th + lk, 2 * k + g), read_row<HD>(Ks, 32 * kw + lk, 2 * k + g), p);
      ds = mfma32(read_row<HD>(Ds, 32 * th + lk, 2 * k + g), read_row<HD>(Vs, 32 * kw + lk, 2 * k + g), ds);
    }
    auto probs = [&](auto masked) {
#pragma unroll
      for (int c4 = 0; c4 < 4; ++c4) {
        const int qi = 8 * c4 + 4 * g;   // 4 consecutive queries of the half
        const v4f32 l4 = *reinterpret_cast<const lds_v4f32_t*>(lr + 4 * (32 * th + qi));
        const v4f32 d4 = *reinterpret_cast<const lds_v4f32_t*>(lr + 256 + 4 * (32 * th + qi));
        const int qlo = kv - qh0 - qi, qhi = (kv < kend ? end : 0) - qh0 - qi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * c4 + e;
          float pv = fast_exp2(p[i] * sc - l4[e] * LOG2E);
          float dd = ds[i] - d4[e];
          if constexpr (decltype(masked)::value) {
            // rows past the last query hold no log-sum-exp or D of this head: both factors go
            const bool in = e >= qlo && e < qhi;
            pv = in ? pv : 0.0f;
            dd = in ? dd : 0.0f;
          }
          p[i] = pv;
          ds[i] = pv * dd;
        }
      }
    };
    if (some) probs(std::true_type{});
    else probs(std::false_type{});
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const bf16x8 pf = acc_slots(p, hh), sf = acc_slots(ds, hh);
#pragma unroll
      for (int d = 0; d < S::DT; ++d) {
        dv[d] = mfma32(read_tr<HD>(Ds, 32 * d, 32 * th + 16 * hh, lane), pf, dv[d]);
        dk[d] = mfma32(read_tr<HD>(Qs, 32 * d, 32 * th + 16 * hh, lane), sf, dk[d]);
      }
    }
  }

  // the second query half's waves hand their partial sums to the first's
  __syncthreads();
  lds_v4f32_t* red = (lds_v4f32_t*)smem_raw + kw * (NACC / 4) * 64 + lane;
  if (th == 1) {
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        red[((2 * d) * 4 + c) * 64] = v4f32{dk[d][4 * c], dk[d][4 * c + 1], dk[d][4 * c + 2], dk[d][4 * c + 3]};
        red[((2 * d + 1) * 4 + c) * 64] = v4f32{dv[d][4 * c], dv[d][4 * c + 1], dv[d][4 * c + 2], dv[d][4 * c + 3]};
      }
  }
  __syncthreads();
  if (th == 1 || kv >= kend) return;
  bf16_t* dst = a.dqkv + (size_t)kv * ld + (H + j) * HD;
  float* part = w.it.slot >= 0 ? a.part + part_at(a, w.it.slot, j, dkdv_part(HD)) + (size_t)(32 * kw + lk) * HD : nullptr;
#pragma unroll
  for (int d = 0; d < S::DT; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const v4f32 ok = red[((2 * d) * 4 + c) * 64], ov = red[((2 * d + 1) * 4 + c) * 64];
      const int dd = 32 * d + 8 * c + 4 * g;
      const float4 k4 = make_float4(dk[d][4 * c] + ok.x, dk[d][4 * c + 1] + ok.y, dk[d][4 * c + 2] + ok.z,
                                    dk[d][4 * c + 3] + ok.w);
      const float4 v4 = make_float4(dv[d][4 * c] + ov.x, dv[d][4 * c + 1] + ov.y, dv[d][4 * c + 2] + ov.z,
                                    dv[d][4 * c + 3] + ov.w);
      if (part) {
        *reinterpret_cast<float4*>(part + dd) = k4;
        *reinterpret_cast<float4*>(part + (size_t)BQ * HD + dd) = v4;
      } else {
        *reinterpret_cast<uint2*>(dst + dd) =
            make_uint2(pack2(k4.x * scale, k4.y * scale), pack2(k4.z * scale, k4.w * scale));
        *reinterpret_cast<uint2*>(dst + Hkv * HD + dd) = make_uint2(pack2(v4.x, v4.y), pack2(v4.z, v4.w));
      }
    }
}

template <int HD>
hipError_t fwd_t(const PrefixArgs& a, hipStream_t s) {
  const unsigned wgs = a.nitems * a.Hkv;
  // One workgroup a CU: groups of waves share its walk, as many as the registers
  // allow (one walk of 129 tiles for each of 8 heads of 128: 187 us with one
  // group, 117 with two). With more workgroups than CUs two of one group share
  // a CU instead.
  constexpr int GR = HD == 64 ? 4 : 2;
  if (wgs <= 256) hipLaunchKernelGGL((prefix_fwd_kernel<HD, GR>), dim3(wgs), dim3(256 * GR), 0, s, a);
  else hipLaunchKernelGGL((prefix_fwd_kernel<HD, 1>), dim3(wgs), dim3(256), 0, s, a);
  if (!a.njoins) return hipGetLastError();
  const unsigned joins = a.njoins * a.Hkv;
  // Many parts: a wave a row (64 tokens after 8,192, 19 parts: 5-7 us, a few
  // lanes a row 15). Few: a few lanes a row (12 answers after 1,500, walks in a few
  // parts: 7.5 us, a wave a row 11.4). Where both counts are high the two are
  // close or a few lanes ahead: 12 of 75 tokens after 1,500 in items of three
  // tiles, nine parts, forward and join 64.6 and 66.0 us at head size 128, 30.7
  // and 35.5 at 64; in single tokens' items of 7 to 26 tiles (19 to 5 parts) 23.0
  // and 20.7 (7), 23.8 and 21.8 (9), 22.8 and 22.7 (11), 33.3 and 33.8 (26).
  if (a.parts > 8) hipLaunchKernelGGL(prefix_fwd_join_kernel<HD>, dim3(joins, BQ / 4), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(prefix_fwd_join_few_kernel<HD>, dim3(joins, BQ * HD / 2048), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int HD>
hipError_t bwd_t(const PrefixArgs& a, hipStream_t s) {
  const long zeros = (long)a.q0 * a.H * (HD / 8);
  if (zeros) hipLaunchKernelGGL(prefix_zero_kernel<HD>, dim3((unsigned)((zeros + 255) / 256)), dim3(256), 0, s, a);
  const unsigned wgs = a.nitems * a.Hkv;
  if (wgs <= 256) hipLaunchKernelGGL((prefix_dq_kernel<HD, 2>), dim3(wgs), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((prefix_dq_kernel<HD, 1>), dim3(wgs), dim3(256), 0, s, a);
  if (a.njoins)
    hipLaunchKernelGGL((prefix_sum_join_kernel<HD, false>), dim3(a.njoins * a.Hkv, BQ * HD / 2048), dim3(256), 0, s, a);
  hipLaunchKernelGGL(prefix_dkdv_kernel<HD>, dim3(a.nkitems * a.Hkv), dim3(512), 0, s, a);
  if (a.nkjoins)
    hipLaunchKernelGGL((prefix_sum_join_kernel<HD, true>), dim3(a.nkjoins * a.Hkv, 2 * BQ * HD / 2048), dim3(256), 0, s,
                       a);
  return hipGetLastError();
}

}  // namespace

size_t prefix_part_floats(int hd, int which) {
  return which == 0 ? fwd_part(hd) : which == 1 ? dq_part(hd) : dkdv_part(hd);
}

hipError_t launch_prefix_fwd(const PrefixArgs& a, hipStream_t s) {
  return a.hd == 64 ? fwd_t<64>(a, s) : a.hd == 128 ? fwd_t<128>(a, s) : hipErrorInvalidValue;
}

hipError_t launch_prefix_bwd(const PrefixArgs& a, hipStream_t s) {
  return a.hd == 64 ? bwd_t<64>(a, s) : a.hd == 128 ? bwd_t<128>(a, s) : hipErrorInvalidValue;
}
