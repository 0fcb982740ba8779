// Attention of new tokens over a paged cache of keys and values and among
// themselves: a step's single tokens, trees of drafted tokens, pieces of prompts.
//
// A sequence's new tokens times the query heads of a group are its rows, token by
// token, for one key/value head. Keys are walked in tiles: the cached ones
// through the page table, then the sequence's new ones from the rows themselves,
// masked by the rows' words or by order. One walk of a block of rows over all its
// tiles is a segment; segments of all sequences, heads and blocks follow one
// another in one line of tiles, which is cut into equal shares, one a workgroup,
// whatever the lengths are. They are on the device, so each workgroup finds its
// share from them by itself; with more than 64 sequences a launch before sums
// them up. A segment that is cut leaves partial results (fp32 O, maximum, sum)
// that a second launch joins, in order, so runs repeat bit for bit.
//
// With 32 rows or fewer a sequence and head a workgroup is one wave, with a ring
// of its own in LDS and no barriers; five of them share a CU, 80 KiB of loads in
// flight. More rows take four waves, 128 rows, that share their tiles.
//
// A page's tile rows come through a buffer descriptor that ends with the
// sequence's last token, so that what a page holds behind it reads as zeros, and
// with nothing where the table names no page. Values of drafted tokens that are
// not finite are taken out of the tile and added for the rows that see them only.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_tile.h"
#include "common.h"
#include "kernels.h"

namespace {

// Workgroups' waves, keys of a tile, and workgroups that run at a time.
template <int HD, int TEAM>
struct Walk {
  static constexpr int KT = TEAM == 1 && HD == 128 ? 32 : 64;
  static constexpr int ROWS = 32 * TEAM, HEAD = HD;
  static constexpr int TB = KT * HD * 2;        // bytes of a tile of keys
  static constexpr int STAGES = 2;
  static constexpr int LDS = STAGES * 2 * TB;
  static constexpr int SHARES = 256 * (TEAM == 1 ? 5 : 2);
  static constexpr int LEAST = 4;               // tiles of a share
};
// Rows of a partial result, and its floats: O [rows][hd], maxima, sums.
__host__ DEV int part_rows(const TreeArgs& a, int rows) {
  const long most = (long)a.max_new * (a.H / a.Hkv);
  return most < rows ? (int)most : rows;
}
__host__ DEV size_t part_floats(const TreeArgs& a, int rows, int hd) { return (size_t)part_rows(a, rows) * (hd + 2); }

DEV int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// One sequence: its cached and new tokens, and its segments.
struct Seq {
  int len, start, n;
  int tc, t, blocks;   // tiles of cached keys, of a segment; blocks of rows
};
template <int KT, int ROWS>
DEV Seq seq_of(const TreeArgs& a, int s) {
  Seq q;
  q.len = clampi(a.lens[s], 0, a.max_pages * a.ps);
  q.start = clampi(a.starts[s], 0, a.n_rows);
  q.n = min(clampi(a.starts[s + 1], q.start, a.n_rows) - q.start, a.max_new);
  q.tc = (q.len + KT - 1) / KT;
  q.t = q.tc + (q.n + KT - 1) / KT;
  q.blocks = (q.n * (a.H / a.Hkv) + ROWS - 1) / ROWS;
  return q;
}

DEV int wave_scan(int x) {   // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// plan[s]: tiles before sequence s, s <= n_seq
template <int KT, int ROWS>
__global__ __launch_bounds__(64) void tree_plan_kernel(TreeArgs a) {
  const int lane = threadIdx.x;
  int before = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    int u = 0;
    if (s0 + lane < a.n_seq) {
      const Seq q = seq_of<KT, ROWS>(a, s0 + lane);
      u = q.t * q.blocks * a.Hkv;
    }
    const int x = wave_scan(u);
    if (s0 + lane < a.n_seq) a.plan[s0 + lane] = before + x - u;
    before += __builtin_amdgcn_readlane(x, 63);
  }
  if (lane == 0) a.plan[a.n_seq] = before;
}

// A cut this near a segment's end goes there: segments of up to `least` tiles
// are never cut, and few tiles are left on one side of a cut.
DEV int cut_slack(int share, int least) { return share <= 2 * least ? share / 2 : max(least / 2, share / 8); }

// The line of tiles. Up to 64 sequences: lane s holds the tiles before sequence
// s, summed up here. More: they are in plan.
template <int KT, int ROWS>
struct Line {
  int base, total, share, slack;
  bool planned;
  DEV void init(const TreeArgs& a, int shares, int least) {
    const int lane = threadIdx.x & 63;
    planned = a.n_seq > 64;
    if (planned) {
      total = __builtin_amdgcn_readfirstlane(a.plan[a.n_seq]);
    } else {
      int u = 0;
      if (lane < a.n_seq) {
        const Seq q = seq_of<KT, ROWS>(a, lane);
        u = q.t * q.blocks * a.Hkv;
      }
      const int x = wave_scan(u);
      base = x - u;
      total = __builtin_amdgcn_readlane(x, 63);
    }
    share = max(least, (total + shares - 1) / shares);
    slack = cut_slack(share, least);
  }
  // the sequence that has tile p < total, and the tiles before it
  DEV int find(const TreeArgs& a, int p, int* before) const {
    const int lane = threadIdx.x & 63;
    if (!planned) {
      const int s = __popcll(__ballot(lane < a.n_seq && base <= p)) - 1;
      *before = __builtin_amdgcn_readlane(base, s);
      return s;
    }
    const int step = (a.n_seq + 63) / 64;   // 64 at most
    const int i = min(lane * step, a.n_seq);
    const int k = (__popcll(__ballot(lane * step < a.n_seq && a.plan[i] <= p)) - 1) * step;
    const int j = min(k + lane, a.n_seq);
    const int b = a.plan[j];
    const int last = __popcll(__ballot(lane < step && k + lane < a.n_seq && b <= p)) - 1;
    *before = __builtin_amdgcn_readlane(b, last);
    return k + last;
  }
  // where the cut at tile p is made, p in the segment [from, from + t)
  DEV int cut(int p, int from, int t) const {
    return p - from <= slack ? from : from + t - p <= slack ? from + t : p;
  }
  DEV int bound(const TreeArgs& a, int w) const {
    const int p = w * share;   // below total + share
    if (p >= total) return total;
    int before;
    const int s = find(a, p, &before);
    const Seq q = seq_of<KT, ROWS>(a, s);
    const int from = before + (p - before) / q.t * q.t;
    return cut(p, from, q.t);
  }
};

// Keys and values of one segment, tile by tile into a wave's (or team's) ring.
template <int HD, int TEAM>
struct Keys {
  using W = Walk<HD, TEAM>;
  static constexpr int U = HD / 8, PER = 16 * U / 64;   // 16-byte units of a row; loads of 16 rows
  const TreeArgs* a;
  const int32_t* table;     // the sequence's
  const bf16_t* rows;       // its new tokens' keys
  uint32_t ld;              // bytes between tokens
  uint32_t page_bytes, v_bytes;   // of a page; from its keys to its values
  size_t head;              // bytes of the heads before this one
  int len, n, tc, lps;
  int win, ids;             // the lane's entry of the table, pages win..win+63
  uint32_t rel[PER], reld[PER];   // the lane's byte offset in 16 rows of a page, of new tokens
  uint64_t seen;            // of the last tile issued: keys that are there

  DEV void init(const TreeArgs& args, int s, const Seq& q, int j, int lane) {
    a = &args;
    table = args.table + (size_t)s * args.max_pages;
    const int slots = args.H + 2 * args.Hkv;
    ld = (uint32_t)slots * HD * 2;
    rows = args.qkv + (size_t)q.start * slots * HD + (size_t)(args.H + j) * HD;
    v_bytes = (uint32_t)args.Hkv * args.ps * HD * 2;
    page_bytes = 2 * v_bytes;
    head = (size_t)j * args.ps * HD * 2;
    len = q.len;
    n = q.n;
    tc = q.tc;
    lps = 31 - __builtin_clz(args.ps);
    win = -64;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int u = i * 64 + lane, row = u / U, c = unit<HD>(row, u % U) - row * U;   // the XOR is its own inverse
      rel[i] = (uint32_t)(row * HD + c * 8) * 2u;
      reld[i] = (uint32_t)row * ld + (uint32_t)c * 16u;
    }
  }

  DEV void issue(int f, lds_char_t* st, int wave, int lane) {
    constexpr int GROUPS = W::KT / 16;
    seen = 0;
    if (f < tc) {
      const int p0 = f * W::KT >> lps, p1 = (f * W::KT + W::KT - 1) >> lps;
      if (p1 >= win + 64 || p0 < win) {
        win = p0;
        ids = table[min(p0 + lane, a->max_pages - 1)];
      }
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const int key = f * W::KT + 16 * q;
        const int page = __builtin_amdgcn_readlane(ids, (key >> lps) - win);
        const int there = (unsigned)page < (unsigned)a->n_pages ? clampi(len - key, 0, 16) : 0;
        seen |= (uint64_t)((1u << there) - 1u) << (16 * q);
        if (q % TEAM != wave % GROUPS % TEAM) continue;
        const char* k = reinterpret_cast<const char*>(a->pages) + (size_t)(there ? page : 0) * page_bytes + head +
                        (size_t)(key & (a->ps - 1)) * HD * 2;
        const v4i32 rk = make_rsrc(k, (uint32_t)there * HD * 2), rv = make_rsrc(k + v_bytes, (uint32_t)there * HD * 2);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          dma16(rk, rel[i], lds_addr(st + (q * PER + i) * 1024));
          dma16(rv, rel[i], lds_addr(st + W::TB + (q * PER + i) * 1024));
        }
      }
    } else {
      const int d0 = (f - tc) * W::KT;
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const int there = clampi(n - d0 - 16 * q, 0, 16);
        seen |= (uint64_t)((1u << there) - 1u) << (16 * q);
        if (q % TEAM != wave % GROUPS % TEAM) continue;
        const char* k = reinterpret_cast<const char*>(rows) + (there ? (size_t)(d0 + 16 * q) * ld : 0);
        const uint32_t bytes = there ? (there - 1) * ld + HD * 2 : 0;
        const v4i32 rk = make_rsrc(k, bytes), rv = make_rsrc(k + (size_t)a->Hkv * HD * 2, bytes);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          dma16(rk, reld[i], lds_addr(st + (q * PER + i) * 1024));
          dma16(rv, reld[i], lds_addr(st + W::TB + (q * PER + i) * 1024));
        }
      }
    }
  }
};

// Rows of a tile of values with an element that is not finite.
template <int HD, int KT>
DEV uint64_t not_finite(const lds_char_t* vs, int lane) {
  constexpr int U = HD / 8;
  uint64_t bad = 0;
#pragma unroll 4
  for (int i = 0; i < KT * U / 64; ++i) {
    const uint4 x = __builtin_bit_cast(uint4, *reinterpret_cast<const lds_v4u32_t*>(vs + (i * 64 + lane) * 16));
    auto special = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
    const uint64_t hit = __ballot(special(x.x) || special(x.y) || special(x.z) || special(x.w));
    if (hit) {
#pragma unroll
      for (int r = 0; r < 64 / U; ++r)
        if (hit >> (r * U) & ((1ull << U) - 1)) bad |= 1ull << (i * (64 / U) + r);
    }
  }
  return bad;
}

template <int HD, int TEAM>
__global__ __launch_bounds__(64 * TEAM, 2) void tree_kernel(TreeArgs a) {
  using W = Walk<HD, TEAM>;
  using S = Shape<HD>;
  constexpr int KT = W::KT, NT = KT / 32;
  __shared__ __attribute__((aligned(1024))) char smem_raw[W::LDS];
  lds_char_t* smem = (lds_char_t*)smem_raw;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lq = lane & 31, g = lane >> 5, me = blockIdx.x, G = a.H / a.Hkv;
  const float sc = LOG2E / sqrtf((float)HD);
  Line<KT, W::ROWS> line;
  line.init(a, W::SHARES, W::LEAST);
  if (me == 0 && wave == 0 && !line.planned) {   // for the launch that joins
    if (lane < a.n_seq) a.plan[lane] = line.base;
    if (lane == 0) a.plan[a.n_seq] = line.total;
  }
  if ((long)me * line.share >= line.total) return;
  const int end = line.bound(a, me + 1);
  for (int p = line.bound(a, me); p < end;) {
    int before;
    const int s = __builtin_amdgcn_readfirstlane(line.find(a, p, &before));
    before = __builtin_amdgcn_readfirstlane(before);
    Seq q = seq_of<KT, W::ROWS>(a, s);
    q.len = __builtin_amdgcn_readfirstlane(q.len);
    q.start = __builtin_amdgcn_readfirstlane(q.start);
    q.n = __builtin_amdgcn_readfirstlane(q.n);
    q.tc = __builtin_amdgcn_readfirstlane(q.tc);
    q.t = __builtin_amdgcn_readfirstlane(q.t);
    const int seg = (p - before) / q.t, j = seg % a.Hkv, block = seg / a.Hkv;
    const int from = before + seg * q.t;
    const int f0 = p - from, f1 = min(end - from, q.t);
    p = from + f1;
    // a block of rows without a mask needs the new tokens up to its last only
    const int last = min(((block + 1) * W::ROWS - 1) / G, q.n - 1);
    const int f_end = a.mask ? f1 : min(f1, q.tc + last / KT + 1);

    Keys<HD, TEAM> keys;
    keys.init(a, s, q, j, lane);
    auto stage = [&](int f) { return smem + (f - f0) % W::STAGES * 2 * W::TB; };
    if (f0 < f_end) keys.issue(f0, stage(f0), wave, lane);
    uint64_t next_seen = keys.seen;

    const int row = block * W::ROWS + 32 * wave + lq;
    const bool on = row < q.n * G;
    const int r = min(row, q.n * G - 1), i = r / G, h = j * G + r - i * G;
    const size_t token = (size_t)q.start + i;
    const bf16_t* qp = a.qkv + token * (a.H + 2 * a.Hkv) * HD + (size_t)h * HD;
    bf16x8 qf[S::KS];
#pragma unroll
    for (int k = 0; k < S::KS; ++k) qf[k] = as_bf16x8(*reinterpret_cast<const uint4*>(qp + 16 * k + 8 * g));
    floatx16 o[S::DT];
#pragma unroll
    for (int d = 0; d < S::DT; ++d) zero(o[d]);
    float m_run = -INFINITY, l_run = 0.0f;

    for (int f = f0; f < f_end; ++f) {
      wait_vmcnt<0>();
      __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
      if constexpr (TEAM > 1) block_barrier();
      const uint64_t there = next_seen;
      if (f + 1 < f_end) {
        keys.issue(f + 1, stage(f + 1), wave, lane);
        next_seen = keys.seen;
      }
      const lds_char_t* Ks = stage(f);
      lds_char_t* Vs = stage(f) + W::TB;
      // the keys that this lane's row sees
      constexpr uint64_t ALL = KT == 64 ? ~0ull : (1ull << KT) - 1;
      uint64_t mine = there, bad = 0;
      if (f >= q.tc) {
        const int d0 = (f - q.tc) * KT;
        if (a.mask) {
          const int32_t* words = a.mask + token * a.mask_words + d0 / 32;
          uint64_t w = d0 / 32 < a.mask_words ? (uint32_t)words[0] : 0u;
          if (KT == 64 && d0 / 32 + 1 < a.mask_words) w |= (uint64_t)(uint32_t)words[1] << 32;
          mine &= w;
        } else if (i < d0 + KT - 1) {
          mine &= i < d0 ? 0ull : (2ull << (i - d0)) - 1;
        }
        // (the whole team's rows, so that its waves agree)
        if (a.mask || block * W::ROWS / G < d0 + KT - 1) {
          bad = not_finite<HD, KT>(Vs, lane);
          if (bad) {
            if constexpr (TEAM > 1) block_barrier();
            for (int u = threadIdx.x; u < KT * HD / 8; u += 64 * TEAM)
              if (bad >> (u / (HD / 8)) & 1) *reinterpret_cast<lds_v4u32_t*>(Vs + u * 16) = v4u32{0, 0, 0, 0};
            __builtin_amdgcn_s_waitcnt(0xC07F);
            if constexpr (TEAM > 1) block_barrier();
          }
        }
      }
      if (__ballot(mine != 0) == 0) continue;

      floatx16 x[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        zero(x[t]);
#pragma unroll
        for (int k = 0; k < S::KS; ++k) x[t] = mfma32(read_row<HD>(Ks, 32 * t + lq, 2 * k + g), qf[k], x[t]);
      }
      float mt = -INFINITY;
      if (__ballot(mine != ALL) == 0) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) mt = fmaxf(mt, x[t][e]);
      } else {
        const uint64_t bits = mine >> (4 * g);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            x[t][e] = bits >> (32 * t + acc_row(e, 0)) & 1 ? x[t][e] : -INFINITY;
            mt = fmaxf(mt, x[t][e]);
          }
      }
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
      const float shift = m_run == -INFINITY ? 0.0f : m_run;   // nothing seen yet
      float rsum = 0.0f;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float w = fast_exp2(fmaf(x[t][e], sc, -shift));
          x[t][e] = w;
          rsum += w;
        }
      l_run += sum32(rsum);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const bf16x8 pf = acc_slots(x[t], hh);
#pragma unroll
          for (int d = 0; d < S::DT; ++d) o[d] = mfma32(read_tr<HD>(Vs, 32 * d, 32 * t + 16 * hh, lane), pf, o[d]);
        }
      // values that are not finite, one token after another
      while (bad) {
        const int k = __builtin_ctzll(bad);
        bad &= bad - 1;
        float w = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) w = (k & ~4) == 32 * t + acc_row(e, 0) ? x[t][e] : w;
        w = __shfl(w, lq + (k >> 2 & 1) * 32);
        const bf16_t* v = a.qkv + ((size_t)q.start + (f - q.tc) * KT + k) * (a.H + 2 * a.Hkv) * HD +
                          (size_t)(a.H + a.Hkv + j) * HD;
        const bool sees = mine >> k & 1;
#pragma unroll
        for (int d = 0; d < S::DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = o[d][e] + w * bf2f(v[32 * d + acc_row(e, 0) + 4 * g]);
            o[d][e] = sees ? y : o[d][e];
          }
      }
    }
    if constexpr (TEAM > 1) __syncthreads();   // the ring is the next segment's
    if (!on) continue;
    if (f0 == 0 && f1 == q.t) {
      const float inv = l_run > 0.0f ? 1.0f / l_run : l_run == 0.0f ? 0.0f : l_run;
      bf16_t* out = a.out + (token * a.H + h) * HD;
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<uint2*>(out + 32 * d + 8 * c + 4 * g) =
              make_uint2(pack2(o[d][4 * c] * inv, o[d][4 * c + 1] * inv),
                         pack2(o[d][4 * c + 2] * inv, o[d][4 * c + 3] * inv));
      if (g == 0 && a.lse) a.lse[(size_t)h * a.n_rows + token] = (m_run + log2f(l_run)) * LN2;
      continue;
    }
    // a share has at most two cut segments: one that begins in it, one that does not
    const int prows = part_rows(a, W::ROWS);
    float* part = a.part + (2 * (size_t)me + (f0 == 0)) * part_floats(a, W::ROWS, HD);
    const int pr = 32 * wave + lq;
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(part + (size_t)pr * HD + 32 * d + 8 * c + 4 * g) =
            make_float4(o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]);
    if (g == 0) {
      part[(size_t)prows * HD + pr] = m_run;
      part[(size_t)prows * HD + prows + pr] = l_run;
    }
  }
}

// The parts of a cut segment's row, a wave a row of one query head.
template <int HD, int TEAM>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  using W = Walk<HD, TEAM>;
  constexpr int LANES = HD / 8, GROUPS = 64 / LANES;
  const int lane = threadIdx.x & 63, G = a.H / a.Hkv;
  const long at = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int token = (int)(at / a.H), h = (int)(at - (long)token * a.H);
  if (token >= a.n_rows) return;
  // the sequence that has the row: the last one that begins at or before it
  int s = -1;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const uint64_t b = __ballot(s0 + lane < a.n_seq && a.starts[min(s0 + lane, a.n_seq)] <= token);
    if (b) s = s0 + 63 - __builtin_clzll(b);
  }
  if (s < 0) return;
  const Seq q = seq_of<W::KT, W::ROWS>(a, s);
  const int i = token - q.start;
  if (i < 0 || i >= q.n) return;
  const int total = a.plan[a.n_seq];
  const int share = max(W::LEAST, (total + W::SHARES - 1) / W::SHARES);
  const int slack = cut_slack(share, W::LEAST);
  const int j = h / G, r = i * G + h - j * G, block = r / W::ROWS, row = r - block * W::ROWS;
  const int from = a.plan[s] + (block * a.Hkv + j) * q.t;
  // cuts w0..w1 lie inside the segment, so shares w0 - 1..w1 have its parts
  const int w0 = (from + slack) / share + 1, w1 = (from + q.t - slack - 1) / share;
  if (w1 < w0) return;
  const int parts = w1 - w0 + 2;
  const int prows = part_rows(a, W::ROWS);
  const size_t floats = part_floats(a, W::ROWS, HD);
  const float* part0 = a.part + 2 * (size_t)(w0 - 1) * floats;
  // part k's place: the first begins in its share, the others do not
  auto place = [&](int k) { return part0 + (2 * (size_t)k + (k == 0)) * floats; };
  float m = -INFINITY;
  for (int k = lane; k < parts; k += 64) m = fmaxf(m, place(k)[(size_t)prows * HD + row]);
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float shift = m == -INFINITY ? 0.0f : m;
  const int c = lane % LANES * 8;
  float l = 0.0f, o[8] = {};
  for (int k0 = 0; k0 < parts; k0 += 64) {
    float wgt = 0.0f;
    if (k0 + lane < parts) {
      const float* p = place(k0 + lane) + (size_t)prows * HD;
      wgt = fast_exp2(p[row] - shift);
      l += wgt * p[prows + row];
    }
    const int n = min(64, parts - k0);
#pragma unroll 4
    for (int k = 0; k < n; k += GROUPS) {
      const int w = k + lane / LANES;
      const float f = __shfl(wgt, min(w, 63));
      if (w < n) {
        const float* p = place(k0 + w) + (size_t)row * HD + c;
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
    for (int x = LANES; x < 64; x <<= 1) o[e] += __shfl_xor(o[e], x);
  if (lane >= LANES) return;
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  *reinterpret_cast<uint4*>(a.out + ((size_t)token * a.H + h) * HD + c) =
      make_uint4(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv), pack2(o[4] * inv, o[5] * inv),
                 pack2(o[6] * inv, o[7] * inv));
  if (c == 0 && a.lse) a.lse[(size_t)h * a.n_rows + token] = (m + log2f(l)) * LN2;
}

int team_of(const TreeArgs& a) { return (long)a.max_new * (a.H / a.Hkv) <= 32 ? 1 : 4; }

template <class Fn>
auto with_walk(const TreeArgs& a, Fn f) {
  const bool wide = a.hd == 128;
  if (team_of(a) == 1) return wide ? f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{})
                                   : f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  return wide ? f(std::integral_constant<int, 128>{}, std::integral_constant<int, 4>{})
              : f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
}

// Tiles of all sequences at their longest, and of one of their segments.
template <int HD, int TEAM>
double most_tiles(const TreeArgs& a, double* segment) {
  using W = Walk<HD, TEAM>;
  *segment = std::ceil((double)a.max_pages * a.ps / W::KT) + std::ceil((double)a.max_new / W::KT);
  return *segment * a.n_seq * a.Hkv * std::ceil((double)a.max_new * (a.H / a.Hkv) / W::ROWS);
}

}  // namespace

size_t tree_workspace(const TreeArgs& a, size_t* part_at) {
  return with_walk(a, [&](auto hd, auto team) -> size_t {
    using W = Walk<decltype(hd)::value, decltype(team)::value>;
    double segment;
    // tiles are counted in 32 bits
    if (most_tiles<decltype(hd)::value, decltype(team)::value>(a, &segment) > 2e9) return 0;
    const size_t plan = ((size_t)a.n_seq + 2) * sizeof(int32_t);
    *part_at = (plan + 255) / 256 * 256;
    return *part_at + (segment > W::LEAST ? 2 * (size_t)W::SHARES * part_floats(a, W::ROWS, W::HEAD) * sizeof(float) : 0);
  });
}

hipError_t launch_tree(const TreeArgs& a, hipStream_t s) {
  if (a.n_rows < 1) return hipSuccess;
  return with_walk(a, [&](auto hd, auto team) -> hipError_t {
    constexpr int HD = decltype(hd)::value, TEAM = decltype(team)::value;
    using W = Walk<HD, TEAM>;
    double segment;
    const double tiles = most_tiles<HD, TEAM>(a, &segment);
    if (a.n_seq > 64) hipLaunchKernelGGL((tree_plan_kernel<W::KT, W::ROWS>), dim3(1), dim3(64), 0, s, a);
    const unsigned shares = (unsigned)std::min((double)W::SHARES, std::ceil(tiles / W::LEAST));
    hipLaunchKernelGGL((tree_kernel<HD, TEAM>), dim3(shares), dim3(64 * TEAM), 0, s, a);
    // segments of no more tiles than the smallest share are never cut
    if (segment > W::LEAST)
      hipLaunchKernelGGL((tree_join_kernel<HD, TEAM>), dim3((unsigned)(((long)a.n_rows * a.H + 3) / 4)), dim3(256), 0,
                         s, a);
    return hipGetLastError();
  });
}
