// Attention of new tokens over a paged cache of keys and values and among
// themselves: a step's single tokens, trees of drafted tokens, pieces of prompts.
//
// A sequence's new tokens times the query heads of a group are its rows, token by
// token, for one key/value head. Keys are walked in tiles: the cached ones
// through the page table, then the sequence's new ones from the rows themselves,
// masked by the rows' words or by order. One walk of a block of rows over all its
// tiles is a segment. Lengths are on the device, so workers find what they do from
// them by themselves (with more than 64 sequences a launch before sums them up):
// where segments are few each is dealt to some workers in equal pieces; otherwise
// segments follow one another in one line of tiles, which is cut into equal
// shares. A segment of several workers leaves partial results (fp32 O, maximum,
// sum) that a second launch joins, in order, so runs repeat bit for bit.
//
// A workgroup's four waves are RB blocks of 32 rows times 4/RB groups that walk a
// share's tiles in turn and merge at a segment's end. With one block of rows and
// many segments each wave is a worker of its own instead, without barriers.
//
// A page's tile rows come through a buffer descriptor that ends with the
// sequence's last token, so that what a page holds behind it reads as zeros, and
// with nothing where the table names no page. Tiles of drafted tokens whose values
// are not all finite go without the matrix product, token by token, so that they
// reach the rows that see them only.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_tile.h"
#include "common.h"
#include "kernels.h"

namespace {

// Keys of a tile, and how the line of tiles is shared out.
template <int HD, int RB>
struct Walk {
  static constexpr int HEAD = HD, ROWS = 32 * RB, GROUPS = 4 / RB;
  static constexpr int KT = HD == 128 && RB < 4 ? 32 : 64;
  static constexpr int TB = KT * HD * 2;        // bytes of a tile of keys
  static constexpr int STAGES = 2;
  static constexpr int RING = STAGES * 2 * TB;  // of a group
  static constexpr int DT = HD / 32, PER = DT > GROUPS ? DT / GROUPS : 1;   // blocks of 32 columns of O; of a group, merging
  // of a wave's O for the others, maxima and sums
  static constexpr int KEEP = (DT - (GROUPS * PER > DT ? 0 : PER)) * 4096 + 512;
  static constexpr int LEAST = 4;               // tiles of a share; segments of no more are never cut
  static constexpr int SLACK = LEAST / 2;       // tiles from a segment's end within which a cut goes there
  // (single tokens of 8 sequences of 200 to 2,048: 21 us with twice as many, 19 so)
  static constexpr int WHOLE = 2 * GROUPS > LEAST ? 2 * GROUPS : LEAST;   // ... nor dealt of these
  static constexpr int TEAMS = 256 * (RB == 1 ? 1 : 2);   // workgroups that run at a time
  static constexpr int MOST = RB == 1 ? 4 * TEAMS : TEAMS;   // shares
  static_assert(GROUPS == 1 || 4 * KEEP <= GROUPS * RING, "the groups' results fit their tiles' space");
};
// Rows of a partial result, and its floats: O [rows][hd], maxima, sums.
__host__ DEV int part_rows(const TreeArgs& a, int rows) {
  const long most = ((long)a.max_new * (a.H / a.Hkv) + 1) / 2 * 2;   // even: parts begin at multiples of 16 bytes
  return most < rows ? (int)most : rows;
}
__host__ DEV size_t part_floats(const TreeArgs& a, int rows, int hd) { return (size_t)part_rows(a, rows) * (hd + 2); }

DEV int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// One sequence: its cached and new tokens, and its segments.
struct Seq {
  int len, start, n;
  int tc, t, blocks;   // tiles of cached keys, of a segment; blocks of rows
};
template <class W>
DEV Seq seq_from(const TreeArgs& a, int len, int start, int n) {
  Seq q;
  q.len = len;
  q.start = start;
  q.n = n;
  q.tc = (len + W::KT - 1) / W::KT;
  q.t = q.tc + (n + W::KT - 1) / W::KT;
  q.blocks = (n * (a.H / a.Hkv) + W::ROWS - 1) / W::ROWS;
  return q;
}
// Whether sequence s ends before it begins, which starts must not: nothing is computed then, as the sums of tiles are
// bounded by rows that belong to one sequence.
DEV bool falls(const TreeArgs& a, int s) { return a.starts[s + 1] < a.starts[s]; }
template <class W>
DEV Seq seq_of(const TreeArgs& a, int s) {
  const int start = clampi(a.starts[s], 0, a.n_rows);
  return seq_from<W>(a, clampi(a.lens[s], 0, a.max_pages * a.ps), start,
                     min(clampi(a.starts[s + 1], start, a.n_rows) - start, a.max_new));
}

// v of the lane that CTRL names, in the rows of ROWS; 0 elsewhere
template <int CTRL, int ROWS>
DEV int dpp(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true);
}
// over the lanes up to each: shifts within rows of 16, then rows' last lanes to the rows behind
DEV int wave_scan(int v) {
  v += dpp<0x111, 0xf>(v);
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);
  return v + dpp<0x143, 0xc>(v);
}

// How the work is divided.
//  dealt  a segment of t tiles goes to pieces_of(t, share) workers; a sequence's
//         base is the number of workers before it
//  line   worker w has tiles w share.. of the line of all segments, a cut within
//         SLACK of a segment's end going there (so segments of LEAST tiles are
//         never cut); a sequence's base is the number of tiles before it
//  solo   line, every wave a worker of its own
enum Division { DEALT, LINE, SOLO };
typedef int Cuts __attribute__((ext_vector_type(2)));   // division, share
// (about t / share: the hardware's reciprocal will do, as all take the same)
template <class W>
DEV int pieces_of(int t, int share) {
  return t <= W::WHOLE ? 1 : max(1, (int)((float)(t + share - 1) * __builtin_amdgcn_rcpf((float)share)));
}
// workers(share): the workers that segments dealt in pieces of `share` tiles take
template <class W, class Fn>
DEV Cuts cuts_of(int total, int segments, int longest, Fn workers) {
  const int even = max(W::WHOLE / 2, (total + W::TEAMS - 1) / W::TEAMS);
  int deal = segments <= W::TEAMS && longest <= W::WHOLE ? even : 0;
  // Pieces of up to 14/32 more tiles than equal shares, the fewest that do, cost less than workers with parts of two
  // segments. Of 16 sequences of 1,000 to 3,001 tokens with 24 drafts each: 42 us with no more, 40 with three in eight,
  // 41 with eight; of three pieces of prompts 45, 40, 41; all in one line 41 and 44.
  if (segments <= W::TEAMS) {
    int k = 15;
#pragma unroll
    for (int step = 8; step; step >>= 1) k -= workers(even + (even * (k - step) + 31) / 32) <= W::TEAMS ? step : 0;
    if (k < 15) deal = even + (even * k + 31) / 32;
  }
  // (single tokens of 64 sequences of 200 to 4,096, 512 segments: 136 us with groups, 100 without; of 64 of 100 to 300:
  // 38, 25)
  const bool solo = W::GROUPS == 4 && segments > W::TEAMS;
  const int shares = solo ? W::MOST : W::TEAMS, share = max(W::LEAST, (total + shares - 1) / shares);
  return Cuts{deal ? DEALT : solo ? SOLO : LINE, deal ? deal : share};
}

DEV int wave_total(int v) { return __builtin_amdgcn_readlane(wave_scan(v), 63); }
DEV int wave_max(int v) {   // of values that are not negative
  v = max(v, dpp<0x111, 0xf>(v));
  v = max(v, dpp<0x112, 0xf>(v));
  v = max(v, dpp<0x114, 0xf>(v));
  v = max(v, dpp<0x118, 0xf>(v));
  v = max(v, dpp<0x142, 0xa>(v));
  return __builtin_amdgcn_readlane(max(v, dpp<0x143, 0xc>(v)), 63);
}

// The plan, for the launches behind: bases of the sequences and their sum, then
// the cuts.
DEV void store_cuts(const TreeArgs& a, int sum, const Cuts& c) {
  a.plan[a.n_seq] = sum;
  a.plan[a.n_seq + 1] = c.x;
  a.plan[a.n_seq + 2] = c.y;
}

template <class W>
__global__ __launch_bounds__(64) void tree_plan_kernel(TreeArgs a) {
  const int lane = threadIdx.x;
  bool bad = false;
  for (int s = lane; s < a.n_seq; s += 64) bad |= falls(a, s);
  if (__ballot(bad) != 0) {
    if (lane == 0) store_cuts(a, 0, Cuts{LINE, W::LEAST});
    return;
  }
  auto over = [&](auto f) {   // the sum over the sequences
    int sum = 0;
    for (int s = lane; s < a.n_seq; s += 64) sum += f(seq_of<W>(a, s));
    return wave_total(sum);
  };
  int most = 0;
  for (int s = lane; s < a.n_seq; s += 64) {
    const Seq q = seq_of<W>(a, s);
    if (q.blocks) most = max(most, q.t);
  }
  const Cuts c = cuts_of<W>(over([&](const Seq& q) { return q.t * q.blocks * a.Hkv; }),
                            over([&](const Seq& q) { return q.blocks * a.Hkv; }), wave_max(most), [&](int share) {
                              return over([&](const Seq& q) { return pieces_of<W>(q.t, share) * q.blocks * a.Hkv; });
                            });
  int before = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    int u = 0;
    if (s0 + lane < a.n_seq) {
      const Seq q = seq_of<W>(a, s0 + lane);
      u = (c.x == DEALT ? pieces_of<W>(q.t, c.y) : q.t) * q.blocks * a.Hkv;
    }
    const int x = wave_scan(u);
    if (s0 + lane < a.n_seq) a.plan[s0 + lane] = before + x - u;
    before += __builtin_amdgcn_readlane(x, 63);
  }
  if (lane == 0) store_cuts(a, before, c);
}

// What a worker knows of it all. Up to 64 sequences: lane s has sequence s. More:
// the plan was made before.
template <class W>
struct Line {
  int base, len, start, n, sum;
  bool planned;
  Cuts cuts;
  DEV void init(const TreeArgs& a) {
    const int lane = threadIdx.x & 63;
    planned = a.n_seq > 64;
    if (planned) {
      sum = __builtin_amdgcn_readfirstlane(a.plan[a.n_seq]);
      cuts.x = __builtin_amdgcn_readfirstlane(a.plan[a.n_seq + 1]);
      cuts.y = __builtin_amdgcn_readfirstlane(a.plan[a.n_seq + 2]);
      return;
    }
    Seq q{};
    bool bad = false;
    if (lane < a.n_seq) {
      q = seq_of<W>(a, lane);
      bad = falls(a, lane);
    }
    len = q.len;
    start = q.start;
    n = q.n;
    const int each = q.blocks * a.Hkv;
    cuts = cuts_of<W>(wave_total(q.t * each), wave_total(each), wave_max(each ? q.t : 0),
                      [&](int share) { return wave_total(pieces_of<W>(q.t, share) * each); });
    const int u = (cuts.x == DEALT ? pieces_of<W>(q.t, cuts.y) : q.t) * each, x = wave_scan(u);
    base = x - u;
    sum = __ballot(bad) ? 0 : __builtin_amdgcn_readlane(x, 63);
  }
  // the sequence that has tile (worker) p < sum, and what is before it
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
  DEV Seq seq(const TreeArgs& a, int s) const {
    if (!planned)
      return seq_from<W>(a, __builtin_amdgcn_readlane(len, s), __builtin_amdgcn_readlane(start, s),
                         __builtin_amdgcn_readlane(n, s));
    const Seq q = seq_of<W>(a, s);
    return seq_from<W>(a, __builtin_amdgcn_readfirstlane(q.len), __builtin_amdgcn_readfirstlane(q.start),
                       __builtin_amdgcn_readfirstlane(q.n));
  }
  // where share w of the line begins
  DEV int bound(const TreeArgs& a, int w) const {
    const int p = w * cuts.y;   // below sum + share
    if (p >= sum) return sum;
    int before;
    const int s = find(a, p, &before);
    const int t = seq(a, s).t, from = before + (p - before) / t * t;
    return p - from <= W::SLACK ? from : from + t - p <= W::SLACK ? from + t : p;
  }
};

// dma16 past the caches, of what nobody else reads soon: pieces of one block of rows
// whose first page has one holder. One token over 131,071: 103 -> 95 us a pass; pages
// that 64 sequences share would take 316 us so instead of 276.
DEV void dma16_once(v4i32 rsrc, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}

// Keys and values of one segment, tile by tile into a group's ring.
template <int HD, int RB>
struct Keys {
  using W = Walk<HD, RB>;
  static constexpr int U = HD / 8, PER = 16 * U / 64;   // 16-byte units of a row; loads of 16 rows
  const TreeArgs* a;
  const int32_t* table;     // the sequence's
  const bf16_t* rows;       // its new tokens' keys
  uint32_t ld;              // bytes between tokens
  uint32_t page_bytes, v_bytes;   // of a page; from its keys to its values
  size_t head;              // bytes of the heads before this one
  int len, n, tc, lps;
  int win, ids;             // the lane's entry of the table, pages win..win+63
  int refs;                 // sequences that have the piece's first page; 0 where other rows walk it too
  uint64_t named;           // of the window: entries that are pages
  uint64_t seen;            // of the last tile issued: keys that are there
  uint32_t base;            // the lane's byte offset in 16 rows of a page, first load

  DEV void init(const TreeArgs& args, int s, const Seq& q, int j, int f0) {
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
    base = RB == 1 ? offset(0, threadIdx.x & 63, HD * 2) : 0;
    look(f0 * W::KT >> lps);
    const int page = __builtin_amdgcn_readfirstlane(ids);
    refs = RB == 1 && q.blocks == 1 && (unsigned)page < (unsigned)args.n_pages ? args.refs[page] : 0;
  }

  DEV void look(int from) {
    win = from;
    ids = table[min(win + (int)(threadIdx.x & 63), a->max_pages - 1)];
    named = __ballot((unsigned)ids < (unsigned)a->n_pages);
  }

  // the lane's part of load i of 16 rows that are `stride` bytes apart
  static constexpr uint32_t turn(int i) { return HD == 128 ? ((i & 1) << 1 | i >> 1) * 16 : i * 16; }   // load i's against load 0's
  static DEV uint32_t offset(int i, int lane, uint32_t stride) {
    const int u = i * 64 + lane, row = u / U, c = unit<HD>(row, u % U) - row * U;   // the XOR is its own inverse
    return (uint32_t)row * stride + (uint32_t)c * 16u;
  }
  // by the waves of a group, `wave` of RB
  DEV void issue(int f, lds_char_t* st, int wave, bool once) {
    constexpr int SIXTEENS = W::KT / 16;
    if (f < tc) {
      const int p0 = f * W::KT >> lps, p1 = (f * W::KT + W::KT - 1) >> lps;
      if (p1 >= win + 64 || p0 < win) look(p0);
      auto page_of = [&](int key) { return __builtin_amdgcn_readlane(ids, (key >> lps) - win); };
      const uint64_t pages = (2ull << (p1 - p0)) - 1;
      seen = W::KT == 64 ? ~0ull : (1ull << W::KT) - 1;
      if ((f + 1) * W::KT > len || (named >> (p0 - win) & pages) != pages) {
        seen = 0;
#pragma unroll
        for (int q = 0; q < SIXTEENS; ++q) {
          const int key = f * W::KT + 16 * q;
          const int there = named >> ((key >> lps) - win) & 1 ? clampi(len - key, 0, 16) : 0;
          seen |= (uint64_t)((1u << there) - 1u) << (16 * q);
        }
      }
      // the loads' offsets are made again for each tile: kept, they would leave too few registers
      uint32_t at = base;
      if constexpr (RB == 1) {
        asm volatile("" : "+v"(at));
      } else {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        at = offset(0, lane, HD * 2);
      }
#pragma unroll 1
      for (int q = wave; q < SIXTEENS; q += RB) {
        const int key = f * W::KT + 16 * q, there = __builtin_popcount((uint32_t)(seen >> (16 * q)) & 0xffffu);
        const char* k = reinterpret_cast<const char*>(a->pages) + (size_t)(there ? page_of(key) : 0) * page_bytes + head +
                        (size_t)(key & (a->ps - 1)) * HD * 2;
        const v4i32 rk = make_rsrc(k, (uint32_t)there * HD * 2), rv = make_rsrc(k + v_bytes, (uint32_t)there * HD * 2);
        if (RB == 1 && once) {
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            dma16_once(rk, ((at ^ turn(i)) + i * 1024), lds_addr(st + (q * PER + i) * 1024));
            dma16_once(rv, ((at ^ turn(i)) + i * 1024), lds_addr(st + W::TB + (q * PER + i) * 1024));
          }
          continue;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          dma16(rk, ((at ^ turn(i)) + i * 1024), lds_addr(st + (q * PER + i) * 1024));
          dma16(rv, ((at ^ turn(i)) + i * 1024), lds_addr(st + W::TB + (q * PER + i) * 1024));
        }
      }
    } else {
      const int d0 = (f - tc) * W::KT;
      int lane = threadIdx.x & 63;
      asm volatile("" : "+v"(lane));   // likewise
      seen = n - d0 >= 64 ? ~0ull : (1ull << max(n - d0, 0)) - 1;
      if constexpr (W::KT < 64) seen &= (1ull << W::KT) - 1;
#pragma unroll 1
      for (int q = wave; q < SIXTEENS; q += RB) {
        const int there = clampi(n - d0 - 16 * q, 0, 16);
        const char* k = reinterpret_cast<const char*>(rows) + (there ? (size_t)(d0 + 16 * q) * ld : 0);
        const uint32_t bytes = there ? (there - 1) * ld + HD * 2 : 0;
        const v4i32 rk = make_rsrc(k, bytes), rv = make_rsrc(k + (size_t)a->Hkv * HD * 2, bytes);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          dma16(rk, offset(i, lane, ld), lds_addr(st + (q * PER + i) * 1024));
          dma16(rv, offset(i, lane, ld), lds_addr(st + W::TB + (q * PER + i) * 1024));
        }
      }
    }
  }
};

DEV bool special(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
// Whether an element of 32 rows of values is not finite.
template <int HD>
DEV bool not_finite(const lds_char_t* vs, int lane) {
  bool hit = false;
#pragma unroll 4
  for (int i = 0; i < HD / 16; ++i) {
    const v4u32 x = *reinterpret_cast<const lds_v4u32_t*>(vs + (i * 64 + lane) * 16);
    hit |= special(x.x) || special(x.y) || special(x.z) || special(x.w);
  }
  return __ballot(hit) != 0;
}

DEV float inverse(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }   // a row that sees nothing: 0

// One walk with the running maximum and sum of a softmax: S = K Qᵀ of 32 keys by 32
// rows, P = exp2(S - max) rounded to bf16 for the product (as in the other
// attention kernels here; two bf16 halves of P would take the output's error from
// 2.3e-3 to 1.7e-3 and cost 2 to 6 %), O += V P, all sums in fp32. Loads of the next
// tile are under way while one is worked on.
// One new token is bound by HBM: 64 sequences of 200 to 4,096 95 us, 131,071 tokens
// 87 us, 64 of 2,048 89 us (5.8, 6.2 and 6.0 TB/s; a read-only stream reaches 6.0 to
// 7.1). 16 trees of 24 drafts over 1,000 to 3,001 tokens take 33 us: 5 of dependent
// loads (lengths, cuts, table, page) before the first tile is under way and 2 until it is
// there, then up to nine tiles of 32 keys a group one after another at 2.3 (0.5 to
// issue loads, 1.1 for scores and softmax, 0.6 for the second product, beside another
// workgroup on the compute unit), 1 to merge the groups, 3 to launch and end. Two
// blocks of rows of heads of 128 take all 256 registers and spill 3, four spill 5.
template <int HD, int RB>
__global__ __launch_bounds__(256, RB == 1 ? 1 : 2) void tree_kernel(TreeArgs a) {
  using W = Walk<HD, RB>;
  using S = Shape<HD>;
  constexpr int KT = W::KT;
  __shared__ __attribute__((aligned(1024))) char smem_raw[W::GROUPS * W::RING];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lq = lane & 31, g = lane >> 5, G = a.H / a.Hkv;
  const int rw = wave % RB, group = wave / RB;   // block of 32 rows, group of the workgroup
  lds_char_t* ring = (lds_char_t*)smem_raw + group * W::RING;
  const float sc = LOG2E / sqrtf((float)HD);
  Line<W> line;
  line.init(a);
  if (blockIdx.x == 0 && wave == 0 && !line.planned) {   // for the launch that joins
    if (lane < a.n_seq) a.plan[lane] = line.base;
    if (lane == 0) store_cuts(a, line.sum, line.cuts);
  }
  const bool solo = line.cuts.x == SOLO, dealt = line.cuts.x == DEALT;
  const int me = solo ? blockIdx.x * 4 + wave : blockIdx.x;
  const int first = solo ? 0 : group, step = solo ? 1 : W::GROUPS;
  int p, end;
  if (dealt) {
    p = me;
    end = min(me + 1, line.sum);
  } else {
    if ((long)me * line.cuts.y >= line.sum) return;
    p = line.bound(a, me);
    end = line.bound(a, me + 1);
  }
  while (p < end) {
    int before;
    const int s = line.find(a, p, &before);
    const Seq q = line.seq(a, s);
    int seg, f0, f1;
    if (dealt) {
      const int n = pieces_of<W>(q.t, line.cuts.y);
      seg = (p - before) / n;
      const int k = p - before - seg * n;
      const int least = q.t / n, more = q.t - least * n;   // tiles of a piece; pieces that have one more
      f0 = k * least + min(k, more);
      f1 = f0 + least + (k < more);
      p = end;
    } else {
      seg = (p - before) / q.t;
      const int from = before + seg * q.t;
      f0 = p - from;
      f1 = min(end - from, q.t);
      p = from + f1;
    }
    const int block = seg / a.Hkv, j = seg - block * a.Hkv;
    // a block of rows without a mask needs the new tokens up to its last only
    const int last = min(((block + 1) * W::ROWS - 1) / G, q.n - 1);
    const int f_end = a.mask ? f1 : min(f1, q.tc + last / KT + 1);

    Keys<HD, RB> keys;
    keys.init(a, s, q, j, f0);
    auto stage = [&](int it) { return ring + it % W::STAGES * 2 * W::TB; };
    if (f0 + first < f_end) keys.issue(f0 + first, stage(0), rw, false);
    uint64_t next_seen = keys.seen;
    const int row = block * W::ROWS + 32 * rw + lq;
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

    for (int it = 0; f0 + it * step < f_end; ++it) {
      const int f = f0 + it * step + first;
      wait_vmcnt<0>();
      __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's reads of the stage that the next loads overwrite are done
      if constexpr (RB > 1) block_barrier();
      const uint64_t there = next_seen;
      if (f + step < f_end) {
        int refs = keys.refs;
        asm volatile("" : "+v"(refs));   // not waited for before
        keys.issue(f + step, stage(it + 1), rw, __builtin_amdgcn_readfirstlane(refs) == 1);
        next_seen = keys.seen;
      }
      if (f >= f_end) continue;
      // 32 keys at a time: the scores of 64 at once would leave too few registers
#pragma unroll 1
      for (int sub = 0; sub < KT / 32; ++sub) {
        const lds_char_t* Ks = stage(it) + sub * 64 * HD;
        const lds_char_t* Vs = Ks + W::TB;
        // the keys that this lane's row sees
        uint32_t mine = (uint32_t)(there >> (32 * sub));
        const bool drafted = f >= q.tc;
        if (drafted) {
          const int d0 = (f - q.tc) * KT + 32 * sub;
          if (a.mask) mine &= d0 / 32 < a.mask_words ? (uint32_t)a.mask[token * a.mask_words + d0 / 32] : 0u;
          else if (i < d0 + 31) mine &= i < d0 ? 0u : (2u << (i - d0)) - 1;
        }
        if (__ballot(mine != 0) == 0) continue;
        const bool all = __ballot(mine != ~0u) == 0;
        const bool bad = drafted && !all && not_finite<HD>(Vs, lane);

        floatx16 x;
        zero(x);
#pragma unroll
        for (int k = 0; k < S::KS; ++k) x = mfma32(read_row<HD>(Ks, lq, 2 * k + g), qf[k], x);
        float mt = -INFINITY;
        if (all) {
#pragma unroll
          for (int e = 0; e < 16; ++e) mt = fmaxf(mt, x[e]);
        } else {
          const uint32_t bits = mine >> (4 * g);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            x[e] = bits >> acc_row(e, 0) & 1 ? x[e] : -INFINITY;
            mt = fmaxf(mt, x[e]);
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
        for (int e = 0; e < 16; ++e) {
          const float w = fast_exp2(fmaf(x[e], sc, -shift));
          x[e] = w;
          rsum += w;
        }
        l_run += sum32(rsum);
        if (!bad) {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const bf16x8 pf = acc_slots(x, hh);
#pragma unroll
            for (int d = 0; d < S::DT; ++d) o[d] = mfma32(read_tr<HD>(Vs, 32 * d, 16 * hh, lane), pf, o[d]);
          }
          continue;
        }
        // one token after another, for the rows that see it (0 times infinity would reach the others)
#pragma unroll 1
        for (int k = 0; k < 32; ++k) {
          float w = 0.0f;
#pragma unroll
          for (int e = 0; e < 16; ++e) w = (k & ~4) == acc_row(e, 0) ? x[e] : w;
          w = __shfl(w, lq + (k >> 2 & 1) * 32);
          const bool sees = mine >> k & 1;
#pragma unroll
          for (int d = 0; d < S::DT; ++d)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint2 v = __builtin_bit_cast(
                  uint2, *reinterpret_cast<const LDS_AS floatx2*>(Vs + unit<HD>(k, 4 * d + c) * 16 + 8 * g));
              const float y[4] = {lo_f(v.x), hi_f(v.x), lo_f(v.y), hi_f(v.y)};
#pragma unroll
              for (int e = 0; e < 4; ++e) o[d][4 * c + e] += w * (sees ? y[e] : 0.0f);
              __builtin_amdgcn_sched_barrier(0);   // one read at a time: this path keeps few registers
            }
        }
      }
    }

    // columns 32 d.. of O that this wave has in the end
    auto has = [&](int d) { return W::GROUPS == 1 || solo || d / W::PER == group; };
    if constexpr (W::GROUPS > 1) {
      if (!solo) {
        // the groups' results through LDS, joined in order, each by the group that has its columns
        __syncthreads();
        auto kept = [&](int of) { return (lds_char_t*)smem_raw + (of * RB + rw) * W::KEEP; };
        auto column = [&](int of, int d) { return kept(of) + 512 + (d - (d / W::PER > of ? W::PER : 0)) * 4096 + lane * 16; };
        const int groups = min(W::GROUPS, max(f_end - f0, 1));   // that had a tile
        if (group < groups) {
          *reinterpret_cast<LDS_AS floatx2*>(kept(group) + lane * 8) = floatx2{m_run, l_run};
#pragma unroll
          for (int d = 0; d < S::DT; ++d)
            if (d / W::PER != group) {
#pragma unroll
              for (int c = 0; c < 4; ++c)
                *reinterpret_cast<lds_v4f32_t*>(column(group, d) + c * 1024) =
                    v4f32{o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]};
            }
        }
        __syncthreads();
        float m = -INFINITY, l = 0.0f, weight[W::GROUPS];
#pragma unroll
        for (int k = 0; k < W::GROUPS; ++k) {
          weight[k] = -INFINITY;
          if (k < groups) {
            weight[k] = reinterpret_cast<const LDS_AS floatx2*>(kept(k) + lane * 8)->x;
            m = fmaxf(m, weight[k]);
          }
        }
#pragma unroll
        for (int k = 0; k < W::GROUPS; ++k)
          if (k < groups) {
            const float lk = reinterpret_cast<const LDS_AS floatx2*>(kept(k) + lane * 8)->y;
            // (sums of rows that met a NaN have no maximum, but count)
            l += weight[k] == -INFINITY ? lk : lk * fast_exp2(weight[k] - m);
            weight[k] = weight[k] == -INFINITY ? 0.0f : fast_exp2(weight[k] - m);
          }
        m_run = m;
        l_run = l;
#pragma unroll
        for (int d = 0; d < S::DT; ++d) {
          if (d / W::PER != group) continue;
          const floatx16 own = o[d];
          zero(o[d]);
#pragma unroll
          for (int k = 0; k < W::GROUPS; ++k) {
            if (k >= groups) continue;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              v4f32 y = {own[4 * c], own[4 * c + 1], own[4 * c + 2], own[4 * c + 3]};
              if (k != d / W::PER) y = *reinterpret_cast<const lds_v4f32_t*>(column(k, d) + c * 1024);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[d][4 * c + e] += y[e] * weight[k];
            }
          }
        }
        __syncthreads();   // the rings are the next segment's
      }
    } else {
      __syncthreads();
    }
    if (!on) continue;
    if (f0 == 0 && f1 == q.t) {
      const float inv = inverse(l_run);
      bf16_t* out = a.out + (token * a.H + h) * HD;
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
        if (has(d)) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint2*>(out + 32 * d + 8 * c + 4 * g) =
                make_uint2(pack2(o[d][4 * c] * inv, o[d][4 * c + 1] * inv),
                           pack2(o[d][4 * c + 2] * inv, o[d][4 * c + 3] * inv));
        }
      if (g == 0 && has(0) && a.lse) a.lse[(size_t)h * a.n_rows + token] = (m_run + log2f(l_run)) * LN2;
      continue;
    }
    // a share of the line has at most two cut segments: one that begins in it, one that does not
    const int prows = part_rows(a, W::ROWS), pr = 32 * rw + lq;
    float* part = a.part + (dealt ? (size_t)me : 2 * (size_t)me + (f0 == 0)) * part_floats(a, W::ROWS, HD);
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
      if (has(d)) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<float4*>(part + (size_t)pr * HD + 32 * d + 8 * c + 4 * g) =
              make_float4(o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]);
      }
    if (g == 0 && has(0)) {
      part[(size_t)prows * HD + pr] = m_run;
      part[(size_t)prows * HD + prows + pr] = l_run;
    }
  }
}

// The parts of a cut segment's row of one query head, WPR waves a row: lane k
// holds part k's maximum and sum (the maximum's weight afterwards), then HD/8
// lanes take the row's elements, 8 each, and the groups of them the parts in turn.
// Dependent loads (sequence, cuts, maxima, elements) bound it: 5 us for 64 tokens'
// rows or 16 rows of 32 parts, 7 for 7,284 rows of 64.
template <int HD, int RB, int WPR>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void tree_join_kernel(TreeArgs a) {
  using W = Walk<HD, RB>;
  constexpr int LANES = HD / 8, GROUPS = 64 / LANES;
  __shared__ float other[WPR][HD + 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = a.H / a.Hkv;
  const long team = (long)blockIdx.y * gridDim.x + blockIdx.x, at = WPR == 1 ? team * 4 + wave : team;
  const int token = (int)(at / a.H), h = (int)(at - (long)token * a.H);
  if (token >= a.n_rows) return;
  // the sequence that has the row: the last one that begins at or before it
  int s = -1;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const uint64_t b = __ballot(s0 + lane < a.n_seq && a.starts[min(s0 + lane, a.n_seq)] <= token);
    if (b) s = s0 + 63 - __builtin_clzll(b);
  }
  if (s < 0) return;
  const int before = a.plan[s];
  const Cuts cuts = {a.plan[a.n_seq + 1], a.plan[a.n_seq + 2]};
  if (a.plan[a.n_seq] == 0) return;
  const Seq q = seq_of<W>(a, s);
  const int i = token - q.start;
  if (i < 0 || i >= q.n) return;
  const int j = h / G, r = i * G + h - j * G, block = r / W::ROWS, row = r - block * W::ROWS;
  const int prows = part_rows(a, W::ROWS);
  const size_t floats = part_floats(a, W::ROWS, HD);
  int parts;
  const float* part0;
  const bool dealt = cuts.x == DEALT;
  if (dealt) {
    parts = pieces_of<W>(q.t, cuts.y);
    if (parts < 2) return;
    part0 = a.part + (size_t)(before + (block * a.Hkv + j) * parts) * floats;
  } else {
    const int from = before + (block * a.Hkv + j) * q.t;
    // cuts w0..w1 lie inside the segment, so shares w0 - 1..w1 have its parts
    const int w0 = (from + W::SLACK) / cuts.y + 1, w1 = (from + q.t - W::SLACK - 1) / cuts.y;
    if (w1 < w0) return;
    parts = w1 - w0 + 2;
    part0 = a.part + 2 * (size_t)(w0 - 1) * floats;
  }
  // part k's place: of the line's, the first begins in its share, the others do not
  auto place = [&](int k) { return part0 + (dealt ? (size_t)k : 2 * (size_t)k + (k == 0)) * floats; };
  // this wave's parts
  const int k_begin = (int)((long)parts * wave / WPR) * (WPR > 1), k_end = WPR > 1 ? (int)((long)parts * (wave + 1) / WPR) : parts;
  float m = -INFINITY;
  for (int k = k_begin + lane; k < k_end; k += 64) m = fmaxf(m, place(k)[(size_t)prows * HD + row]);
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const int c = lane % LANES * 8;
  float l = 0.0f, o[8] = {};
  for (int k0 = k_begin; k0 < k_end; k0 += 64) {
    float wgt = 0.0f;
    if (k0 + lane < k_end) {
      const float* p = place(k0 + lane) + (size_t)prows * HD;
      const float mk = p[row], lk = p[prows + row];
      wgt = mk == -INFINITY ? 0.0f : fast_exp2(mk - m);
      l += mk == -INFINITY ? lk : wgt * lk;
    }
    const int n = min(64, k_end - k0);
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
  if constexpr (WPR > 1) {
    if (lane < LANES) {
#pragma unroll
      for (int e = 0; e < 8; ++e) other[wave][c + e] = o[e];
      if (lane == 0) {
        other[wave][HD] = m;
        other[wave][HD + 1] = l;
      }
    }
    __syncthreads();
    if (wave > 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WPR; ++w) top = fmaxf(top, other[w][HD]);
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) {
      const float mw = other[w][HD], lw = other[w][HD + 1], f = mw == -INFINITY ? 0.0f : fast_exp2(mw - top);
      l += mw == -INFINITY ? lw : f * lw;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += f * other[w][c + e];
    }
    m = top;
  }
  if (lane >= LANES) return;
  const float inv = inverse(l);
  *reinterpret_cast<uint4*>(a.out + ((size_t)token * a.H + h) * HD + c) =
      make_uint4(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv), pack2(o[4] * inv, o[5] * inv),
                 pack2(o[6] * inv, o[7] * inv));
  if (c == 0 && a.lse) a.lse[(size_t)h * a.n_rows + token] = (m + log2f(l)) * LN2;
}

// A row's place in its sequence: behind the cached tokens and the new ones that it
// sees besides itself.
__global__ __launch_bounds__(256) void tree_positions_kernel(TreeArgs a, int32_t* positions) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= a.n_rows) return;
  int lo = 0, hi = a.n_seq;   // sequences that begin at or before the row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.starts[mid] <= row) lo = mid + 1;
    else hi = mid;
  }
  int position = 0;
  if (lo > 0) {
    const int start = clampi(a.starts[lo - 1], 0, a.n_rows), end = clampi(a.starts[lo], start, a.n_rows);
    if (row >= start && row < end) {
      int before = row - start;
      if (a.mask) {
        before = -1;
        for (int k = 0; k < a.mask_words; ++k) before += __popc(a.mask[(size_t)row * a.mask_words + k]);
      }
      position = clampi(a.lens[lo - 1], 0, a.max_pages * a.ps) + max(before, 0);
    }
  }
  positions[row] = position;
}

template <int V>
using Int = std::integral_constant<int, V>;

// f(head size, blocks of rows of a workgroup): as many as a sequence's rows fill. 16 sequences of 1,000 to 3,000
// tokens, heads of 128, with 1, 2, 4 blocks: 24 rows 38, 37, 42 us; 48 rows 52, 40, 44; 96 rows 77, 57, 49; heads of
// 64: 24 rows 35, 32, 42; 48 rows 51, 36, 46; 100 rows 89, 57, 51.
template <class Fn>
auto with_walk(const TreeArgs& a, Fn f) {
  const long rows = (long)a.max_new * (a.H / a.Hkv);
  if (a.hd == 128) return rows <= 32 ? f(Int<128>{}, Int<1>{}) : rows <= 64 ? f(Int<128>{}, Int<2>{}) : f(Int<128>{}, Int<4>{});
  return rows <= 32 ? f(Int<64>{}, Int<1>{}) : rows <= 64 ? f(Int<64>{}, Int<2>{}) : f(Int<64>{}, Int<4>{});
}

// `teams` workgroups of 256 threads: a dimension of a grid has less than 2^32 threads, which 2^26 rows reach
dim3 join_grid(long teams) {
  return teams < 1l << 24 ? dim3((unsigned)teams) : dim3((unsigned)((teams + 1) / 2), 2);
}

// Tiles of all sequences at their longest, and of one of their segments. Blocks of rows are bounded by the rows, too:
// one piece of a prompt among many single tokens has many, the others have one each.
template <class W>
double most_tiles(const TreeArgs& a, double* segment) {
  *segment = std::ceil((double)a.max_pages * a.ps / W::KT) + std::ceil((double)a.max_new / W::KT);
  const double G = a.H / a.Hkv;
  return *segment * a.Hkv *
         std::min(a.n_seq * std::ceil(a.max_new * G / W::ROWS), std::floor(a.n_rows * G / W::ROWS) + a.n_seq);
}

}  // namespace

size_t tree_workspace(const TreeArgs& a, size_t* part_at) {
  return with_walk(a, [&](auto hd, auto rb) -> size_t {
    using W = Walk<decltype(hd)::value, decltype(rb)::value>;
    double segment;
    if (most_tiles<W>(a, &segment) > 2e9) return 0;   // tiles are counted in 32 bits
    *part_at = (((size_t)a.n_seq + 3) * sizeof(int32_t) + 255) / 256 * 256;
    return *part_at + (segment > W::LEAST ? 2 * (size_t)W::MOST * part_floats(a, W::ROWS, W::HEAD) * sizeof(float) : 0);
  });
}

hipError_t launch_tree_positions(const TreeArgs& a, int32_t* positions, hipStream_t s) {
  if (a.n_rows < 1) return hipSuccess;
  hipLaunchKernelGGL(tree_positions_kernel, dim3((a.n_rows + 255) / 256), dim3(256), 0, s, a, positions);
  return hipGetLastError();
}

hipError_t launch_tree(const TreeArgs& a, hipStream_t s) {
  if (a.n_rows < 1) return hipSuccess;
  return with_walk(a, [&](auto hd, auto rb) -> hipError_t {
    constexpr int HD = decltype(hd)::value, RB = decltype(rb)::value;
    using W = Walk<HD, RB>;
    double segment;
    const double tiles = most_tiles<W>(a, &segment);
    if (a.n_seq > 64) hipLaunchKernelGGL((tree_plan_kernel<W>), dim3(1), dim3(64), 0, s, a);
    const unsigned teams = (unsigned)std::min((double)W::TEAMS, tiles);
    hipLaunchKernelGGL((tree_kernel<HD, RB>), dim3(teams), dim3(256), 0, s, a);
    if (segment > W::LEAST) {
      const long rows = (long)a.n_rows * a.H;
      // 8 waves a row where rows are few and their parts many: one token over 131,071 of one key/value head with 8 query
      // heads 48 us with one wave, 27 with 8, of 8 heads with 16 94 and 92; 16 trees of 24 drafts 40 and 68
      if (rows <= 512) hipLaunchKernelGGL((tree_join_kernel<HD, RB, 8>), dim3((unsigned)rows), dim3(512), 0, s, a);
      else hipLaunchKernelGGL((tree_join_kernel<HD, RB, 1>), join_grid((rows + 3) / 4), dim3(256), 0, s, a);
    }
    return hipGetLastError();
  });
}
