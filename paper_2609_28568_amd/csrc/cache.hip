// The pages of a cache of keys and values: forking, appending, compacting. A
// page is one piece of memory in each layer, [2: keys, values][Hkv][ps][hd], so
// that a key/value head's tokens are consecutive rows for the attention and a
// page moves as one run of bytes.
//
// The books (table, lengths, counts of holders) are kept on the device: which
// pages are taken follows from the counts alone, so results do not depend on
// which workgroup comes first. Books of a call are one launch of few
// workgroups, bound by a few dependent memory round trips (forking 16 sequences
// of 1,500 tokens 2.0 us, appending to them 5.6; finding which of 15 sequences' pages
// move 3.4, with some hundred pages; the counts of all pages are passed over two and
// three times, which with 57,344 of them takes an append 7 us more); the tokens and
// pages they name are moved by a second one, bound by HBM (prompts, 561 MB read and
// written, 91 us: 6.2 TB/s; 175 MB of moved pages 30 us: 5.8 TB/s).
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace {

constexpr int BOOK = 1024;   // threads of the one workgroup that keeps the books
constexpr int WAVES = BOOK / 64;
struct __attribute__((packed, aligned(4))) Four { int32_t r[4]; };

// Exclusive prefix sum of v over the workgroup's waves, in their order (v the
// wave's own); *total: the sum. `parts`: WAVES ints of LDS of their own.
DEV int waves_before(int v, int* parts, int* total) {
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) parts[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int p = parts[w];
    before += w < wave ? p : 0;
    all += p;
  }
  *total = all;
  return before;
}
// ... over its threads.
DEV int threads_before(int v, int* parts, int* total) {
  const int lane = threadIdx.x & 63;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return waves_before(__builtin_amdgcn_readlane(x, 63), parts, total) + x - v;
}

// The pages of a wave's run, four a lane, 256 a step: f(first of the lane's four,
// a bit for each of them that someone holds, bits that are pages).
template <class Fn>
DEV void each_page(const CacheArgs& c, Fn f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int run = ((c.n_pages + WAVES * 256 - 1) / (WAVES * 256)) * 256, p1 = min((wave + 1) * run, c.n_pages);
  for (int p0 = wave * run; p0 < p1; p0 += 256) {
    const int p = p0 + 4 * lane;
    uint32_t held = 0, there = 0;
    int r[4] = {0, 0, 0, 0};
    if (p + 4 <= p1) {
      const Four q = *reinterpret_cast<const Four*>(c.refs + p);
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = q.r[k];
      there = 15;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (p + k < p1) {
          r[k] = c.refs[p + k];
          there |= 1u << k;
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) held |= r[k] != 0 ? 1u << k : 0u;
    f(p, held & there, there);
  }
}
// How many of a lane's four pages that `bits` names there are in the lanes before; *all: in the wave.
DEV int lanes_before(uint32_t bits, int* all) {
  int before = 0, sum = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint64_t b = __ballot(bits >> k & 1);
    before += __popcll(b & ((1ull << (threadIdx.x & 63)) - 1));
    sum += __popcll(b);
  }
  *all = sum;
  return before;
}

DEV int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// A column of the table (one page of every sequence) follows from that column
// alone, so a workgroup takes some of them, reads the old ones into LDS and
// writes the new ones. Lengths go with the first workgroup.
__global__ __launch_bounds__(256) void fork_kernel(CacheArgs c, const int32_t* src, const int32_t* keep, int cols) {
  extern __shared__ int32_t old[];
  const int col0 = blockIdx.x * cols, n = c.n_seq * cols;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int col = col0 + i % cols;
    old[i] = col < c.max_pages ? c.table[(size_t)(i / cols) * c.max_pages + col] : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int s = i / cols, k = i - s * cols, col = col0 + k;
    if (col >= c.max_pages) continue;
    const int from = src[s];
    int page = (unsigned)from < (unsigned)c.n_seq ? old[from * cols + k] : -1;
    if (keep && (long)col * c.ps >= keep[s]) page = -1;
    const int was = old[i];
    if (page == was) continue;
    c.table[(size_t)s * c.max_pages + col] = page;
    if ((unsigned)was < (unsigned)c.n_pages) atomicSub(c.refs + was, 1);
    if ((unsigned)page < (unsigned)c.n_pages) atomicAdd(c.refs + page, 1);
  }
  if (blockIdx.x) return;
  __syncthreads();
  for (int s = threadIdx.x; s < c.n_seq; s += 256) old[s] = c.lens[s];
  __syncthreads();
  for (int s = threadIdx.x; s < c.n_seq; s += 256) {
    const int from = src[s];
    int len = (unsigned)from < (unsigned)c.n_seq ? old[from] : 0;
    if (keep) len = min(len, max(keep[s], 0));
    c.lens[s] = len;
  }
}

// What sequence s appends: tokens, and the place of the first.
struct Add {
  int len, n;
};
DEV Add adding(const CacheArgs& c, const AppendArgs& a, int s) {
  Add r;
  r.len = clampi(c.lens[s], 0, c.max_pages * c.ps);
  const int b = clampi(a.starts[s], 0, a.n_rows), e = clampi(a.starts[s + 1], b, a.n_rows);
  r.n = min(e - b, a.max_new);
  if (a.counts) r.n = clampi(a.counts[s], 0, a.path ? a.max_new : r.n);
  return r;
}

// Pages for the new tokens: how many each sequence needs, which are free, and
// the i-th needed is the i-th free one. Leaves a record (length, tokens, shared
// page, its copy) for every sequence and the list of those that copy.
__global__ __launch_bounds__(BOOK) void append_book_kernel(CacheArgs c, AppendArgs a) {
  __shared__ int32_t end[CACHE_MAX_SEQ], shared_page[CACHE_MAX_SEQ], first_col[CACHE_MAX_SEQ];
  __shared__ int parts[3][WAVES];
  __shared__ int copies;
  int32_t* head = c.scratch;
  int4* rec = reinterpret_cast<int4*>(c.scratch + CACHE_HEADER);
  int32_t* copying = c.scratch + CACHE_HEADER + 4 * c.n_seq;   // [n_seq] at most n_pages
  int32_t* freed = copying + c.n_pages;
  const int tid = threadIdx.x;
  if (tid == 0) copies = 0;

  int nfree = 0;   // of the wave's run of pages
  each_page(c, [&](int, uint32_t held, uint32_t there) {
    int n;
    lanes_before(there & ~held, &n);
    nfree += n;
  });

  const int each = (c.n_seq + BOOK - 1) / BOOK;
  int need = 0, over = 0;
  for (int k = 0; k < each; ++k) {
    const int s = tid * each + k;
    if (s >= c.n_seq) break;
    const Add d = adding(c, a, s);
    const int at = d.len / c.ps, from = (d.len + c.ps - 1) / c.ps, to = (int)(((long)d.len + d.n + c.ps - 1) / c.ps);
    int page = -1;
    if (d.n > 0 && d.len % c.ps) {
      page = c.table[(size_t)s * c.max_pages + at];
      if ((unsigned)page >= (unsigned)c.n_pages || c.refs[page] < 2) page = -1;
    }
    shared_page[s] = page;
    first_col[s] = from;
    need += (page >= 0) + to - from;
    end[s] = need;   // within the thread's run of sequences
    over += max(0, to - c.max_pages);
    rec[s] = make_int4(d.len, d.n, page, -1);
  }
  int total, nfrees, overs;
  const int before = threads_before(need, parts[0], &total);
  int rank = waves_before(nfree, parts[1], &nfrees);
  threads_before(over, parts[2], &overs);
  const int missing = max(0, total - nfrees) + overs;
  if (tid == 0) *c.missing = missing;
  if (missing) {   // nothing to move
    for (int s = tid; s < c.n_seq; s += BOOK) rec[s] = make_int4(0, 0, -1, -1);
    if (tid == 0) head[0] = 0;
    return;
  }
  for (int k = 0; k < each; ++k) {
    const int s = tid * each + k;
    if (s >= c.n_seq) break;
    end[s] += before;
    const int4 r = rec[s];
    c.lens[s] = r.x + r.y;
    if (r.z >= 0) copying[atomicAdd(&copies, 1)] = s;
  }
  each_page(c, [&](int p, uint32_t held, uint32_t there) {
    int n, at = rank + lanes_before(there & ~held, &n);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((there & ~held) >> k & 1) {
        if (at < total) freed[at] = p + k;
        ++at;
      }
    rank += n;
  });
  __syncthreads();
  if (tid == 0) head[0] = copies;
  for (int i = tid; i < total; i += BOOK) {
    int lo = 0, hi = c.n_seq - 1;   // the first sequence whose end lies past i
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (end[mid] > i) hi = mid;
      else lo = mid + 1;
    }
    const int s = lo, k = i - (s ? end[s - 1] : 0), page = freed[i], was = shared_page[s];
    const int col = first_col[s] + k - (was >= 0);
    c.table[(size_t)s * c.max_pages + col] = page;
    c.refs[page] = 1;
    if (was >= 0 && k == 0) {
      atomicSub(c.refs + was, 1);
      reinterpret_cast<int32_t*>(rec + s)[3] = page;
    }
  }
}

DEV size_t page_at(const CacheArgs& c, int layer, int page) {   // in elements
  return ((size_t)layer * c.n_pages + page) * (2 * (size_t)c.Hkv * c.ps * c.hd);
}

// The sequence that has row `row`: the last one that begins at or before it, -1
// where none does. By all lanes, in one load of starts, or two past 64 sequences.
DEV int seq_of_row(const int32_t* starts, int n_seq, int row) {
  const int lane = threadIdx.x & 63, step = (n_seq + 63) / 64;
  const int i = lane * step;
  int s = __popcll(__ballot(i < n_seq && starts[min(i, n_seq)] <= row)) - 1;
  if (step > 1 && s >= 0) {
    s *= step;
    const int j = s + lane;
    s += __popcll(__ballot(lane < step && j < n_seq && starts[min(j, n_seq)] <= row)) - 1;
  }
  return s;
}

// Tokens into their places, a wave one token of one layer (of the rows, or of
// the path's entries: a wave each of n_seq * max_new, 63 single tokens beside a
// piece of 2,048 in 28 layers were 789 us a pass, 81 so), and behind those blocks the shared pages' tokens, a wave one head of one page. Written past the
// caches: prompts of a batch, 561 MB read and written, 115 us a pass through
// them, 106 past them (5.3 TB/s); with 8 tokens a wave 143 and 136.
__global__ __launch_bounds__(64) void append_move_kernel(CacheArgs c, AppendArgs a, int items, int nt) {
  const int4* rec = reinterpret_cast<const int4*>(c.scratch + CACHE_HEADER);
  const int lane = threadIdx.x;
  const int hu = c.hd / 8, units = 2 * c.Hkv * hu;   // 16-byte units of a head, of a token
  if ((int)blockIdx.x < nt) {
    const int layer = blockIdx.y;
    for (int item = blockIdx.x; item < items; item += nt) {
      const int s = a.path ? item / a.max_new : seq_of_row(a.starts, c.n_seq, item);
      if (s < 0) continue;
      const int4 r = rec[s];
      const int b = clampi(a.starts[s], 0, a.n_rows), e = clampi(a.starts[s + 1], b, a.n_rows);
      const int i = a.path ? item - s * a.max_new : item - b;
      if ((unsigned)i >= (unsigned)r.y) continue;
      const int row = a.path ? a.path[item] : i;
      const int pos = r.x + i, page = c.table[(size_t)s * c.max_pages + pos / c.ps];
      if ((unsigned)row >= (unsigned)min(e - b, a.max_rows) || (unsigned)page >= (unsigned)c.n_pages) continue;
      const uint4* from = reinterpret_cast<const uint4*>(
          a.qkv + layer * a.layer_stride + (size_t)(b + row) * (a.H + 2 * c.Hkv) * c.hd + (size_t)a.H * c.hd);
      uint4* to = reinterpret_cast<uint4*>(c.pages + page_at(c, layer, page) + (size_t)(pos % c.ps) * c.hd);
      constexpr int FLIGHT = 4;
      for (int u0 = lane; u0 < units; u0 += 64 * FLIGHT) {
        uint4 v[FLIGHT];
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) v[k] = u0 + 64 * k < units ? from[u0 + 64 * k] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
          const int u = u0 + 64 * k, h = u / hu;
          if (u < units) st_stream(to + (size_t)h * c.ps * hu + (u - h * hu), v[k]);
        }
      }
    }
    return;
  }
  const int32_t* copying = c.scratch + CACHE_HEADER + 4 * c.n_seq;
  const int layer = blockIdx.y, n = c.scratch[0] * 2 * c.Hkv;
  for (int i = blockIdx.x - nt; i < n; i += gridDim.x - nt) {
    const int s = copying[i / (2 * c.Hkv)], h = i % (2 * c.Hkv);
    const int4 r = rec[s];
    const uint4* from = reinterpret_cast<const uint4*>(c.pages + page_at(c, layer, r.z) + (size_t)h * c.ps * c.hd);
    uint4* to = reinterpret_cast<uint4*>(c.pages + page_at(c, layer, r.w) + (size_t)h * c.ps * c.hd);
    const int m = r.x % c.ps * hu;
#pragma unroll 4
    for (int u = lane; u < m; u += 64) to[u] = from[u];
  }
}

// Which page moves where: the k-th page in use at or above their number to the
// k-th free one below.
__global__ __launch_bounds__(BOOK) void compact_book_kernel(CacheArgs c) {
  __shared__ int parts[3][WAVES];
  int32_t* head = c.scratch;
  int32_t* holes = c.scratch + CACHE_HEADER + 4 * c.n_seq;   // the k-th move's target
  int32_t* from = holes + c.n_pages;                         // ... and source
  const int tid = threadIdx.x;
  int mine = 0, used, nholes, moves;
  each_page(c, [&](int, uint32_t held, uint32_t) {
    int n;
    lanes_before(held, &n);
    mine += n;
  });
  waves_before(mine, parts[0], &used);   // pages in use
  // of pages below `used` those that are free, of the others those in use
  auto below = [&](int p) { return p >= used ? 0u : p + 4 <= used ? 15u : (1u << (used - p)) - 1; };
  int hole = 0, move = 0;
  each_page(c, [&](int p, uint32_t held, uint32_t there) {
    int n;
    lanes_before(there & ~held & below(p), &n);
    hole += n;
    lanes_before(held & ~below(p), &n);
    move += n;
  });
  hole = waves_before(hole, parts[1], &nholes);
  move = waves_before(move, parts[2], &moves);
  each_page(c, [&](int p, uint32_t held, uint32_t there) {
    const uint32_t h = there & ~held & below(p), m = held & ~below(p);
    int nh, nm, at = hole + lanes_before(h, &nh), to = move + lanes_before(m, &nm);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (h >> k & 1) holes[at++] = p + k;
      if (m >> k & 1) from[to++] = p + k;
    }
    hole += nh;
    move += nm;
  });
  if (tid == 0) {
    head[0] = moves;
    head[1] = used;
  }
  __syncthreads();
  for (int k = tid; k < moves; k += BOOK) {
    const int a = from[k], b = holes[k];
    c.refs[b] = c.refs[a];
    c.refs[a] = 0;
  }
}

// The pages' contents and the table's entries. A move's target is found from its
// source by a search in the sorted list.
__global__ __launch_bounds__(256) void compact_move_kernel(CacheArgs c) {
  const int32_t* head = c.scratch;
  const int32_t* holes = c.scratch + CACHE_HEADER + 4 * c.n_seq;
  const int32_t* from = holes + c.n_pages;
  const int moves = head[0], used = head[1];
  if (moves == 0) return;
  const long entries = (long)c.n_seq * c.max_pages, step = (long)gridDim.x * 256;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < entries; i += step) {
    const int p = c.table[i];
    if (p < used || p >= c.n_pages) continue;
    int lo = 0, hi = moves - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (from[mid] >= p) hi = mid;
      else lo = mid + 1;
    }
    if (from[lo] == p) c.table[i] = holes[lo];
  }
  const int units = 2 * c.Hkv * c.ps * c.hd / 8;   // of a page, a multiple of 256
  const int pieces = (units + 1023) / 1024;
  const long per = (long)c.L * pieces, items = moves * per;
  for (long i = blockIdx.x; i < items; i += gridDim.x) {
    const int k = (int)(i / per), layer = (int)((i - k * per) / pieces);
    const int u0 = (int)(i - k * per - (long)layer * pieces) * 1024;
    const uint4* src = reinterpret_cast<const uint4*>(c.pages + page_at(c, layer, from[k])) + u0;
    uint4* dst = reinterpret_cast<uint4*>(c.pages + page_at(c, layer, holes[k])) + u0;
    const int n = min(4, (units - u0) / 256);
    uint4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)   // (past the caches: 175 MB of pages 53 -> 48 us a pass)
      v[q] = q < n ? ld_stream(src + q * 256 + threadIdx.x) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < n) dst[q * 256 + threadIdx.x] = v[q];
  }
}

}  // namespace

hipError_t launch_cache_fork(const CacheArgs& c, const int32_t* src, const int32_t* keep, hipStream_t s) {
  // columns of a workgroup: 64 KiB of LDS hold them for all sequences, and the lengths afterwards. Few, so that many
  // workgroups share the table: 16 answers of 1,500 tokens begun and appended to 25.3 us with 64, 22.4 with 16 or 4
  const int cols = std::min(16, std::max(1, 16384 / c.n_seq));
  const size_t lds = sizeof(int32_t) * (size_t)c.n_seq * cols;
  hipLaunchKernelGGL(fork_kernel, dim3((c.max_pages + cols - 1) / cols), dim3(256), lds, s, c, src, keep, cols);
  return hipGetLastError();
}

hipError_t launch_cache_append(const CacheArgs& c, const AppendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(append_book_kernel, dim3(1), dim3(BOOK), 0, s, c, a);
  // a grid's dimension has less than 2^32 threads: past 2^20 tokens a layer waves take several
  const int items = a.path ? c.n_seq * a.max_new : a.n_rows, nt = std::min(items, 1 << 20);
  // heads to copy at most; waves that find none cost 0.5 us, and 16 shared pages in 28 layers 22.4 us with 2,048, 18.3
  // with 8,192
  const unsigned nc = (unsigned)std::min((long)c.n_seq * 2 * c.Hkv, std::max(1l, 8192l / c.L));
  hipLaunchKernelGGL(append_move_kernel, dim3(nt + nc, c.L), dim3(64), 0, s, c, a, items, nt);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheArgs& c, hipStream_t s) {
  hipLaunchKernelGGL(compact_book_kernel, dim3(1), dim3(BOOK), 0, s, c);
  hipLaunchKernelGGL(compact_move_kernel, dim3(2048), dim3(256), 0, s, c);
  return hipGetLastError();
}
