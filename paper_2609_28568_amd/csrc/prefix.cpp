// Host side of attention over a shared prefix (prefix.hip): the layout's
// tables and the items that the kernels' workgroups walk, laid down once per
// layout, and the entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <functional>
#include <new>
#include <vector>

#include "prefix.h"

namespace {

constexpr int ROWS = 128, TILE = 64;   // rows of an item, keys (or queries) of a tile

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

struct Tables {
  int N = 0, P = 0, q0 = 0, nq = 0, fslots = 0, kslots = 0;
  double pairs = 0.0;
  std::vector<int32_t> first, end, pos;
  std::vector<PrefixItem> items, kitems;
  std::vector<PrefixJoin> joins, kjoins;
};

int parts_of(int nt, int per) { return 2l * nt > 3l * per ? (nt + per - 1) / per : 1; }

// Cut walks into items of about `per` tiles where they are longer than that by
// half, and put the longest items first, so that no long one starts last.
void deal(const std::vector<PrefixItem>& walks, int per, std::vector<PrefixItem>& items,
          std::vector<PrefixJoin>& joins, int& slots) {
  for (const PrefixItem& w : walks) {
    const int nt = w.f1, parts = parts_of(nt, per);
    if (parts > 1) joins.push_back({w.row, slots, parts, 0});
    for (int i = 0; i < parts; ++i) {
      PrefixItem it = w;
      it.f0 = (int)((long)nt * i / parts);
      it.f1 = (int)((long)nt * (i + 1) / parts);
      it.slot = parts > 1 ? slots++ : -1;
      it.tiles = nt;
      items.push_back(it);
    }
  }
  std::stable_sort(items.begin(), items.end(),
                   [](const PrefixItem& a, const PrefixItem& b) { return a.f1 - a.f0 > b.f1 - b.f0; });
}

// Microseconds that items of about `per` tiles take: each workgroup slot takes
// the next longest item when it is free, an item costs its start and end and
// its tiles, one that shares its walk also its partial result, and those are
// joined by a launch that reads them all. Measured (forward, head size 128, one
// walk of 129 tiles for each of 8 heads, per 5, 6, 8, 12, 16, 24, 40, 129: 21.9,
// 21.3, 21.6, 23.3, 25.7, 30.9, 38.8, 117; this gives 21.3, 21.1, 21.5, 23.4,
// 25.4, 30.7, 39.8, 118; with head size 64 measured 13.2, 13.2, 13.3, 15.0, 16.5,
// 19.7, 24.9, 68.2, chosen 12.8). One sequence of 8,256 tokens, 2 heads, walks of
// 2 to 129 tiles, whole backward for dK/dV's lengths, per 8, 12, 16, 24, 40, 64, 129:
//   head size 128   244, 213, 218, 202, 220, 269, 321; chosen 198
//   head size 64    138, 124, 128, 121, 136, 171, 206; chosen 117
// and its forward, whose choice is off there:
//   head size 128   69, 62, 62, 61, 81, 90, 112; chosen 78
//   head size 64    42, 38, 41, 44, 63, 58, 69; chosen 50
// dQ walks the forward's items: its best lengths were the forward's, within 2 %.
constexpr int CUS = 256;
struct Costs {
  int slots;            // workgroups that run at a time
  double tile;          // a tile of a workgroup with a CU to itself
  double shared;        // ... with all slots taken, where those are two a CU
  double part_bytes;    // of a partial result
};
double estimate(const std::vector<PrefixItem>& walks, int per, int Hkv, const Costs& c) {
  std::vector<int> n;
  long parts = 0;
  for (const PrefixItem& w : walks) {
    const int k = parts_of(w.f1, per);
    if (k > 1) parts += k;
    for (int i = 0; i < k; ++i) n.push_back((int)((long)w.f1 * (i + 1) / k - (long)w.f1 * i / k));
  }
  std::sort(n.rbegin(), n.rend());
  const double wgs = (double)n.size() * Hkv;
  const double tile = wgs <= CUS || c.slots == CUS ? c.tile : std::min(1.0, wgs / c.slots) * c.shared;
  std::vector<double> heap(std::max(1, c.slots / Hkv), 0.0);   // when each of one head's slots is free
  for (int t : n) {
    std::pop_heap(heap.begin(), heap.end(), std::greater<double>());
    heap.back() += 6.0 + t * tile;
    std::push_heap(heap.begin(), heap.end(), std::greater<double>());
  }
  const double traffic = 2.0 * parts * Hkv * c.part_bytes / 4e6;   // written and read, at 4 TB/s
  return *std::max_element(heap.begin(), heap.end()) + (parts ? 4.0 + traffic : 0.0);
}

// The length of items with the least estimate: whole walks, or what shares the
// tiles out over a third of the slots to four times as many.
int item_tiles(const std::vector<PrefixItem>& walks, int Hkv, const Costs& c) {
  long total = 0;
  for (const PrefixItem& w : walks) total += w.f1;
  int best = 1 << 30;
  // plenty of items: only walks longer than a workgroup's share of all tiles are cut (2.2 million single
  // tokens after a prefix of 100, whose keys' walk is 34,375 tiles: backward 46.5 ms with it whole, 1.3 so)
  if (walks.size() > 16384) return (int)std::min((long)best, std::max(2l, total * Hkv / c.slots));
  double least = estimate(walks, best, Hkv, c);
  for (int r = 1; r <= 12; ++r) {
    const long wgs = (long)c.slots * r / 3;
    const int per = (int)std::max(2l, (total * Hkv + wgs - 1) / wgs);
    const double t = estimate(walks, per, Hkv, c);
    if (t < 0.97 * least) {
      least = t;
      best = per;
    }
  }
  return best;
}

Tables lay_out(const qwen3_prefix_config& c, const int32_t* lens) {
  Tables t;
  const int G = c.n_head / c.n_kv_head;
  t.P = c.prefix_len;
  t.N = t.P;
  for (int i = 0; i < c.n_seq; ++i) t.N += lens[i];
  t.q0 = c.prefix_queries ? 0 : t.P;
  t.nq = t.N - t.q0;
  t.first.assign(t.N, 0);
  t.end.assign(t.N, t.N);
  t.pos.resize(t.N);
  for (int i = 0; i < t.P; ++i) t.pos[i] = i;
  for (int i = 0, at = t.P; i < c.n_seq; at += lens[i], ++i)
    for (int k = 0; k < lens[i]; ++k) {
      t.first[at + k] = at;
      t.end[at + k] = at + lens[i];
      t.pos[at + k] = t.P + k;
    }
  for (int i = t.q0; i < t.N; ++i) t.pairs += i < t.P ? i + 1.0 : t.P + (i - t.first[i] + 1.0);

  std::vector<PrefixItem> walks;
  const long rows = (long)t.nq * G;
  for (long r = 0; r < rows; r += ROWS) {
    const int ta = t.q0 + (int)(r / G), tb = t.q0 + (int)((std::min(r + ROWS, rows) - 1) / G);
    PrefixItem w{};
    w.row = (int)r;
    w.npre = (std::min(t.P, tb + 1) + TILE - 1) / TILE;
    w.own = tb >= t.P ? t.first[std::max(ta, t.P)] : 0;
    w.f1 = w.npre + (tb >= t.P ? (tb + 1 - w.own + TILE - 1) / TILE : 0);
    walks.push_back(w);
  }
  const bool narrow = c.head_dim == 64;
  const double bytes[] = {4.0 * prefix_part_floats(c.head_dim, 0), 4.0 * prefix_part_floats(c.head_dim, 2)};
  deal(walks, item_tiles(walks, c.n_kv_head, {2 * CUS, narrow ? 0.5 : 0.87, narrow ? 1.4 : 2.8, bytes[0]}), t.items,
       t.joins, t.fslots);

  walks.clear();
  auto keys = [&](int from, int to) {
    for (int k = from; k < to; k += ROWS) {
      PrefixItem w{};
      w.row = k;
      w.t0 = std::max(k, t.q0);
      w.t1 = t.end[std::min(k + ROWS, to) - 1];
      w.f1 = (w.t1 - w.t0 + TILE - 1) / TILE * G;
      walks.push_back(w);
    }
  };
  keys(0, t.P);
  keys(t.P, t.N);
  deal(walks, item_tiles(walks, c.n_kv_head, {CUS, narrow ? 1.2 : 1.85, 0.0, bytes[1]}), t.kitems, t.kjoins, t.kslots);
  return t;
}

// The device buffer: tables, then the backward's D and the partial results.
struct Places {
  size_t first, end, pos, items, joins, kitems, kjoins, dsum, part, total;
};
Places places(const qwen3_prefix_config& c, const Tables& t) {
  Places p{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += align256(bytes);
    return at;
  };
  p.first = take(t.N * 4ul);
  p.end = take(t.N * 4ul);
  p.pos = take(t.N * 4ul);
  p.items = take(t.items.size() * sizeof(PrefixItem));
  p.joins = take(t.joins.size() * sizeof(PrefixJoin));
  p.kitems = take(t.kitems.size() * sizeof(PrefixItem));
  p.kjoins = take(t.kjoins.size() * sizeof(PrefixJoin));
  p.dsum = take((size_t)t.nq * c.n_head * 4);
  const size_t f = (size_t)t.fslots * c.n_kv_head, k = (size_t)t.kslots * c.n_kv_head;
  p.part = take(4 * std::max({f * prefix_part_floats(c.head_dim, 0), f * prefix_part_floats(c.head_dim, 1),
                              k * prefix_part_floats(c.head_dim, 2)}));
  p.total = std::max(o, (size_t)256);
  return p;
}

// (a reason of up to 15 letters needs no memory)
gpt2_status fail(gpt2_status st, const char* why) {
  set_qwen3_error(why);
  return st;
}

// Bytes of q|k|v, of the rows of out and dout, and of lse.
struct Bytes {
  size_t qkv, rows, lse;
  explicit Bytes(const PrefixArgs& a)
      : qkv((size_t)a.N * (a.H + 2 * a.Hkv) * a.hd * sizeof(bf16_t)),
        rows((size_t)a.nq * a.H * a.hd * sizeof(bf16_t)),
        lse((size_t)a.nq * a.H * sizeof(float)) {}
};

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

std::string prefix_check(const qwen3_prefix_config* c, const int32_t* lens) {
  if (!c) return "null config";
  if (c->n_head < 1 || c->n_kv_head < 1 || c->n_head % c->n_kv_head || c->n_head > 4096)
    return "n_head must be a multiple of n_kv_head, both positive";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->prefix_len < 0 || c->n_seq < 0 || (c->n_seq > 0 && !lens)) return "prefix_len, n_seq or seq_lens is bad";
  long n = c->prefix_len;
  for (int i = 0; i < c->n_seq; ++i) {
    if (lens[i] < 0) return "a sequence's length is negative";
    n += lens[i];
    // far more than the 32-bit offsets reach, and the sum and the bytes below stay within 64 bits
    if (n >= (1l << 32)) return "the rows of q|k|v exceed 32-bit offsets";
  }
  if (n - (c->prefix_queries ? 0 : c->prefix_len) < 1) return "no token has a query";
  if ((n + 2 * ROWS) * (c->n_head + 2 * c->n_kv_head) * c->head_dim * 2 >= (1l << 32))
    return "the rows of q|k|v exceed 32-bit offsets";
  return "";
}

size_t prefix_bytes(const qwen3_prefix_config& c, const int32_t* lens) { return places(c, lay_out(c, lens)).total; }

hipError_t prefix_make(const qwen3_prefix_config& c, const int32_t* lens, void* d_plan, size_t plan_bytes,
                       hipStream_t s, qwen3_prefix* out, bool* fits) {
  const Tables t = lay_out(c, lens);
  const Places p = places(c, t);
  *fits = plan_bytes >= p.total;
  if (!*fits) return hipErrorInvalidValue;
  // the copy and the wait below would end a capture
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipError_t e = hipStreamIsCapturing(s, &capture)) return e;
  if (capture != hipStreamCaptureStatusNone) return hipErrorStreamCaptureUnsupported;
  char* d = static_cast<char*>(d_plan);
  std::vector<char> host(p.dsum);
  auto put = [&](size_t at, const void* from, size_t bytes) {
    if (bytes) std::memcpy(host.data() + at, from, bytes);
  };
  put(p.first, t.first.data(), t.N * 4ul);
  put(p.end, t.end.data(), t.N * 4ul);
  put(p.pos, t.pos.data(), t.N * 4ul);
  put(p.items, t.items.data(), t.items.size() * sizeof(PrefixItem));
  put(p.joins, t.joins.data(), t.joins.size() * sizeof(PrefixJoin));
  put(p.kitems, t.kitems.data(), t.kitems.size() * sizeof(PrefixItem));
  put(p.kjoins, t.kjoins.data(), t.kjoins.size() * sizeof(PrefixJoin));
  hipError_t e = hipMemcpyAsync(d, host.data(), host.size(), hipMemcpyHostToDevice, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);   // the host copy goes out of scope
  if (e != hipSuccess) return e;
  PrefixArgs& a = out->args;
  a = PrefixArgs{};
  a.N = t.N; a.P = t.P; a.q0 = t.q0; a.nq = t.nq;
  a.H = c.n_head; a.Hkv = c.n_kv_head; a.hd = c.head_dim;
  auto at = [&](size_t o) { return static_cast<void*>(d + o); };
  a.first = static_cast<int32_t*>(at(p.first));
  a.end = static_cast<int32_t*>(at(p.end));
  a.items = static_cast<PrefixItem*>(at(p.items));
  a.joins = static_cast<PrefixJoin*>(at(p.joins));
  a.kitems = static_cast<PrefixItem*>(at(p.kitems));
  a.kjoins = static_cast<PrefixJoin*>(at(p.kjoins));
  a.dsum = static_cast<float*>(at(p.dsum));
  a.part = static_cast<float*>(at(p.part));
  a.nitems = (int)t.items.size();
  a.njoins = (int)t.joins.size();
  for (const PrefixJoin& j : t.joins) a.parts = std::max(a.parts, (int)j.parts);
  a.nkitems = (int)t.kitems.size();
  a.nkjoins = (int)t.kjoins.size();
  out->positions = static_cast<int32_t*>(at(p.pos));
  out->pairs = t.pairs;
  return hipSuccess;
}

extern "C" {

gpt2_status qwen3_prefix_size(const qwen3_prefix_config* cfg, const int32_t* seq_lens, size_t* bytes_out) {
  try {
    const std::string why = prefix_check(cfg, seq_lens);
    if (!why.empty()) return fail(GPT2_ERR_INVALID_ARG, why.c_str());
    if (!bytes_out) return fail(GPT2_ERR_INVALID_ARG, "bytes_out is NULL");
    *bytes_out = prefix_bytes(*cfg, seq_lens);
    return GPT2_OK;
  } catch (const std::bad_alloc&) {
    return fail(GPT2_ERR_DEVICE, "out of memory");
  }
}

gpt2_status qwen3_prefix_create(const qwen3_prefix_config* cfg, const int32_t* seq_lens, void* d_plan,
                                size_t plan_bytes, void* hip_stream, qwen3_prefix** out) {
  try {
    const std::string why = prefix_check(cfg, seq_lens);
    if (!why.empty()) return fail(GPT2_ERR_INVALID_ARG, why.c_str());
    if (!d_plan || !out || reinterpret_cast<uintptr_t>(d_plan) % 256)
      return fail(GPT2_ERR_INVALID_ARG, "d_plan is NULL or not 256-byte aligned, or out is NULL");
    std::unique_ptr<qwen3_prefix> p(new qwen3_prefix());
    bool fits = false;
    const hipError_t e = prefix_make(*cfg, seq_lens, d_plan, plan_bytes, static_cast<hipStream_t>(hip_stream), p.get(),
                                     &fits);
    if (!fits) return fail(GPT2_ERR_INVALID_ARG, "d_plan is smaller than qwen3_prefix_size says");
    if (e == hipErrorStreamCaptureUnsupported)
      return fail(GPT2_ERR_STATE, "a layout is not made while its stream is captured");
    if (e != hipSuccess) return fail(GPT2_ERR_DEVICE, hipGetErrorString(e));
    *out = p.release();
    return GPT2_OK;
  } catch (const std::bad_alloc&) {
    return fail(GPT2_ERR_DEVICE, "out of memory");
  }
}

gpt2_status qwen3_prefix_forward(const qwen3_prefix* p, const void* d_qkv, void* d_out, float* d_lse,
                                 void* hip_stream) {
  if (!p || !d_qkv || !d_out || !d_lse) return fail(GPT2_ERR_INVALID_ARG, "null argument");
  if (!aligned16(d_qkv) || !aligned16(d_out) || reinterpret_cast<uintptr_t>(d_lse) % 4)
    return fail(GPT2_ERR_INVALID_ARG, "a pointer is not aligned");
  const Bytes n(p->args);
  if (overlap(d_out, n.rows, d_qkv, n.qkv) || overlap(d_lse, n.lse, d_qkv, n.qkv) ||
      overlap(d_lse, n.lse, d_out, n.rows))
    return fail(GPT2_ERR_INVALID_ARG, "out or lse overlaps another buffer");
  PrefixArgs a = p->args;
  a.qkv = static_cast<const bf16_t*>(d_qkv);
  a.out = static_cast<bf16_t*>(d_out);
  a.lse = d_lse;
  const hipError_t e = launch_prefix_fwd(a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GPT2_OK : fail(GPT2_ERR_DEVICE, hipGetErrorString(e));
}

gpt2_status qwen3_prefix_backward(const qwen3_prefix* p, const void* d_qkv, const void* d_out, const float* d_lse,
                                  const void* d_dout, void* d_dqkv, void* hip_stream) {
  if (!p || !d_qkv || !d_out || !d_lse || !d_dout || !d_dqkv) return fail(GPT2_ERR_INVALID_ARG, "null argument");
  if (!aligned16(d_qkv) || !aligned16(d_out) || !aligned16(d_dout) || !aligned16(d_dqkv) ||
      reinterpret_cast<uintptr_t>(d_lse) % 4)
    return fail(GPT2_ERR_INVALID_ARG, "a pointer is not aligned");
  const Bytes n(p->args);
  if (overlap(d_dqkv, n.qkv, d_qkv, n.qkv) || overlap(d_dqkv, n.qkv, d_out, n.rows) ||
      overlap(d_dqkv, n.qkv, d_dout, n.rows) || overlap(d_dqkv, n.qkv, d_lse, n.lse))
    return fail(GPT2_ERR_INVALID_ARG, "dqkv overlaps another buffer");
  PrefixArgs a = p->args;
  a.qkv = static_cast<const bf16_t*>(d_qkv);
  a.out = static_cast<bf16_t*>(const_cast<void*>(d_out));
  a.lse = const_cast<float*>(d_lse);
  a.dout = static_cast<const bf16_t*>(d_dout);
  a.dqkv = static_cast<bf16_t*>(d_dqkv);
  const hipError_t e = launch_prefix_bwd(a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GPT2_OK : fail(GPT2_ERR_DEVICE, hipGetErrorString(e));
}

void qwen3_prefix_destroy(qwen3_prefix* p) { delete p; }

}  // extern "C"
