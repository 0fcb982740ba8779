// Entry points of the cache's pages, the attention over it and the adjustment
// of logits: checks of the arguments.
#include <hip/hip_runtime.h>

#include "decode.h"
#include "prefix.h"

namespace {

gpt2_status refuse(const char* why) {
  set_qwen3_error(why);
  return GPT2_ERR_INVALID_ARG;
}

gpt2_status done(hipError_t e) {
  if (e == hipSuccess) return GPT2_OK;
  set_qwen3_error(hipGetErrorString(e));
  return GPT2_ERR_DEVICE;
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

size_t pages_bytes(const qwen3_cache& c) {
  return (size_t)c.n_layer * c.n_pages * 2 * c.n_kv_head * c.page_size * c.head_dim * sizeof(bf16_t);
}

// Sizes of a cache; its buffers too unless sizes_only.
const char* cache_check(const qwen3_cache* c, bool sizes_only = false) {
  if (!c) return "null cache";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return "page_size must be 16, 32, 64, 128 or 256";
  if (c->n_layer < 1 || c->n_layer > 65535 || c->n_kv_head < 1 || c->n_kv_head > 4096)
    return "n_layer or n_kv_head out of range";
  if (c->n_pages < 1 || c->n_seq < 1 || c->n_seq > CACHE_MAX_SEQ || c->max_pages < 1 ||
      (long)c->max_pages * c->page_size >= 1l << 30 || c->n_pages >= 1 << 28)
    return "n_pages, n_seq or max_pages out of range";
  if (sizes_only) return nullptr;
  if (!c->d_pages || !c->d_table || !c->d_lens || !c->d_refs || !c->d_short || !c->d_scratch)
    return "null buffer of the cache";
  if (!aligned(c->d_pages, 16) || !aligned(c->d_scratch, 16) || !aligned(c->d_table, 4) || !aligned(c->d_lens, 4) ||
      !aligned(c->d_refs, 4) || !aligned(c->d_short, 4))
    return "a buffer of the cache is not aligned";
  return nullptr;
}

const char* heads_check(const qwen3_cache& c, int32_t n_head, int32_t n_rows) {
  if (n_head < 1 || n_head > 4096 || n_head % c.n_kv_head) return "n_head must be a multiple of n_kv_head, 4096 at most";
  if (n_rows < 0 || n_rows >= 1 << 28) return "n_rows out of range";
  return nullptr;
}

// Whether a call that changes the cache writes into a buffer: its books, and its pages if `pages`.
bool writes(const qwen3_cache& c, const void* p, size_t bytes, bool pages) {
  const size_t n = 4ul * c.n_seq;
  return overlap(p, bytes, c.d_table, n * c.max_pages) || overlap(p, bytes, c.d_lens, n) ||
         overlap(p, bytes, c.d_refs, 4ul * c.n_pages) || overlap(p, bytes, c.d_short, 4) ||
         overlap(p, bytes, c.d_scratch, sizeof(int32_t) * cache_scratch_ints(c.n_seq, c.n_pages)) ||
         (pages && overlap(p, bytes, c.d_pages, pages_bytes(c)));
}

}  // namespace

CacheArgs cache_args(const qwen3_cache& c) {
  CacheArgs a{};
  a.L = c.n_layer; a.Hkv = c.n_kv_head; a.hd = c.head_dim; a.ps = c.page_size;
  a.n_pages = c.n_pages; a.n_seq = c.n_seq; a.max_pages = c.max_pages;
  a.pages = static_cast<bf16_t*>(c.d_pages);
  a.table = c.d_table; a.lens = c.d_lens; a.refs = c.d_refs; a.missing = c.d_short;
  a.scratch = static_cast<int32_t*>(c.d_scratch);
  return a;
}

const bf16_t* cache_layer(const qwen3_cache& c, int layer) {
  return static_cast<const bf16_t*>(c.d_pages) +
         (size_t)layer * c.n_pages * 2 * c.n_kv_head * c.page_size * c.head_dim;
}

const char* tree_check(const qwen3_cache* c, const qwen3_tree* t, bool sizes_only, TreeArgs* a) {
  if (const char* why = cache_check(c, sizes_only)) return why;
  if (!t) return "null description";
  if (const char* why = heads_check(*c, t->n_head, t->n_rows)) return why;
  if ((long)t->n_rows * t->n_head >= 1l << 26) return "n_rows * n_head must stay below 2^26";   // a launch's threads
  if (t->max_new < 1 || t->max_new >= 1 << 28) return "max_new out of range";
  if (t->layer < 0 || t->layer >= c->n_layer) return "layer out of range";
  *a = TreeArgs{};
  a->H = t->n_head; a->Hkv = c->n_kv_head; a->hd = c->head_dim; a->ps = c->page_size;
  a->n_pages = c->n_pages; a->n_seq = c->n_seq; a->max_pages = c->max_pages;
  a->n_rows = t->n_rows; a->max_new = t->max_new < t->n_rows ? t->max_new : t->n_rows;
  if (a->max_new < 1) a->max_new = 1;
  a->mask_words = t->mask_words;
  if (!sizes_only) {
    a->pages = cache_layer(*c, t->layer);
    a->table = c->d_table; a->lens = c->d_lens; a->refs = c->d_refs;
  }
  return nullptr;
}

const char* append_check(const qwen3_cache* c, const AppendArgs& a) {
  if (const char* why = cache_check(c)) return why;
  if (const char* why = heads_check(*c, a.H, a.n_rows)) return why;
  // (the pages that all sequences may need stay below 2^31)
  if (a.max_new < 1 || ((a.path || a.max_new >= 1 << 22) && (long)a.max_new * c->n_seq >= 1l << 25))
    return "max_new out of range";
  if (!a.starts || (!a.qkv && a.n_rows > 0)) return "null argument";
  if (a.path && !a.counts) return "a path needs counts";
  if (!aligned(a.qkv, 16) || !aligned(a.starts, 4) || !aligned(a.counts, 4) || !aligned(a.path, 4))
    return "a pointer is not aligned";
  if (a.layer_stride % 8 || a.layer_stride > 1ul << 40) return "layer_stride must be a multiple of 8, 2^40 at most";
  const size_t row = (size_t)(a.H + 2 * c->n_kv_head) * c->head_dim;
  const size_t all = a.n_rows ? ((c->n_layer - 1) * a.layer_stride + a.n_rows * row) * sizeof(bf16_t) : 0;
  const size_t n = 4ul * c->n_seq;
  const struct { const void* p; size_t bytes; } in[] = {
      {a.qkv, all}, {a.starts, n + 4}, {a.counts, n}, {a.path, n * a.max_new}};
  for (const auto& i : in)
    if (i.p && writes(*c, i.p, i.bytes, true)) return "an input overlaps what the call writes";
  return nullptr;
}

extern "C" {

gpt2_status qwen3_cache_scratch(const qwen3_cache* c, size_t* bytes_out) {
  if (const char* why = cache_check(c, true)) return refuse(why);
  if (!bytes_out) return refuse("bytes_out is NULL");
  *bytes_out = sizeof(int32_t) * cache_scratch_ints(c->n_seq, c->n_pages);
  return GPT2_OK;
}

gpt2_status qwen3_cache_fork(const qwen3_cache* c, const int32_t* d_src, const int32_t* d_keep, void* hip_stream) {
  if (const char* why = cache_check(c)) return refuse(why);
  if (!d_src) return refuse("d_src is NULL");
  if (!aligned(d_src, 4) || !aligned(d_keep, 4)) return refuse("a pointer is not aligned");
  for (const int32_t* p : {d_src, d_keep})
    if (p && writes(*c, p, 4ul * c->n_seq, false)) return refuse("d_src or d_keep overlaps what the call writes");
  return done(launch_cache_fork(cache_args(*c), d_src, d_keep, static_cast<hipStream_t>(hip_stream)));
}

gpt2_status qwen3_cache_append(const qwen3_cache* c, const void* d_qkv, int32_t n_head, int32_t n_rows,
                               size_t layer_stride, const int32_t* d_starts, const int32_t* d_counts,
                               const int32_t* d_path, int32_t max_new, void* hip_stream) {
  const AppendArgs a{static_cast<const bf16_t*>(d_qkv), n_head, n_rows, max_new, layer_stride, d_starts, d_counts, d_path};
  if (const char* why = append_check(c, a)) return refuse(why);
  return done(launch_cache_append(cache_args(*c), a, static_cast<hipStream_t>(hip_stream)));
}

gpt2_status qwen3_cache_compact(const qwen3_cache* c, void* hip_stream) {
  if (const char* why = cache_check(c)) return refuse(why);
  return done(launch_cache_compact(cache_args(*c), static_cast<hipStream_t>(hip_stream)));
}

gpt2_status qwen3_tree_size(const qwen3_cache* c, const qwen3_tree* t, size_t* bytes_out) {
  TreeArgs a;
  if (const char* why = tree_check(c, t, true, &a)) return refuse(why);
  if (!bytes_out) return refuse("bytes_out is NULL");
  size_t at;
  const size_t bytes = tree_workspace(a, &at);
  if (!bytes) return refuse("the sequences are too many or too long");
  *bytes_out = bytes;
  return GPT2_OK;
}

gpt2_status qwen3_tree_attention(const qwen3_cache* c, const qwen3_tree* t, const void* d_qkv, const int32_t* d_starts,
                                 const int32_t* d_mask, void* d_out, float* d_lse, void* d_workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  TreeArgs a;
  if (const char* why = tree_check(c, t, false, &a)) return refuse(why);
  if (d_mask && (t->mask_words < 1 || t->mask_words > 1 << 20)) return refuse("mask_words out of range");
  size_t at;
  const size_t need = tree_workspace(a, &at);
  if (!need) return refuse("the sequences are too many or too long");
  if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < need)
    return refuse("the workspace is NULL, not 256-byte aligned, or smaller than qwen3_tree_size says");
  if (t->n_rows == 0) return GPT2_OK;
  if (!d_qkv || !d_starts || !d_out) return refuse("null argument");
  if (!aligned(d_qkv, 16) || !aligned(d_out, 16) || !aligned(d_starts, 4) || !aligned(d_mask, 4) || !aligned(d_lse, 4))
    return refuse("a pointer is not aligned");
  const size_t n = t->n_rows, row = (size_t)c->head_dim * sizeof(bf16_t);
  const size_t qkv = n * (t->n_head + 2 * c->n_kv_head) * row, out = n * t->n_head * row, lse = 4 * n * t->n_head;
  const size_t seqs = 4ul * c->n_seq;
  const struct { const void* p; size_t bytes; } in[] = {
      {d_qkv, qkv}, {d_starts, seqs + 4}, {d_mask, d_mask ? 4 * n * t->mask_words : 0}, {c->d_pages, pages_bytes(*c)},
      {c->d_table, seqs * c->max_pages}, {c->d_lens, seqs}, {c->d_refs, 4ul * c->n_pages}, {d_workspace, need}};
  for (const auto& i : in)
    if (i.p && (overlap(d_out, out, i.p, i.bytes) || (d_lse && overlap(d_lse, lse, i.p, i.bytes))))
      return refuse("out or lse overlaps another buffer");
  if (d_lse && overlap(d_out, out, d_lse, lse)) return refuse("out or lse overlaps another buffer");
  a.starts = d_starts;
  a.mask = d_mask;
  a.qkv = static_cast<const bf16_t*>(d_qkv);
  a.out = static_cast<bf16_t*>(d_out);
  a.lse = d_lse;
  a.plan = static_cast<int32_t*>(d_workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(d_workspace) + at);
  return done(launch_tree(a, static_cast<hipStream_t>(hip_stream)));
}

gpt2_status qwen3_tree_positions(const qwen3_cache* c, const qwen3_tree* t, const int32_t* d_starts,
                                 const int32_t* d_mask, int32_t* d_positions, void* hip_stream) {
  TreeArgs a;
  if (const char* why = tree_check(c, t, false, &a)) return refuse(why);
  if (d_mask && (t->mask_words < 1 || t->mask_words > 1 << 20)) return refuse("mask_words out of range");
  if (t->n_rows == 0) return GPT2_OK;
  if (!d_starts || !d_positions) return refuse("null argument");
  if (!aligned(d_starts, 4) || !aligned(d_mask, 4) || !aligned(d_positions, 4)) return refuse("a pointer is not aligned");
  const size_t out = 4ul * t->n_rows;
  if (overlap(d_positions, out, d_starts, 4ul * c->n_seq + 4) || overlap(d_positions, out, c->d_lens, 4ul * c->n_seq) ||
      (d_mask && overlap(d_positions, out, d_mask, out * t->mask_words)))
    return refuse("the positions overlap an input");
  a.starts = d_starts;
  a.mask = d_mask;
  return done(launch_tree_positions(a, d_positions, static_cast<hipStream_t>(hip_stream)));
}

gpt2_status qwen3_adjust_logits(const qwen3_logits* l, const void* d_logits, void* d_out, void* hip_stream) {
  if (!l) return refuse("null description");
  if (l->rows < 0 || l->rows > 65535 || l->vocab < 1 || l->vocab > 1 << 26) return refuse("rows or vocab out of range");
  if (l->dtype != 0 && l->dtype != 1) return refuse("dtype must be 0 (fp32) or 1 (bf16)");
  if (l->logits_stride < l->vocab || l->out_stride < l->vocab || l->logits_stride > 1l << 40 || l->out_stride > 1l << 40)
    return refuse("a stride is smaller than vocab, or larger than 2^40");
  if (l->n_bias < 0 || l->n_bias > 1024) return refuse("n_bias must be in 0..1024");
  if (l->n_masks < 0 || l->path_len < 0 || l->path_len > 1 << 20) return refuse("n_masks or path_len out of range");
  if (l->d_history && (l->n_seq < 1 || l->history_stride < 1 || l->history_stride > 1 << 28 || !l->d_lens))
    return refuse("a history needs n_seq, history_stride and d_lens");
  if (l->n_bias > 0 && (!l->d_bias_ids || !l->d_bias)) return refuse("null biases");
  if (l->n_masks > 0 && !l->d_masks) return refuse("null masks");
  if (l->path_len > 0 && !l->d_path) return refuse("null path");
  if (l->rows == 0) return GPT2_OK;
  if (!d_logits || !d_out) return refuse("null argument");
  const size_t size = l->dtype ? sizeof(bf16_t) : sizeof(float);
  if (!aligned(d_logits, size) || !aligned(d_out, size)) return refuse("a pointer is not aligned");
  const size_t rows = 4ul * l->rows, seqs = l->d_history ? 4ul * l->n_seq : 0;
  const struct { const void* p; size_t bytes; } in[] = {
      {l->d_history, seqs * l->history_stride}, {l->d_prompt_lens, seqs}, {l->d_lens, seqs}, {l->d_row_seq, rows},
      {l->d_path, rows * l->path_len}, {l->d_repetition, rows}, {l->d_frequency, rows}, {l->d_presence, rows},
      {l->d_bias_ids, rows * l->n_bias}, {l->d_bias, rows * l->n_bias},
      {l->d_masks, 4ul * l->n_masks * ((l->vocab + 31) / 32)}, {l->d_row_mask, l->n_masks ? rows : 0}};
  for (const auto& i : in)
    if (!aligned(i.p, 4)) return refuse("a pointer is not aligned");
  const bool same = d_logits == d_out;
  if (same && l->logits_stride != l->out_stride) return refuse("in place, the strides must be the same");
  const size_t in_bytes = size * ((l->rows - 1) * l->logits_stride + l->vocab);
  const size_t out_bytes = size * ((l->rows - 1) * l->out_stride + l->vocab);
  if (overlap(d_out, out_bytes, d_logits, in_bytes, true)) return refuse("out overlaps the logits without being them");
  for (const auto& i : in)
    if (i.p && overlap(d_out, out_bytes, i.p, i.bytes)) return refuse("out overlaps another input");
  qwen3_logits a = *l;
  if (!a.path_len) a.d_path = nullptr;
  return done(launch_adjust_logits(a, d_logits, d_out, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
