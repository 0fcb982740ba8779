/*
 * qwen3_prompt.h - further entry points of the Qwen3-shaped adapter step
 * (qwen3.h, whose conventions hold here): rotary positions with several axes,
 * attention over sequences that share a prefix (answers to one prompt), both
 * alone and in the step, and the orthogonalised optimizer step. Calls without
 * a model take the stream to enqueue on; it belongs to the current device, and
 * so do the pointers. qwen3_last_error(NULL) says why such a call failed.
 */
#ifndef QWEN3_PROMPT_MI355X_H
#define QWEN3_PROMPT_MI355X_H

#include "qwen3.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Head norm and rotary embedding at positions with several axes (time,
 * height and width of images and video; one axis is the ordinary embedding).
 * Pair i of a head is elements i and i + head_dim/2, turned by the angle
 * position[axis(i)] * theta^(-2i/head_dim). sections[a] pairs take axis a:
 *   interleaved 0: the first sections[0] pairs axis 0, the next sections[1]
 *     axis 1, and so on;
 *   interleaved 1: pair i takes axis i mod n_axes while i / n_axes is below
 *     that axis' section, and axis 0 otherwise; every section but the first
 *     must end within the head (a + n_axes (sections[a] - 1) < head_dim / 2).
 * Sections sum to head_dim / 2. */
typedef struct qwen3_rotary {
  int32_t n_tokens, n_head, n_kv_head, head_dim;   /* head_dim 32, 64, 128 or 256 */
  int32_t n_axes, sections[4];                     /* 1..4 axes */
  int32_t interleaved;
  float theta, rms_eps;
} qwen3_rotary;

/* d_qkv, d_out: bf16 rows of n_tokens tokens (2^25 at most), q [n_head * head_dim] | k
 * [n_kv_head * head_dim] | v likewise, 16-byte aligned. d_positions: int32
 * [n_axes, n_tokens], any values. d_q_norm, d_k_norm: bf16 [head_dim] gains of
 * the RMSNorm of every query and key head before the turn, 16-byte aligned, or
 * both NULL for none. Values pass through; d_out may be d_qkv, and overlaps it
 * in no other way. Angles are in fp64, all else in fp32, the result rounded once.
 * qwen3_rotary_backward: from d_dout (the gradient of d_out) and the same
 * d_qkv, positions and gains, the gradient of d_qkv to d_dqkv, which may be
 * d_dout or d_qkv and overlaps them in no other way. The gains are frozen;
 * without them d_qkv is not read and may be NULL. INVALID_ARG for what is not as
 * said here; nothing is launched then, nor for n_tokens 0. */
gpt2_status qwen3_rotary_forward(const qwen3_rotary* r, const void* d_qkv,
                                 const int32_t* d_positions,
                                 const void* d_q_norm, const void* d_k_norm,
                                 void* d_out, void* hip_stream);
gpt2_status qwen3_rotary_backward(const qwen3_rotary* r, const void* d_dout,
                                  const void* d_qkv, const int32_t* d_positions,
                                  const void* d_q_norm, const void* d_k_norm,
                                  void* d_dqkv, void* hip_stream);

/* Positions of the tokens of the step, from the next qwen3_forward on:
 * d_positions int32 [n_axes, B*T], read by every forward and by the backward
 * that follows it, the caller's to keep; sections and interleaved as above
 * (head_dim 128, theta from the config). NULL goes back to the default, each
 * token's place in its sequence on one axis (n_axes, sections and interleaved
 * are not looked at then). A backward takes the positions of its forward. */
gpt2_status qwen3_set_positions(qwen3_model* m, const int32_t* d_positions,
                                int32_t n_axes, const int32_t* sections,
                                int32_t interleaved);

/* Attention over packed sequences that share one prefix, such as answers to
 * one prompt, whose keys and values are then there, and read, once. The rows
 * are tokens: prefix_len of the prefix, then n_seq sequences one after another
 * of seq_lens[i] >= 0 tokens. A token sees itself, what precedes it in its own
 * sequence, and the whole prefix (a token of the prefix: what precedes it
 * there). Query head h reads key/value head h / (n_head / n_kv_head); scores
 * are scaled by 1/sqrt(head_dim). prefix_len 0 is packed causal attention,
 * n_seq 0 one causal sequence.
 * prefix_queries 1: every token has a query. 0: only the sequences' tokens have
 * (the prefix was processed before); out, lse and dout then hold their rows
 * only, and the prefix' queries are not read. */
typedef struct qwen3_prefix_config {
  int32_t n_head, n_kv_head, head_dim;   /* head_dim 64 or 128 */
  int32_t prefix_len, n_seq;
  int32_t prefix_queries;
} qwen3_prefix_config;

typedef struct qwen3_prefix qwen3_prefix;   /* opaque host-side handle */

/* A layout and its device buffer, d_plan: qwen3_prefix_size bytes, 256-byte
 * aligned, the caller's, holding the layout's tables and the calls' scratch.
 * Laid out once per set of lengths and used by any number of calls, one at a
 * time: calls (or captured graphs) that may run at the same time take a layout
 * each. create writes the tables through hip_stream and synchronises it;
 * ERR_STATE, and the capture goes on, while that stream is captured.
 * INVALID_ARG for lengths or sizes out of range (no query at all; rows beyond
 * 4 GiB), a NULL or unaligned buffer. */
gpt2_status qwen3_prefix_size(const qwen3_prefix_config* cfg,
                              const int32_t* seq_lens, size_t* bytes_out);
gpt2_status qwen3_prefix_create(const qwen3_prefix_config* cfg,
                                const int32_t* seq_lens, void* d_plan,
                                size_t plan_bytes, void* hip_stream,
                                qwen3_prefix** out);
/* d_qkv bf16 [tokens, (n_head + 2 n_kv_head) * head_dim]; d_out bf16 [rows,
 * n_head * head_dim], rows the tokens with queries; d_lse fp32 [n_head, rows],
 * the log-sum-exp of the scaled scores; d_qkv, d_out 16-byte aligned. The three
 * do not overlap. */
gpt2_status qwen3_prefix_forward(const qwen3_prefix* p, const void* d_qkv,
                                 void* d_out, float* d_lse, void* hip_stream);
/* The gradient of d_qkv to d_dqkv (written whole, over none of the inputs; zero
 * where a prefix has no queries) from d_dout, that of d_out, and the forward's
 * d_qkv, d_out and d_lse. A key's gradient sums over its group's query heads and, in
 * the prefix, over all sequences, in fp32 and in a fixed order.
 * Both: what a token does not see must be finite all the same; infinite or NaN
 * rows of one sequence can reach its neighbours' (0 times NaN in a product). */
gpt2_status qwen3_prefix_backward(const qwen3_prefix* p, const void* d_qkv,
                                  const void* d_out, const float* d_lse,
                                  const void* d_dout, void* d_dqkv,
                                  void* hip_stream);
void qwen3_prefix_destroy(qwen3_prefix* p);

/* The step's tokens as one prefix and sequences over it, from the next
 * qwen3_forward on: the model's B must be 1 and prefix_len plus the sequences'
 * lengths its T. Attention is as above, and unless qwen3_set_positions gives
 * others, a sequence's positions go on from the prefix' end. The prefix' last
 * token has one target only: let every sequence begin with the prompt's last
 * token and loss_from begin behind the prefix, and each answer's first token
 * is predicted within its own sequence. d_plan: qwen3_layout_size bytes,
 * 256-byte aligned, the caller's to keep while the layout is in use (by the
 * next forwards, a backward that follows one, and graphs that either is captured
 * into). Synchronises the stream, and is refused in a capture, as above.
 * d_plan NULL goes back to B sequences of T tokens. */
gpt2_status qwen3_layout_size(const qwen3_model* m, int32_t prefix_len,
                              int32_t n_seq, const int32_t* seq_lens,
                              size_t* bytes_out);
gpt2_status qwen3_set_layout(qwen3_model* m, int32_t prefix_len, int32_t n_seq,
                             const int32_t* seq_lens, void* d_plan,
                             size_t plan_bytes);

/* Optimizer step with an orthogonalised update (gpt2.h, gpt2_muon) in place
 * of AdamW: clip as qwen3_adamw_step does, then for every projection's A
 * [r, in] and B [out, r], with momentum M in adam_m (adam_v is unused),
 *   M = momentum M + g,  U = g + momentum M (nesterov) or M,
 *   W -= lr (weight_decay W + scale sqrt(max(rows, cols)) orthogonalised(U));
 * lora_bf16 is rewritten. d_workspace: qwen3_muon_size bytes, 256-byte
 * aligned, scratch until the call's kernels have run. Errors as
 * qwen3_adamw_step's and gpt2_muon_step's. */
gpt2_status qwen3_muon_size(const qwen3_config* cfg, size_t* bytes_out);
gpt2_status qwen3_muon_step(qwen3_model* m, const gpt2_muon* how,
                            void* d_workspace, size_t workspace_bytes,
                            float* d_grad_norm_out);

#ifdef __cplusplus
}
#endif

#endif
