/*
 * qwen3_prompt.h - further entry points of the Qwen3-shaped adapter step
 * (qwen3.h, whose conventions hold here): rotary positions with several axes,
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

/* d_qkv, d_out: bf16 rows of n_tokens tokens, q [n_head * head_dim] | k
 * [n_kv_head * head_dim] | v likewise, 16-byte aligned. d_positions: int32
 * [n_axes, n_tokens], any values. d_q_norm, d_k_norm: bf16 [head_dim] gains of
 * the RMSNorm of every query and key head before the turn, 16-byte aligned, or
 * both NULL for none. Values pass through; d_out may be d_qkv. Angles are in
 * fp64, all else in fp32, the result rounded once.
 * qwen3_rotary_backward: from d_dout (the gradient of d_out) and the same
 * d_qkv, positions and gains, the gradient of d_qkv to d_dqkv, which may be
 * d_dout. The gains are frozen; without them d_qkv is not read and may be
 * NULL. INVALID_ARG for what is not as said here; nothing is launched then,
 * nor for n_tokens 0. */
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
