/*
 * qwen3_prompt.h - further entry points of the Qwen3-shaped adapter step
 * (qwen3.h, whose conventions hold here): the orthogonalised optimizer step.
 */
#ifndef QWEN3_PROMPT_MI355X_H
#define QWEN3_PROMPT_MI355X_H

#include "qwen3.h"

#ifdef __cplusplus
extern "C" {
#endif

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
