// The layout of packed sequences that share a prefix, as the host keeps it.
#pragma once

#include <memory>
#include <string>

#include "../../include/qwen3_prompt.h"
#include "kernels.h"

struct qwen3_prefix {
  PrefixArgs args;            // device addresses of the tables and the scratch filled in
  const int32_t* positions;   // device [N]: places 0..P-1 in the prefix, then P, P+1, ... in each sequence
  double pairs;               // (query, key) pairs of one query head
};

// Why the layout is refused, or empty.
std::string prefix_check(const qwen3_prefix_config* c, const int32_t* seq_lens);
// Bytes of the device buffer of a layout that prefix_check accepts. Throws std::bad_alloc.
size_t prefix_bytes(const qwen3_prefix_config& c, const int32_t* seq_lens);
// Its tables written to d_plan (synchronises the stream), unless plan_bytes is
// too few for it; hipErrorStreamCaptureUnsupported, with nothing enqueued, in a
// capture. Throws std::bad_alloc.
hipError_t prefix_make(const qwen3_prefix_config& c, const int32_t* seq_lens, void* d_plan, size_t plan_bytes,
                       hipStream_t s, qwen3_prefix* out, bool* fits);

// the reason of the last failure of a call without a model, for qwen3_last_error
void set_qwen3_error(const char* why);
