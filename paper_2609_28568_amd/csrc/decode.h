// The paged cache and attention over it, as the model's forward uses them.
#pragma once

#include "../../include/qwen3_decode.h"
#include "kernels.h"

// Why a description is refused, or null; *a gets its sizes and, unless
// sizes_only, the cache's addresses (of the layer's pages).
const char* tree_check(const qwen3_cache* c, const qwen3_tree* t, bool sizes_only, TreeArgs* a);
// the layer's pages
const bf16_t* cache_layer(const qwen3_cache& c, int layer);
// Why an append is refused, or null.
const char* append_check(const qwen3_cache* c, const AppendArgs& a);
CacheArgs cache_args(const qwen3_cache& c);
