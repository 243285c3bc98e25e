// What the operators of token trees (tree_ops.hip, tree_attention.hip) share
// with each other and with the model's forwards.
#pragma once

#include "sd.h"
#include "sd_internal.h"

namespace sdk {

// Refuses a layer that breaks the rules of sd_kv_layer.
sd_status check_layer(const sd_kv_layer *kv);

// Refuses a rotary form for a head_dim.
sd_status check_rope(const sd_rope *rope, int32_t head_dim);
// Angle per position of pair i, and the factor on cosines and sines, of a
// checked form (float64, on the host).
double rope_frequency(const sd_rope &rope, int32_t i);
double rope_gain(const sd_rope &rope);

// sd_tree_attention for the last n rows of a tree of `nodes` (mask: the words
// of those rows); sd_tree_attention itself has n = nodes.
sd_status tree_attention(const sd_kv_layer *kv, const float *q, int64_t ld_q, int32_t n_heads, int32_t n, int32_t nodes,
                         int32_t prefix, const uint64_t *mask, float scale, float *out, int64_t ld_out, void *workspace,
                         size_t workspace_bytes, hipStream_t s);
size_t tree_attention_bytes(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t nodes, int32_t prefix);

}  // namespace sdk
