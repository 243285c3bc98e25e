// The operators of token trees (tree_ops.hip, tree_attention.hip): arguments
// and launchers.
#pragma once

#include "sd.h"
#include "sd_internal.h"

namespace sdk {

// Refuses a layer that breaks the rules of sd_kv_layer.
sd_status check_layer(const sd_kv_layer *kv);

struct RopeArgs {
    // frequency of pair i: f = exp2(i * step); YARN then weighs f and f / factor
    double step, inv_factor, turns, beta_slow, inv_beta;
    float gain;
    int32_t half, interleaved, yarn;  // half: pairs of a head
    const float *qkv;
    int64_t ld_qkv;
    const int32_t *positions;
    int32_t pos0, n, n_heads, n_kv_heads, head_dim;
    float *q;
    int64_t ld_q;
    void *k, *v;
    int64_t head_stride, row_stride;
    int32_t slot;
};
// Checks a rotary form for a head_dim and fills its part of RopeArgs.
sd_status rope_form(const sd_rope *rope, int32_t head_dim, RopeArgs *out);

}  // namespace sdk
