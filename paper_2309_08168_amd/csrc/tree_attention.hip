// Attention of a tree's nodes over a cached prefix and their own ancestors.
//
// Row r of head h: o = sum_k p_k v_k / sum_k p_k, p_k = exp(scale q.k - max),
// over every prefix key and the nodes whose bit is set in row r of the mask.
// The query heads of a kv head and the nodes share its keys: the n G rows of a kv
// head (G query heads each, row = node G + head) are one matrix of queries.
//
// Keys come in blocks of 64 (one word of the mask): first the prefix, its last
// block cut off, then the nodes in blocks of their own, so that a block's visible
// keys are one 64-bit word a row.  The blocks are split over work-groups,
// each leaving an unnormalised output with its maximum and sum, which a second
// kernel joins in order; a single share is normalised at once.
#include "tree.h"

#include <algorithm>
#include <cmath>
#include <string>

#include "host_api.h"

using namespace sdk;

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int KB = 64;  // keys of a block

struct TreeAttnArgs {
    const float *q;
    int64_t ld_q;
    const void *k, *v;
    int64_t head_stride, row_stride;
    const uint64_t *mask;  // [n][words], or null: row r sees nodes 0 .. r
    float *out;
    int64_t ld_out;
    float *part_o;    // [splits][n H][D] unnormalised outputs
    float2 *part_ml;  // [splits][n H]: (maximum, sum), in units of log2
    float scale;      // of the scores, times log2(e)
    int32_t n, words, prefix, n_heads, n_kv_heads, G, rows, q_tiles;  // rows = n G
    int32_t prefix_blocks, blocks, splits, per_split;                 // per_split: blocks of a share
};

// Block b: its first key, how many keys it has, and whether they are nodes.
struct Block {
    int first, len, node0;  // node0: the first node, or -1
};
__device__ __forceinline__ Block block_of(const TreeAttnArgs &a, int b) {
    Block k;
    if (b < a.prefix_blocks) {
        k.first = KB * b;
        k.len = min(KB, a.prefix - k.first);
        k.node0 = -1;
    } else {
        k.node0 = KB * (b - a.prefix_blocks);
        k.first = a.prefix + k.node0;
        k.len = min(KB, a.n - k.node0);
    }
    return k;
}
// The keys of a block that a node sees, as bits.
__device__ __forceinline__ uint64_t visible(const TreeAttnArgs &a, const Block &k, int node) {
    const uint64_t all = k.len >= 64 ? ~0ull : (1ull << k.len) - 1;
    if (k.node0 < 0)
        return all;
    if (a.mask)
        return a.mask[(int64_t)node * a.words + (k.node0 >> 6)] & all;
    const int last = node - k.node0;
    return last < 0 ? 0 : (last >= 63 ? ~0ull : (2ull << last) - 1) & all;
}

__device__ __forceinline__ void load4(const float *p, float (&x)[4]) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        x[j] = v[j];
}
__device__ __forceinline__ void load4(const uint16_t *p, float (&x)[4]) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    x[0] = __uint_as_float(v.x << 16);
    x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16);
    x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// ---------------------------------------------------------------------------
// In float32: a work-group of four waves takes 16 rows of a kv head, each wave
// 16 keys of every block of its share.  Scores S^T[key][row] = K q are
// 16x16x4 float32 matrix products: lane (c = lane % 16, g = lane / 16) gives
// elements 16 j + 4 g + u of key c and of row c in step (j, u), so both come by
// 16-byte loads straight from memory, and receives the keys 4 g + v, v = 0..3,
// of row c.  The value products O^T[e][row] += V^T P^T take the reduction slots
// (step v, slot g) as key 4 g + v, so weights stay in their lanes and a V operand
// is one element of row 4 g + v.  The waves keep states of their own and merge
// at the end.
constexpr int TA_WAVES = 4;

template <typename TK, int D>
__global__ __launch_bounds__(TA_WAVES * 64) void k_tree_attn_f32(TreeAttnArgs a) {
    constexpr int ES = D / 16, OP = 17;
    __shared__ float tile[TA_WAVES][D * OP];
    __shared__ float2 ml[TA_WAVES][16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g4 = lane >> 4;
    const int qt = blockIdx.x % a.q_tiles, g = blockIdx.x / a.q_tiles, split = blockIdx.y;
    const int b0 = split * a.per_split, b1 = min(a.blocks, b0 + a.per_split);
    const TK *K = static_cast<const TK *>(a.k) + (int64_t)g * a.head_stride;
    const TK *V = static_cast<const TK *>(a.v) + (int64_t)g * a.head_stride;
    const int row = min(qt * 16 + c, a.rows - 1), node = row / a.G, head = g * a.G + row - node * a.G;

    float qx[ES][4];
#pragma unroll
    for (int j = 0; j < ES; ++j) {
        load4(a.q + (int64_t)node * a.ld_q + (int64_t)head * D + 16 * j + 4 * g4, qx[j]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            qx[j][u] *= a.scale;
    }
    float m_run = -INFINITY, l_run = 0.0f;
    f32x4_t o[ES];
#pragma unroll
    for (int t = 0; t < ES; ++t)
        o[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    for (int b = b0; b < b1; ++b) {
        const Block k = block_of(a, b);
        if (16 * wave >= k.len)
            continue;  // uniform over the wave
        // keys past the block read its last one; their scores are masked
        const TK *kp = K + (int64_t)(k.first + min(16 * wave + c, k.len - 1)) * a.row_stride + 4 * g4;
        f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < ES; ++j) {
            float kx[4];
            load4(kp + 16 * j, kx);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[u], qx[j][u], s, 0, 0, 0);
        }
        const uint32_t see = (uint32_t)(visible(a, k, node) >> (16 * wave + 4 * g4)) & 15u;
        float mx = -INFINITY;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            s[v] = (see >> v) & 1 ? s[v] : -INFINITY;
            mx = fmaxf(mx, s[v]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float sc = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_use);
        float p[4];
        l_run *= sc;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            p[v] = __builtin_amdgcn_exp2f(s[v] - m_use);
        l_run += (p[0] + p[1]) + (p[2] + p[3]);
        m_run = m_new;
        const TK *vp[4];
        float vx[ES][4];
        bool odd = false;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            vp[v] = V + (int64_t)(k.first + min(16 * wave + 4 * g4 + v, k.len - 1)) * a.row_stride;
#pragma unroll
        for (int t = 0; t < ES; ++t) {
            o[t] *= sc;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                vx[t][v] = load1(vp[v] + 16 * t + c);
                odd |= !finite(vx[t][v]);
            }
        }
        if (k.node0 < 0 || !__any(odd)) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int t = 0; t < ES; ++t)
                    o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[t][v], p[v], o[t], 0, 0, 0);
        } else {
            // an infinity or NaN among the nodes' values: a row that does not
            // see it must not add 0 times it.  Lane (c, g4) holds elements
            // 16 t + 4 g4 + u of row c.
            for (int key = 0; key < 16; ++key) {
                const TK *vr = V + (int64_t)(k.first + min(16 * wave + key, k.len - 1)) * a.row_stride + 4 * g4;
                float pk = p[0];
#pragma unroll
                for (int v = 1; v < 4; ++v)
                    pk = (key & 3) == v ? p[v] : pk;
                pk = __shfl(pk, 16 * (key >> 2) + c, 64);
#pragma unroll
                for (int t = 0; t < ES; ++t) {
                    float w[4];
                    load4(vr + 16 * t, w);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        o[t][u] = pk != 0.0f ? fmaf(pk, w[u], o[t][u]) : o[t][u];
                }
            }
        }
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    // the waves' states, merged in wave order
    float *to = tile[wave];
#pragma unroll
    for (int t = 0; t < ES; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            to[(16 * t + 4 * g4 + u) * OP + c] = o[t][u];
    if (g4 == 0)
        ml[wave][c] = make_float2(m_run, l_run);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * D; i += TA_WAVES * 64) {
        const int rc = i / D, e = i - rc * D, rr = qt * 16 + rc;
        if (rr >= a.rows)
            break;  // i only grows
        float m = -INFINITY, L = 0.0f, O = 0.0f;
#pragma unroll
        for (int w = 0; w < TA_WAVES; ++w)
            m = fmaxf(m, ml[w][rc].x);
        const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < TA_WAVES; ++w) {
            // (a wave without keys has weight zero, output zero)
            const float wt = __builtin_amdgcn_exp2f(ml[w][rc].x - mu);
            L = fmaf(wt, ml[w][rc].y, L);
            O = fmaf(wt, tile[w][e * OP + rc], O);
        }
        const int nd = rr / a.G, hd = g * a.G + rr - nd * a.G;
        if (a.splits == 1) {
            a.out[(int64_t)nd * a.ld_out + (int64_t)hd * D + e] = L == 0.0f ? 0.0f : O / L;
        } else {
            const int64_t slot = ((int64_t)split * a.n + nd) * a.n_heads + hd;
            a.part_o[slot * D + e] = O;
            if (e == 0)
                a.part_ml[slot] = make_float2(m, L);
        }
    }
}

// The shares of a (node, head) joined in order: D / 4 lanes, four elements each.
__global__ __launch_bounds__(256) void k_tree_join(TreeAttnArgs a, int D, int lanes) {
    const int64_t slots = (int64_t)a.n * a.n_heads;
    const int64_t slot = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes;
    if (slot >= slots)
        return;
    const int e = 4 * (threadIdx.x % lanes);
    float m = -INFINITY;
    for (int s = 0; s < a.splits; ++s)
        m = fmaxf(m, a.part_ml[s * slots + slot].x);
    const float mu = m == -INFINITY ? 0.0f : m;
    float L = 0.0f;
    f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < a.splits; ++s) {
        const float2 v = a.part_ml[s * slots + slot];
        const float w = __builtin_amdgcn_exp2f(v.x - mu);
        L = fmaf(w, v.y, L);
        O += w * *reinterpret_cast<const f32x4_t *>(a.part_o + (s * slots + slot) * D + e);
    }
    const int nd = (int)(slot / a.n_heads), hd = (int)(slot - (int64_t)nd * a.n_heads);
    *reinterpret_cast<f32x4_t *>(a.out + (int64_t)nd * a.ld_out + (int64_t)hd * D + e) =
        L == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / L;
}

// Shares of the keys: about four work-groups per CU, at least two blocks each.
constexpr int TA_GROUPS = 1024;

void plan(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t prefix, TreeAttnArgs *a) {
    a->n = n;
    a->words = (n + 63) / 64;
    a->prefix = prefix;
    a->n_heads = n_heads;
    a->n_kv_heads = kv->n_kv_heads;
    a->G = n_heads / kv->n_kv_heads;
    a->rows = n * a->G;
    a->q_tiles = (a->rows + 15) / 16;
    a->prefix_blocks = (prefix + KB - 1) / KB;
    a->blocks = a->prefix_blocks + a->words;
    const int units = a->q_tiles * a->n_kv_heads;
    const int want = std::max(1, std::min((a->blocks + 1) / 2, (TA_GROUPS + units - 1) / units));
    a->per_split = (a->blocks + want - 1) / want;
    a->splits = (a->blocks + a->per_split - 1) / a->per_split;
}

size_t o_bytes(const TreeAttnArgs &a, int D) { return sizeof(float) * (size_t)a.splits * a.n * a.n_heads * D; }
size_t workspace_of(const TreeAttnArgs &a, int D) {
    return a.splits == 1 ? 0 : o_bytes(a, D) + sizeof(float2) * (size_t)a.splits * a.n * a.n_heads;
}

sd_status check_sizes(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t prefix) {
    const sd_status st = check_layer(kv);
    if (st != SD_OK)
        return st;
    if (n < 1 || n > SD_TREE_MAX || n_heads < 1 || n_heads > 4096 || n_heads % kv->n_kv_heads)
        return report(SD_ERR_INVALID_ARG, "a tree has 1 to " + std::to_string(SD_TREE_MAX) +
                                              " nodes; n_heads is a multiple of n_kv_heads, at most 4096");
    if (prefix < 0 || (int64_t)prefix + n > kv->capacity)
        return report(SD_ERR_CAPACITY, "a layer of capacity " + std::to_string(kv->capacity) + " does not hold " +
                                           std::to_string(n) + " nodes after " + std::to_string(prefix) +
                                           " positions");
    return SD_OK;
}

template <typename TK>
void launch_f32(const TreeAttnArgs &a, int D, hipStream_t s) {
    const dim3 grid((unsigned)(a.q_tiles * a.n_kv_heads), (unsigned)a.splits), block(TA_WAVES * 64);
    if (D == 16)
        hipLaunchKernelGGL((k_tree_attn_f32<TK, 16>), grid, block, 0, s, a);
    else if (D == 32)
        hipLaunchKernelGGL((k_tree_attn_f32<TK, 32>), grid, block, 0, s, a);
    else if (D == 64)
        hipLaunchKernelGGL((k_tree_attn_f32<TK, 64>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_tree_attn_f32<TK, 128>), grid, block, 0, s, a);
}

sd_status tree_attention(const sd_kv_layer *kv, const float *q, int64_t ld_q, int32_t n_heads, int32_t n,
                         int32_t prefix, const uint64_t *mask, float scale, float *out, int64_t ld_out,
                         void *workspace, size_t workspace_bytes, hipStream_t s) {
    const sd_status st = check_sizes(kv, n_heads, n, prefix);
    if (st != SD_OK)
        return st;
    const int D = kv->head_dim;
    auto aligned = [](const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; };
    if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(mask, 8))
        return report(SD_ERR_INVALID_ARG, "q and out must be set and 16-byte aligned, mask 8-byte aligned");
    if (ld_q % 4 || ld_out % 4 || ld_q < (int64_t)n_heads * D || ld_out < (int64_t)n_heads * D)
        return report(SD_ERR_INVALID_ARG, "ld_q and ld_out must hold a row and be multiples of 4");
    if (!std::isfinite(scale))
        return report(SD_ERR_INVALID_ARG, "scale must be finite");
    TreeAttnArgs a{};
    plan(kv, n_heads, n, prefix, &a);
    const size_t need = workspace_of(a, D);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
        return report(SD_ERR_INVALID_ARG, "these sizes need " + std::to_string(need) +
                                              " bytes of 16-byte aligned workspace");
    a.q = q;
    a.ld_q = ld_q;
    a.k = kv->k;
    a.v = kv->v;
    a.head_stride = kv->head_stride;
    a.row_stride = kv->row_stride;
    a.mask = mask;
    a.out = out;
    a.ld_out = ld_out;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + o_bytes(a, D));
    a.scale = (scale == 0.0f ? 1.0f / std::sqrt((float)D) : scale) * 1.4426950408889634f;
    if (kv->dtype == SD_BF16)
        launch_f32<uint16_t>(a, D, s);
    else
        launch_f32<float>(a, D, s);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        const int lanes = D / 4, per = 256 / lanes;
        hipLaunchKernelGGL(k_tree_join, dim3((unsigned)((n * n_heads + per - 1) / per)), dim3(256), 0, s, a, D, lanes);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SD_OK : report(SD_ERR_DEVICE, std::string("tree attention: ") + hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t sd_tree_attention_workspace(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t prefix) {
    if (check_sizes(kv, n_heads, n, prefix) != SD_OK)
        return 0;
    TreeAttnArgs a{};
    plan(kv, n_heads, n, prefix, &a);
    return workspace_of(a, kv->head_dim);
}

sd_status sd_tree_attention(const sd_kv_layer *kv, const float *q, int64_t ld_q, int32_t n_heads, int32_t n,
                            int32_t prefix, const uint64_t *mask, float scale, float *out, int64_t ld_out,
                            void *workspace, size_t workspace_bytes, void *hip_stream) {
    SD_GUARD(return tree_attention(kv, q, ld_q, n_heads, n, prefix, mask, scale, out, ld_out, workspace,
                                   workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));)
}

}  // extern "C"
