// Attention of a batch's rows: over the pages of a cache (sd_paged_attention) and
// over packed keys and values (sd_prompt_attention).
//
// Row i of a sequence, head h: o = sum_k p_k v_k / sum_k p_k, p_k = exp(scale q.k -
// max), over the keys 0 .. past + i.  The m rows of a sequence and the G query heads
// of a kv head share its keys: its m G rows (row = i G + head) are cut into tiles,
// and the keys of a tile into shares, each leaving an unnormalised output with its
// maximum and sum, which a second kernel joins in order; a single share is
// normalised at once.
#include "paged.h"

#include <algorithm>
#include <cmath>
#include <string>

#include "host_api.h"
#include "rope.h"
#include "sd_internal.h"

using namespace sdk;

namespace {

struct BatchAttnArgs {
    const void *q;
    int64_t ld_q;
    void *out;
    int64_t ld_out;
    const void *k, *v;
    int64_t page_stride, head_stride, row_stride;
    const int32_t *table;    // null: packed, key j of a sequence in row first + j
    const int32_t *lengths;  // null: a sequence is its rows
    const int32_t *starts;   // null: max_rows a sequence
    int64_t ld_table;
    float *part_o;    // [splits][n H][D] unnormalised outputs
    float2 *part_ml;  // [splits][n H]: (maximum, sum), in units of log2
    float scale;      // of the scores, times log2(e)
    int32_t n, n_seqs, max_rows, max_length, n_pages, page_shift;
    int32_t n_heads, n_kv_heads, G;
    int32_t tile, slots, one_tile;     // rows of a tile; tiles at most; whether a sequence has at most one
    int32_t splits, per_split, block;  // shares of the keys; blocks of a share; keys of a block
};

__device__ __forceinline__ int32_t start_of(const BatchAttnArgs &a, int32_t s) {
    return a.starts ? a.starts[s] : s * a.max_rows;
}
__device__ __forceinline__ SeqRows rows_of(const BatchAttnArgs &a, int32_t s) {
    SeqRows r = seq_rows(start_of(a, s), start_of(a, s + 1), a.lengths ? a.lengths[s] : 0, a.n, a.max_rows);
    if (!a.lengths)
        r.past = 0;
    return r;
}

// Tile `t` of the call: its sequence, the rows of it, and the first row of the tile
// among the m G of a kv head (m G or more: there is no such tile).  The tiles of
// sequence s start at slot floor(starts[s] G / tile) + s, which leaves each at
// least as many as it has, and needs no sum over the sequences before.
struct Tile {
    int32_t seq, row0;
    SeqRows rows;
};
__device__ __forceinline__ Tile tile_of(const BatchAttnArgs &a, int32_t t) {
    Tile w;
    if (a.one_tile) {
        w.seq = t;
        w.rows = rows_of(a, t);
        w.row0 = 0;
        return w;
    }
    const auto slot = [&](int32_t j) { return (int64_t)start_of(a, j) * a.G / a.tile + j; };
    w.seq = min(wave_count(a.n_seqs, t, slot), a.n_seqs - 1);
    w.rows = rows_of(a, w.seq);
    const int64_t row0 = ((int64_t)t - slot(w.seq)) * a.tile, most = (int64_t)w.rows.m * a.G;
    w.row0 = (int32_t)(row0 < 0 || row0 > most ? most : row0);
    return w;
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// The NW waves' states of ROWS rows from row0 on (o [wave][row][D + 4], waves
// `pitch` floats apart; (maximum, sum) [wave][row]) merged in wave order: the
// result of a single share, or its part of several.
template <typename TX, int D, int NW, int ROWS>
__device__ __forceinline__ void merge_waves(const BatchAttnArgs &a, const Tile &w, const float *o, int pitch,
                                            const float2 *ml, int g, int split) {
#pragma unroll
    for (int i = threadIdx.x; i < ROWS * D / 4; i += NW * 64) {
        const int rc = i / (D / 4), e = 4 * (i % (D / 4)), rr = w.row0 + rc;
        if (rr >= w.rows.m * a.G)
            break;  // i only grows
        float m = -INFINITY, L = 0.0f;
        f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NW; ++v)
            m = fmaxf(m, ml[v * ROWS + rc].x);
        const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            // (a wave without keys has weight zero, output zero)
            const float wt = __builtin_amdgcn_exp2f(ml[v * ROWS + rc].x - mu);
            L = fmaf(wt, ml[v * ROWS + rc].y, L);
            O += wt * load4(o + v * pitch + rc * (D + 4) + e);
        }
        const int node = rr / a.G, head = g * a.G + rr - node * a.G;
        const int64_t row = w.rows.first + node;
        if (a.splits == 1) {
            store4(static_cast<TX *>(a.out) + row * a.ld_out + (int64_t)head * D + e,
                   L == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / L);
        } else {
            const int64_t slot = ((int64_t)split * a.n + row) * a.n_heads + head;
            store4(a.part_o + slot * D + e, O);
            if (e == 0)
                a.part_ml[slot] = make_float2(m, L);
        }
    }
}

// ---------------------------------------------------------------------------
// In float32: a work-group of four waves takes 16 rows of a kv head, each wave
// 16 keys of every block of its share.  Scores S^T[key][row] = K q are
// 16x16x4 float32 matrix products: lane (c = lane % 16, g = lane / 16) gives
// elements 16 j + 4 g + u of key c and of row c in step (j, u), and receives the
// keys 4 g + v, v = 0..3, of row c.  The value products O^T[e][row] += V^T P^T
// take the reduction slots (step v, slot g) as key 4 g + v, so weights stay in
// their lanes; tile t's row i is element 64 (t / 4) + 4 i + t % 4, so adjacent
// elements of row 4 g + v are a lane's operands of four tiles.  V is asked for before
// the scores and the next block's K after them.  The waves keep states of their
// own and merge at the end.  A wave's 16 keys lie in one page.
constexpr int KB = 64, NW = 4;

template <int W, typename T>
__device__ __forceinline__ void load_some(const T *p, float (&x)[W]) {
    if constexpr (W == 4) {
        const f32x4_t y = load4(p);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            x[u] = y[u];
    } else {
#pragma unroll
        for (int u = 0; u < W; ++u)
            x[u] = load1(p + u);
    }
}

template <typename TX, typename TK, int D>
__global__ __launch_bounds__(NW * 64, 2) void k_batch_attn_f32(BatchAttnArgs a) {
    constexpr int ES = D / 16, OP = D + 4, W = ES < 4 ? ES : 4;  // W: adjacent elements of V
    __shared__ __attribute__((aligned(16))) float tile[NW][16 * OP];
    __shared__ float2 ml[NW][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15,
              g4 = lane >> 4;
    const int g = blockIdx.x % a.n_kv_heads, split = blockIdx.y;
    const Tile w = tile_of(a, blockIdx.x / a.n_kv_heads);
    const int rows = w.rows.m * a.G;
    if (w.row0 >= rows)
        return;  // uniform
    auto sees = [&](int rr) { return seen_from(w.rows.past + rr / a.G, a.max_length); };
    const int klen = sees(min(w.row0 + 15, rows - 1)), kall = sees(w.row0);
    const int b0 = split * a.per_split, b1 = min(b0 + a.per_split, (klen + KB - 1) / KB);
    if (a.splits > 1 && b0 >= b1)
        return;
    const TK *K = static_cast<const TK *>(a.k) + (int64_t)g * a.head_stride;
    const TK *V = static_cast<const TK *>(a.v) + (int64_t)g * a.head_stride;
    const int rr = min(w.row0 + c, rows - 1), node = rr / a.G, head = g * a.G + rr - node * a.G;
    const int see = seen_from(w.rows.past + node, a.max_length);

    f32x4_t qx[ES];
#pragma unroll
    for (int j = 0; j < ES; ++j)
        qx[j] = load4(static_cast<const TX *>(a.q) + (int64_t)(w.rows.first + node) * a.ld_q + (int64_t)head * D + 16 * j +
                      4 * g4) *
                a.scale;
    // o[t][u]: this element of row c
    auto element = [&](int t, int u) { return 16 * W * (t / W) + W * (4 * g4 + u) + t % W; };
    float m_run = -INFINITY, l_run = 0.0f;
    f32x4_t o[ES];
#pragma unroll
    for (int t = 0; t < ES; ++t)
        o[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    // the page of this wave's keys of block b, -1 where there are none
    auto page_of = [&](int b) {
        const int first = KB * b + 16 * wave;
        if (first >= klen)
            return -1;
        if (!a.table)
            return 0;
        const int page = a.table[(int64_t)w.seq * a.ld_table + (first >> a.page_shift)];
        return (uint32_t)page < (uint32_t)a.n_pages ? page : -1;
    };
    auto place = [&](int b, int page) -> int64_t {
        const int first = KB * b + 16 * wave;
        return a.table ? page * a.page_stride + (int64_t)(first & ((1 << a.page_shift) - 1)) * a.row_stride
                       : (int64_t)(w.rows.first + first) * a.row_stride;
    };
    // keys past the last read that one; their scores are masked
    f32x4_t kx[ES];
    auto load_k = [&](int b, int page) {
        const TK *kp = K + place(b, page) + min(c, klen - 1 - KB * b - 16 * wave) * a.row_stride + 4 * g4;
#pragma unroll
        for (int j = 0; j < ES; ++j)
            kx[j] = load4(kp + 16 * j);
    };
    int page = page_of(b0), next = page_of(b0 + 1);
    if (b0 < b1 && page >= 0)
        load_k(b0, page);
    for (int b = b0; b < b1; ++b) {
        const int after = page_of(b + 2);
        const int first = KB * b + 16 * wave;
        const bool some = page >= 0;  // uniform over the wave
        f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
        float vx[4][ES / W][W];
        const TK *vb = V + place(b, page);
        if (some) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const TK *vp = vb + min(4 * g4 + v, klen - 1 - first) * a.row_stride + W * c;
#pragma unroll
                for (int t = 0; t < ES / W; ++t)
                    load_some<W>(vp + 16 * W * t, vx[v][t]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < ES; ++j)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[j][u], qx[j][u], s, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (b + 1 < b1 && next >= 0)
            load_k(b + 1, next);
        page = next;
        next = after;
        if (!some)
            continue;
        const bool part = first + 16 > kall;  // uniform: some row does not see every key
        float mx = -INFINITY;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (part)
                s[v] = first + 4 * g4 + v < see ? s[v] : -INFINITY;
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
#pragma unroll
        for (int t = 0; t < ES; ++t)
            o[t] *= sc;
        bool odd = false;
        if (part) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int t = 0; t < ES; ++t)
                    odd |= !finite(vx[v][t / W][t % W]);
        }
        if (__any(odd)) {
            // An infinity or NaN among values that some row does not see: it must
            // not add 0 times it.  They are taken out of the operands, and
            // added here, from memory, where they belong.
            for (int key = 0; key < 16; ++key) {
                const TK *vr = vb + min(key, klen - 1 - first) * a.row_stride;
                float pk = p[0];
#pragma unroll
                for (int v = 1; v < 4; ++v)
                    pk = (key & 3) == v ? p[v] : pk;
                pk = __shfl(pk, 16 * (key >> 2) + c, 64);
#pragma unroll
                for (int t = 0; t < ES; ++t)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float x = load1(vr + element(t, u));
                        if (pk != 0.0f && !finite(x))
                            o[t][u] = fmaf(pk, x, o[t][u]);
                    }
            }
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int t = 0; t < ES; ++t)
                    vx[v][t / W][t % W] = finite(vx[v][t / W][t % W]) ? vx[v][t / W][t % W] : 0.0f;
        }
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int t = 0; t < ES; ++t)
                o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[v][t / W][t % W], p[v], o[t], 0, 0, 0);
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    // the waves' states, merged in wave order
    float *to = tile[wave];
#pragma unroll
    for (int t = 0; t < ES; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            to[c * OP + element(t, u)] = o[t][u];
    if (g4 == 0)
        ml[wave][c] = make_float2(m_run, l_run);
    __syncthreads();
    merge_waves<TX, D, NW, 16>(a, w, &tile[0][0], 16 * OP, &ml[0][0], g, split);
}

// The shares of a (row, head) joined: a work-group each.  D / 4 lanes hold a row, the
// groups of lanes take the shares in turn and add up in order.
constexpr int JOIN_THREADS = 256;
template <typename TX, int D>
__global__ __launch_bounds__(JOIN_THREADS) void k_batch_join(BatchAttnArgs a) {
    constexpr int LANES = D / 4, NG = JOIN_THREADS / LANES;
    __shared__ f32x4_t red[NG][LANES];
    const int64_t slots = (int64_t)a.n * a.n_heads, slot = blockIdx.x;
    const int lane = threadIdx.x & 63, e = threadIdx.x % LANES, gi = threadIdx.x / LANES;
    const int row = (int)(slot / a.n_heads), head = (int)(slot - (int64_t)row * a.n_heads);
    // the shares that hold keys of the row
    int s;
    if (a.starts) {
        s = wave_count(a.n_seqs, row, [&](int j) { return (int64_t)a.starts[j]; });
        if (s >= a.n_seqs)
            return;  // uniform
    } else {
        s = row / a.max_rows;
    }
    const SeqRows rows = rows_of(a, s);
    const int i = row - rows.first;
    if (i < 0 || i >= rows.m)
        return;
    const int keys = a.per_split * a.block;
    const int shares = min(a.splits, (seen_from(rows.past + i, a.max_length) + keys - 1) / keys);
    const float *po = a.part_o + slot * D + 4 * e;
    const float2 *pm = a.part_ml + slot;
    float m = -INFINITY;
    for (int j = lane; j < shares; j += 64)
        m = fmaxf(m, pm[j * slots].x);
    m = wave_max_all(m);
    const float mu = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f;
    for (int j = lane; j < shares; j += 64) {
        const float2 v = pm[j * slots];
        sum = fmaf(__builtin_amdgcn_exp2f(v.x - mu), v.y, sum);
    }
    const float total = wave_sum_all(sum);
    f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int j = gi; j < shares; j += NG)
        O += __builtin_amdgcn_exp2f(pm[j * slots].x - mu) * load4(po + j * slots * D);
    red[gi][e] = O;
    __syncthreads();
    if (gi > 0)
        return;
#pragma unroll
    for (int j = 1; j < NG; ++j)
        O += red[j][e];
    store4(static_cast<TX *>(a.out) + (int64_t)row * a.ld_out + (int64_t)head * D + 4 * e,
           total == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / total);
}

// Tiles, and shares of the keys, from the sizes alone (what lies in device memory
// is not known here).
void plan(BatchAttnArgs *a) {
    a->tile = 16;
    a->block = KB;
    const int64_t most = (int64_t)a->max_rows * a->G;
    a->one_tile = most <= a->tile;
    a->slots = (int32_t)(a->one_tile ? a->n_seqs : (int64_t)a->n * a->G / a->tile + a->n_seqs);
    const int blocks = (a->max_length + a->block - 1) / a->block;
    const int64_t units = (int64_t)a->slots * a->n_kv_heads;
    const int want = a->lengths ? (int)std::max<int64_t>(1, std::min<int64_t>(blocks / 2, 512 / units)) : 1;
    a->per_split = (blocks + want - 1) / want;
    a->splits = (blocks + a->per_split - 1) / a->per_split;
}

size_t o_bytes(const BatchAttnArgs &a, int D) { return sizeof(float) * (size_t)a.splits * a.n * a.n_heads * D; }
size_t workspace_of(const BatchAttnArgs &a, int D) {
    return a.splits == 1 ? 0 : o_bytes(a, D) + sizeof(float2) * (size_t)a.splits * a.n * a.n_heads;
}

template <typename TX, typename TK>
void launch_f32(const BatchAttnArgs &a, int D, hipStream_t s) {
    const dim3 grid((unsigned)(a.slots * a.n_kv_heads), (unsigned)a.splits), block(NW * 64);
    if (D == 16)
        hipLaunchKernelGGL((k_batch_attn_f32<TX, TK, 16>), grid, block, 0, s, a);
    else if (D == 32)
        hipLaunchKernelGGL((k_batch_attn_f32<TX, TK, 32>), grid, block, 0, s, a);
    else if (D == 64)
        hipLaunchKernelGGL((k_batch_attn_f32<TX, TK, 64>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_batch_attn_f32<TX, TK, 128>), grid, block, 0, s, a);
}

template <typename TX>
void launch_join(const BatchAttnArgs &a, int D, hipStream_t s) {
    const dim3 grid((unsigned)(a.n * a.n_heads)), block(JOIN_THREADS);
    if (D == 16)
        hipLaunchKernelGGL((k_batch_join<TX, 16>), grid, block, 0, s, a);
    else if (D == 32)
        hipLaunchKernelGGL((k_batch_join<TX, 32>), grid, block, 0, s, a);
    else if (D == 64)
        hipLaunchKernelGGL((k_batch_join<TX, 64>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_batch_join<TX, 128>), grid, block, 0, s, a);
}

// What both entry points take besides their keys.
sd_status check_call(const void *q, int64_t ld_q, int32_t x_dtype, int32_t n_heads, int32_t n, int32_t n_seqs,
                     int32_t n_kv_heads, int D, const void *out, int64_t ld_out, float *scale) {
    const sd_status st = check_rows(n, n_heads, n_kv_heads);
    if (st != SD_OK)
        return st;
    if (x_dtype != SD_F32 && x_dtype != SD_BF16)
        return report(SD_ERR_INVALID_ARG, "x_dtype must be SD_F32 or SD_BF16");
    if ((int64_t)n * n_heads > 1 << 26 || (int64_t)n_seqs * n_kv_heads > 1 << 22)
        return report(SD_ERR_INVALID_ARG, "a call has at most 2^26 rows times heads and 2^22 sequences times kv heads");
    if (!scale)
        return SD_OK;
    if (!q || !out || !aligned16(q) || !aligned16(out))
        return report(SD_ERR_INVALID_ARG, "q and out must be set and 16-byte aligned");
    const int unit = x_dtype == SD_BF16 ? 8 : 4;
    if (ld_q % unit || ld_out % unit || ld_q < (int64_t)n_heads * D || ld_out < (int64_t)n_heads * D)
        return report(SD_ERR_INVALID_ARG, "ld_q and ld_out must hold a row and be multiples of 16 bytes");
    // (the scores are taken in units of log2)
    *scale = (*scale == 0.0f ? 1.0f / std::sqrt((float)D) : *scale) * 1.4426950408889634f;
    if (!std::isfinite(*scale))
        return report(SD_ERR_INVALID_ARG, "scale, and scale log2(e), must be finite");
    return SD_OK;
}

sd_status launch(const BatchAttnArgs &a, int32_t x_dtype, int32_t dtype, int D, hipStream_t s) {
    if (x_dtype == SD_BF16) {
        if (dtype == SD_BF16)
            launch_f32<uint16_t, uint16_t>(a, D, s);
        else
            launch_f32<uint16_t, float>(a, D, s);
    } else if (dtype == SD_BF16) {
        launch_f32<float, uint16_t>(a, D, s);
    } else {
        launch_f32<float, float>(a, D, s);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        if (x_dtype == SD_BF16)
            launch_join<uint16_t>(a, D, s);
        else
            launch_join<float>(a, D, s);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SD_OK : report(SD_ERR_DEVICE, std::string("batch attention: ") + hipGetErrorString(e));
}

// The sizes of a call over pages, checked.
sd_status paged_sizes(const sd_kv_pages *kv, const sd_batch *batch, int32_t n_heads, int32_t n, bool addresses,
                      BatchAttnArgs *a) {
    sd_status st = check_pages(kv);
    if (st != SD_OK || (st = check_rows(n, n_heads, kv->n_kv_heads)) != SD_OK ||
        (st = check_batch(batch, kv, n, addresses)) != SD_OK)
        return st;
    a->k = kv->k;
    a->v = kv->v;
    a->page_stride = kv->page_stride;
    a->head_stride = kv->head_stride;
    a->row_stride = kv->row_stride;
    a->table = batch->table;
    a->lengths = batch->lengths;
    a->starts = batch->starts;
    a->ld_table = batch->ld_table;
    a->n = n;
    a->n_seqs = batch->n_seqs;
    a->max_rows = std::min(batch->max_rows, n);
    a->max_length = positions_of(*batch, *kv);
    a->n_pages = kv->n_pages;
    a->page_shift = log2_of(kv->page_size);
    a->n_heads = n_heads;
    a->n_kv_heads = kv->n_kv_heads;
    a->G = n_heads / kv->n_kv_heads;
    return SD_OK;
}

sd_status paged_attention(const sd_kv_pages *kv, const sd_batch *batch, const void *q, int64_t ld_q, int32_t x_dtype,
                          int32_t n_heads, int32_t n, float scale, void *out, int64_t ld_out, void *workspace,
                          size_t workspace_bytes, hipStream_t s) {
    BatchAttnArgs a{};
    sd_status st = paged_sizes(kv, batch, n_heads, n, true, &a);
    if (st != SD_OK || (st = check_call(q, ld_q, x_dtype, n_heads, n, a.n_seqs, a.n_kv_heads, kv->head_dim, out, ld_out,
                                        &scale)) != SD_OK)
        return st;
    plan(&a);
    const size_t need = workspace_of(a, kv->head_dim);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need))
        return report(SD_ERR_INVALID_ARG, "these sizes need " + std::to_string(need) +
                                              " bytes of 16-byte aligned workspace");
    a.q = q;
    a.ld_q = ld_q;
    a.out = out;
    a.ld_out = ld_out;
    a.scale = scale;
    if (need) {
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + o_bytes(a, kv->head_dim));
    }
    return launch(a, x_dtype, kv->dtype, kv->head_dim, s);
}

sd_status prompt_attention(const sd_kv_layer *kv, const int32_t *starts, int32_t n_seqs, const void *q, int64_t ld_q,
                           int32_t x_dtype, int32_t n_heads, int32_t n, float scale, void *out, int64_t ld_out,
                           hipStream_t s) {
    sd_status st = check_layer(kv);
    if (st != SD_OK || (st = check_rows(n, n_heads, kv->n_kv_heads)) != SD_OK)
        return st;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || (!starts && n_seqs != 1) || ((uintptr_t)starts & 3))
        return report(SD_ERR_INVALID_ARG, "n_seqs must be in [1, 65536], and 1 without starts, which are 4-byte aligned");
    if ((st = check_call(q, ld_q, x_dtype, n_heads, n, n_seqs, kv->n_kv_heads, kv->head_dim, out, ld_out, &scale)) != SD_OK)
        return st;
    if (n > kv->capacity)
        return report(SD_ERR_CAPACITY, "a layer of capacity " + std::to_string(kv->capacity) + " does not hold " +
                                           std::to_string(n) + " rows");
    BatchAttnArgs a{};
    a.q = q;
    a.ld_q = ld_q;
    a.out = out;
    a.ld_out = ld_out;
    a.k = kv->k;
    a.v = kv->v;
    a.head_stride = kv->head_stride;
    a.row_stride = kv->row_stride;
    a.starts = starts;
    a.scale = scale;
    a.n = a.max_rows = a.max_length = n;
    a.n_seqs = n_seqs;
    a.n_heads = n_heads;
    a.n_kv_heads = kv->n_kv_heads;
    a.G = n_heads / kv->n_kv_heads;
    plan(&a);
    return launch(a, x_dtype, kv->dtype, kv->head_dim, s);
}

}  // namespace

extern "C" {

size_t sd_paged_attention_workspace(const sd_kv_pages *kv, const sd_batch *batch, int32_t x_dtype, int32_t n_heads,
                                    int32_t n) {
    BatchAttnArgs a{};
    if (paged_sizes(kv, batch, n_heads, n, false, &a) != SD_OK ||
        check_call(nullptr, 0, x_dtype, n_heads, n, a.n_seqs, a.n_kv_heads, kv->head_dim, nullptr, 0, nullptr) != SD_OK)
        return 0;
    plan(&a);
    return workspace_of(a, kv->head_dim);
}

sd_status sd_paged_attention(const sd_kv_pages *kv, const sd_batch *batch, const void *q, int64_t ld_q, int32_t x_dtype,
                             int32_t n_heads, int32_t n, float scale, void *out, int64_t ld_out, void *workspace,
                             size_t workspace_bytes, void *hip_stream) {
    SD_GUARD(return paged_attention(kv, batch, q, ld_q, x_dtype, n_heads, n, scale, out, ld_out, workspace,
                                    workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));)
}

sd_status sd_prompt_attention(const sd_kv_layer *kv, const int32_t *starts, int32_t n_seqs, const void *q, int64_t ld_q,
                              int32_t x_dtype, int32_t n_heads, int32_t n, float scale, void *out, int64_t ld_out,
                              void *hip_stream) {
    SD_GUARD(return prompt_attention(kv, starts, n_seqs, q, ld_q, x_dtype, n_heads, n, scale, out, ld_out,
                                     reinterpret_cast<hipStream_t>(hip_stream));)
}

}  // extern "C"
