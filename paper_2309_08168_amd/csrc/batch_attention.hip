// Attention of a batch's rows: over the pages of a cache (sd_paged_attention) and
// over packed keys and values (sd_prompt_attention).
//
// Row i of a sequence, head h: o = sum_k p_k v_k / sum_k p_k, p_k = exp(scale q.k -
// max), over the keys 0 .. past + i.  The m rows of a sequence and the G query heads
// of a kv head share its keys: its m G rows (row = i G + head) are cut into tiles,
// and the keys of a tile into shares, each leaving an unnormalised output with its
// maximum and sum, which a second kernel joins in order; a single share is
// normalised at once.  One pass over the keys: a running maximum m and sum l of a row,
// which, with o, are multiplied by exp(m - m') where m rises to m'.
//
// A call reads the keys and values of its sequences, q, and writes out; it computes 4 D
// flops a (row, head, key).  Tokens and short chains are bound by the read (k_batch_attn_few,
// streams), chunks and prompts by the matrix cores (k_batch_attn_wide for bfloat16 queries,
// k_batch_attn_mfma), float32 caches by either (k_batch_attn_f32).
#include "paged.h"

#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "attn_mfma.h"
#include "host_api.h"

using namespace sdk;

namespace {

constexpr int KB = 64, KB_FEW = 32, NW = 4;  // keys of a block; waves

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
    int32_t paged;                     // whether over pages
    int32_t waves;                     // of a work-group
    int32_t chunks, span;              // of the streams: chunks (0: no streams), keys of a span
    int32_t *spans;                    // [n_seqs + 2]: spans before each sequence, and of a chunk
    int32_t tile, slots, one_tile;     // rows of a tile; tiles at most; whether a sequence has at most one
    int32_t splits, per_split, block;  // shares of the keys; blocks of a share; keys of a block
    int32_t wide;                      // whether k_batch_attn_wide takes it
};

// An address that is the same in every lane, in scalar registers.
__device__ __forceinline__ const uint16_t *uniform(const uint16_t *p) {
    const uint64_t x = (uint64_t)p;
    return (const uint16_t *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 |
                              (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x));
}

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
    int64_t before = 0;  // the slots of the sequences before
    w.seq = t;
    if (!a.one_tile && a.starts && a.n_seqs < 64) {
        // (one round trip: a lane's start, the next one's and its length)
        const int lane = threadIdx.x & 63, j = min(lane, a.n_seqs);
        const int32_t start = a.starts[j], length = a.lengths ? a.lengths[min(j, a.n_seqs - 1)] : 0;
        const int64_t own = (int64_t)start * a.G / a.tile + j;
        const int seq = min((int)__popcll(__ballot(lane >= 1 && lane <= a.n_seqs && own <= t)), a.n_seqs - 1);
        w.seq = seq;
        const int32_t first = __builtin_amdgcn_readlane(start, seq);
        w.rows = seq_rows(first, __builtin_amdgcn_readlane(start, seq + 1), __builtin_amdgcn_readlane(length, seq), a.n,
                          a.max_rows);
        if (!a.lengths)
            w.rows.past = 0;
        const int64_t row0 = (t - ((int64_t)first * a.G / a.tile + seq)) * a.tile, most = (int64_t)w.rows.m * a.G;
        w.row0 = (int32_t)(row0 < 0 || row0 > most ? most : row0);
        return w;
    }
    if (!a.one_tile) {
        const auto slot = [&](int32_t j) { return (int64_t)start_of(a, j) * a.G / a.tile + j; };
        w.seq = min(wave_count(a.n_seqs, t, slot), a.n_seqs - 1);
        before = slot(w.seq);
    }
    w.seq = __builtin_amdgcn_readfirstlane(w.seq);
    w.rows = rows_of(a, w.seq);
    w.rows.first = __builtin_amdgcn_readfirstlane(w.rows.first);
    w.rows.m = __builtin_amdgcn_readfirstlane(w.rows.m);
    w.rows.past = __builtin_amdgcn_readfirstlane(w.rows.past);
    const int64_t row0 = a.one_tile ? 0 : (t - before) * a.tile, most = (int64_t)w.rows.m * a.G;
    w.row0 = __builtin_amdgcn_readfirstlane((int32_t)(row0 < 0 || row0 > most ? most : row0));
    return w;
}

// The waves' states of ROWS rows from row0 on (o [wave][row][D + 4], waves `pitch`
// floats apart; (maximum, sum) [wave][row]) merged in wave order: the result, or with
// part >= 0 that part's state, its rows adjacent there from `part` on, or by
// packed row and head with a.chunks 0.
template <typename TX, int D, int ROWS, int W>
__device__ __forceinline__ void merge_waves(const BatchAttnArgs &a, const Tile &w, const float *o, int pitch,
                                            const float2 *ml, int g, int part) {
#pragma unroll
    for (int i = threadIdx.x; i < ROWS * D / 4; i += W * 64) {
        const int rc = i / (D / 4), e = 4 * (i % (D / 4)), rr = w.row0 + rc;
        if (rr >= w.rows.m * a.G)
            break;  // i only grows
        float m = -INFINITY, L = 0.0f;
        f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < W; ++v)
            m = fmaxf(m, ml[v * ROWS + rc].x);
        const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int v = 0; v < W; ++v) {
            // (a wave without keys has weight zero, output zero)
            const float wt = __builtin_amdgcn_exp2f(ml[v * ROWS + rc].x - mu);
            L = fmaf(wt, ml[v * ROWS + rc].y, L);
            O += wt * load4(o + v * pitch + rc * (D + 4) + e);
        }
        const int node = rr / a.G, head = g * a.G + rr - node * a.G;
        const int64_t row = w.rows.first + node;
        if (part < 0) {
            store4(static_cast<TX *>(a.out) + row * a.ld_out + (int64_t)head * D + e,
                   L == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / L);
        } else {
            const int64_t slot = a.chunks ? (int64_t)part * a.tile + rc : ((int64_t)part * a.n + row) * a.n_heads + head;
            store4(a.part_o + slot * D + e, O);
            if (e == 0)
                a.part_ml[slot] = make_float2(m, L);
        }
    }
}

// ---------------------------------------------------------------------------
// Streams.  Where every sequence is one tile, the keys of a kv head are one stream:
// the spans (of `span` keys) of all its sequences one after the other, cut into
// chunks of as many spans each, a work-group a chunk.  So every work-group
// has the same work, whatever the lengths are: 64 sequences of 500 to 8000 keys
// took 224 us with a work-group a sequence, 190 of 4250 each.  A chunk that holds a sequence
// whole normalises its result; of others a chunk has at most two, one that began
// before it (part 0) and one that goes on after it (part 1).
constexpr int MAX_STREAM = 1024;  // sequences: every work-group adds up their spans

struct Stream {
    int32_t pre[MAX_STREAM + 1], wave[8], first;
};
// Spans of a sequence: one at least where it has rows, which get zeros.
__device__ __forceinline__ int32_t spans_of(const BatchAttnArgs &a, const SeqRows &r) {
    return r.m == 0 ? 0 : max(1, (seen_from(r.past + r.m - 1, a.max_length) + a.span - 1) / a.span);
}
// The spans [at, end) of chunk c and the sequence that `at` is in; false: none.
template <int W>  // waves
__device__ __forceinline__ bool chunk_of(const BatchAttnArgs &a, Stream &st, int32_t c, int32_t *at, int32_t *end,
                                         int32_t *seq) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (a.n_seqs + W * 64 - 1) / (W * 64);
    int32_t own[MAX_STREAM / (W * 64)], sum = 0;
#pragma unroll
    for (int j = 0; j < MAX_STREAM / (W * 64); ++j) {
        const int s = tid * per + j;
        own[j] = j < per && s < a.n_seqs ? spans_of(a, rows_of(a, s)) : 0;
        sum += own[j];
    }
    int32_t upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t y = __shfl_up(upto, d, 64);
        upto += lane >= d ? y : 0;
    }
    if (lane == 63)
        st.wave[wave] = upto;
    __syncthreads();
    int32_t before = upto - sum, total = 0;
#pragma unroll
    for (int v = 0; v < W; ++v) {
        before += v < wave ? st.wave[v] : 0;
        total += st.wave[v];
    }
    const int32_t len = max((total + a.chunks - 1) / a.chunks, 1);
    *at = c * len;
    *end = min(*at + len, total);
#pragma unroll
    for (int j = 0; j < MAX_STREAM / (W * 64); ++j) {
        const int s = tid * per + j;
        if (j < per && s < a.n_seqs) {
            st.pre[s] = before;
            if (before <= *at && *at < before + own[j])
                st.first = s;
            before += own[j];
            if (s == a.n_seqs - 1)
                st.pre[a.n_seqs] = before;
        }
    }
    __syncthreads();
    *seq = st.first;
    return *at < *end;
}
// What the join reads, by one work-group.
template <int W>
__device__ __forceinline__ void keep_spans(const BatchAttnArgs &a, const Stream &st) {
    const int32_t total = st.pre[a.n_seqs], len = max((total + a.chunks - 1) / a.chunks, 1);
    for (int s = threadIdx.x; s <= a.n_seqs; s += W * 64)
        a.spans[s] = st.pre[s];
    if (threadIdx.x == 0)
        a.spans[a.n_seqs + 1] = len;
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
//
// Tokens: bound by the read (8 sequences of 700 to 1500 keys, 40 heads of 128, 88 us, 4.5
// TB/s).  Prompts: four of 3115 rows, 4 heads of 64, 285 us, 70 of the 154 TFLOP/s that a
// large float32 product reaches; 700 rows, 64 heads on 8 of 128, 126 us, 64.  Float32
// products and vector operations take turns (32 products 1035 cycles of a SIMD, 128
// multiply-adds 364, both 1351), but a softmax left out gains 2 to 7%, and loads left out 11
// to 24: the rest is the start and the merge of tiles of 16 rows, few blocks each.  Tiles of
// 32 rows: 136 -> 124 us at 64 heads, 81 -> 93 at 4.  K by whole rows, lane offsets kept,
// chains of products cut in four, a maximum that may lag: none faster, or slower by 5%.

template <typename TX, int D>
__global__ __launch_bounds__(NW * 64, 2) void k_batch_attn_f32(BatchAttnArgs a) {
    constexpr int ES = D / 16, OP = D + 4, W = ES < 4 ? ES : 4;  // W: elements of a load of V
    typedef float vec_t __attribute__((ext_vector_type(W)));
    __shared__ __attribute__((aligned(16))) float tile[NW][16 * OP];
    __shared__ float2 ml[NW][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15,
              g4 = lane >> 4;
    const int g = blockIdx.x % a.n_kv_heads, split = blockIdx.y;
    // (from the last tile, which has the most keys, to the first)
    const Tile w = tile_of(a, a.slots - 1 - blockIdx.x / a.n_kv_heads);
    const int rows = w.rows.m * a.G;
    if (w.row0 >= rows)
        return;  // uniform
    auto sees = [&](int rr) { return seen_from(w.rows.past + rr / a.G, a.max_length); };
    const int klen = sees(min(w.row0 + 15, rows - 1)), kall = sees(w.row0);
    const int b0 = split * a.per_split, b1 = min(b0 + a.per_split, (klen + KB - 1) / KB);
    if (a.splits > 1 && b0 >= b1)
        return;
    const float *K = static_cast<const float *>(a.k) + (int64_t)g * a.head_stride;
    const float *V = static_cast<const float *>(a.v) + (int64_t)g * a.head_stride;
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
        const float *kp = K + place(b, page) + min(c, klen - 1 - KB * b - 16 * wave) * a.row_stride + 4 * g4;
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
        vec_t vx[4][ES / W];
        const float *vb = V + place(b, page);
        if (some) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float *vp = vb + min(4 * g4 + v, klen - 1 - first) * a.row_stride + W * c;
#pragma unroll
                for (int t = 0; t < ES / W; ++t)
                    vx[v][t] = *reinterpret_cast<const vec_t *>(vp + 16 * W * t);
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
                const float *vr = vb + min(key, klen - 1 - first) * a.row_stride;
                float pk = p[0];
#pragma unroll
                for (int v = 1; v < 4; ++v)
                    pk = (key & 3) == v ? p[v] : pk;
                pk = __shfl(pk, 16 * (key >> 2) + c, 64);
#pragma unroll
                for (int t = 0; t < ES; ++t)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float x = vr[element(t, u)];
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
    merge_waves<TX, D, 16, NW>(a, w, &tile[0][0], 16 * OP, &ml[0][0], g, a.splits > 1 ? split : -1);
}

// ---------------------------------------------------------------------------
// bfloat16 caches: matrix cores.  bfloat16 queries and softmax weights are one
// bfloat16 term each (the scores are scaled in float32); float32 ones (q times scale
// log2(e)) are held as three terms that add up to them exactly, so that only the
// float32 sums round.
//
// NQ x NK waves take 32 NQ rows of a kv head; the K and V rows of a block come
// straight into LDS one block ahead, and all waves read them there.  NK = 2 waves
// share a block's keys where there are few rows.  32 keys at a time: scores S^T =
// K q as 32x32x16 products leave lane (col, half) the keys 8 (v / 4) + 4 half +
// v % 4, v = 0..15, of row col; values v = 8 j .. 8 j + 7 are the slots of the
// j-th 16-key value product, so the weights stay in their lanes and V^T is read
// to match, transposed on its way out of LDS.
//
// LDS lines are 256 bytes, 16 chunks of 16 bytes: 128 / D rows.  Chunk p of line s
// lies at p ^ swz(s), which spreads the 16 rows of a K read and the four rows of a
// V read over all banks; the loads permute the chunks of a line on the way in.
// The 16 rows of a group lie in one page, so a load of a group's rows (heads of 32 and
// more) has one base.
//
// Bound by the matrix cores: 1023 float32 rows, 40 heads of 128, 39.6 us, 0.81 PFLOP/s issued
// (three terms), where a large product of random operands reaches 1.42.  A weight of a bfloat16
// call is rounded to bfloat16 for its product with V, by 2^-8 of it at most; a second term would take half again as many products (the few rows of
// k_batch_attn_few have it, where the read hides it).

// Where the four 16-key groups of a block start: elements from a head's first, and
// whether there are keys (a bit each).
struct Groups {
    int64_t off[4];
    uint32_t ok;
};
// Their entries of the table, asked for a block ahead of what needs them.
struct Entries {
    int32_t page[4];
};
template <bool PAGED>
__device__ __forceinline__ Entries entries_of(const BatchAttnArgs &a, const Tile &w, int first, int klen) {
    Entries e;
    if constexpr (!PAGED)
        return e;
    const int32_t *row = a.table + (int64_t)w.seq * a.ld_table;
    e.page[0] = first < klen ? row[first >> a.page_shift] : -1;
    if (a.page_shift < 6) {
#pragma unroll
        for (int j = 1; j < 4; ++j)
            e.page[j] = first + 16 * j < klen ? row[(first + 16 * j) >> a.page_shift] : -1;
    }
    return e;
}
template <bool PAGED>
__device__ __forceinline__ Groups groups_of(const BatchAttnArgs &a, const Tile &w, const Entries &e, int first, int klen) {
    Groups k;
    k.ok = 15;  // (keys past the last are masked by their number)
    if (PAGED && a.page_shift < 6) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // (without a page: any rows, which are masked, and taken for finite)
            const int page = __builtin_amdgcn_readfirstlane(e.page[j]);
            const bool there = (uint32_t)page < (uint32_t)a.n_pages;
            k.off[j] = (there ? page * a.page_stride : 0) +
                       (int64_t)((first + 16 * j) & ((1 << a.page_shift) - 1)) * a.row_stride;
            k.ok &= there || first + 16 * j >= klen ? 15u : ~(1u << j);
        }
        return k;
    }
    if constexpr (PAGED) {
        const int page = __builtin_amdgcn_readfirstlane(e.page[0]);
        const bool there = (uint32_t)page < (uint32_t)a.n_pages;
        k.off[0] = (there ? page * a.page_stride : 0) + (int64_t)(first & ((1 << a.page_shift) - 1)) * a.row_stride;
        k.ok = there ? 15 : 0;
    } else {
        k.off[0] = (int64_t)(w.rows.first + first) * a.row_stride;
    }
    k.off[1] = k.off[2] = k.off[3] = 0;
    return k;
}
// Where row r of a block starts, its rows all following the first (one) or by groups.
__device__ __forceinline__ int64_t row_at(const Groups &k, bool one, int r, int64_t row_stride) {
    // (the four as values: chosen by address, they would lie in memory)
    const int64_t o0 = k.off[0], o1 = k.off[1], o2 = k.off[2], o3 = k.off[3];
    const int j = one ? 0 : r >> 4;
    return (j == 0 ? o0 : j == 1 ? o1 : j == 2 ? o2 : o3) + (one ? r : r & 15) * row_stride;
}
// The keys of a block that are seen by one who sees `count` of them, as bits.
__device__ __forceinline__ uint64_t seen_bits(int count, uint32_t ok) {
    uint64_t groups = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        groups |= (ok >> j) & 1 ? 0xffffull << (16 * j) : 0;
    return (count >= 64 ? ~0ull : count <= 0 ? 0 : (1ull << count) - 1) & groups;
}

// Where keys come from: packed, pages (tiles, and shares of their keys), or pages as a
// stream (a tile a sequence).
enum Source { PACKED, PAGES, STREAM };

template <typename TX, int D, int NQ, int NK, Source FROM>
__global__ __launch_bounds__(64 * NQ * NK, 2) void k_batch_attn_mfma(BatchAttnArgs a) {
    constexpr bool EXACT = sizeof(TX) == 4, PAGED = FROM != PACKED;
    constexpr int T = EXACT ? X_TERMS : 1, WAVES = NQ * NK, ES = D / 16, ET = D < 32 ? 1 : D / 32;
    using L = Lines<D>;
    __shared__ __attribute__((aligned(1024))) uint16_t kv[2][2][KB * D];  // [block % 2][K, V]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31,
              half = lane >> 5;
    const int wq = wave % NQ, wk = wave / NQ;
    const int g = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const uint16_t *K = static_cast<const uint16_t *>(a.k) + (int64_t)g * a.head_stride;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + (int64_t)g * a.head_stride;
    __shared__ typename std::conditional<FROM == STREAM, Stream, int>::type stream;
    int32_t seq = 0, at = 0, end = 1;  // of a stream: the sequence, the spans left
    if constexpr (FROM == STREAM) {
        const bool some = chunk_of<WAVES>(a, stream, rest, &at, &end, &seq);
        if (blockIdx.x == 0)
            keep_spans<WAVES>(a, stream);
        if (!some)
            return;  // uniform
    }

    // A wave takes every WAVES-th KB of K's and of V's rows.  Whole blocks: lane
    // offsets that do not change, from the block's first row where its rows follow
    // one another (packed, or pages of a block and more), else from a group's.
    constexpr int NU = (L::C + WAVES - 1) / WAVES, ROWS = 4 * L::RPL;  // loads of a wave; rows of a load
    const bool one = !PAGED || a.page_shift >= 6, near = (one || D > 16) && near_rows(a.row_stride);
    uint32_t off[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const int u = wave + WAVES * i, s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
        off[i] = (uint32_t)(2 * ((int64_t)((s * L::RPL + p / L::C) & (one ? 63 : 15)) * a.row_stride + 8 * (p % L::C)));
    }
    for (;;) {
        Tile w;
        int b0, b1, part = 0;  // blocks of keys; the part of the result, or -1: all of it
        int klen, kall, done = 0;
        auto sees = [&](int rr) { return seen_from(w.rows.past + rr / a.G, a.max_length); };
        if constexpr (FROM == STREAM) {
            seq = __builtin_amdgcn_readfirstlane(seq);
            w.seq = seq;
            w.row0 = 0;
            w.rows = rows_of(a, seq);
        } else {
            // (from the last tile, which has the most keys, to the first)
            w = tile_of(a, a.slots - 1 - rest % a.slots);
        }
        const int rows = w.rows.m * a.G;
        if (w.row0 >= rows)
            return;  // uniform
        klen = __builtin_amdgcn_readfirstlane(sees(min(w.row0 + 32 * NQ, rows) - 1));
        kall = __builtin_amdgcn_readfirstlane(sees(w.row0));
        if constexpr (FROM == STREAM) {
            const int32_t from = at - stream.pre[seq], all = stream.pre[seq + 1] - stream.pre[seq];
            done = min(all - from, end - at);
            b0 = __builtin_amdgcn_readfirstlane(from);
            b1 = __builtin_amdgcn_readfirstlane(from + done);
            part = from == 0 && done == all ? -1 : 2 * (g * a.chunks + rest) + (from == 0);
        } else if constexpr (FROM == PAGES) {
            part = a.splits > 1 ? rest / a.slots : -1;
            b0 = rest / a.slots * a.per_split;
            b1 = b0 + a.per_split;
        } else {
            part = -1;
            b0 = 0;
            b1 = INT32_MAX;
        }
        b1 = min(b1, (klen + KB - 1) / KB);
        if (FROM == PAGES && part >= 0 && b0 >= b1)
            return;
        const int r0 = w.row0 + wq * 32;
        const bool live = r0 < rows;  // uniform over the wave: a wave without rows loads and waits with the others
        const int row = min(r0 + col, rows - 1), node = row / a.G, head = g * a.G + row - node * a.G;
        const int see = seen_from(w.rows.past + node, a.max_length);
        auto load_block = [&](const Groups &k, int first, int buf) {
            if (first + KB <= klen && near) {
                const uint16_t *k0 = uniform(K + k.off[0]), *v0 = uniform(V + k.off[0]);
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const int u = wave + WAVES * i;
                    if (L::C % WAVES == 0 || u < L::C) {  // uniform over the wave
                        if (!one) {
                            const int64_t o = row_at(k, false, ROWS * u / 16 * 16, a.row_stride);
                            k0 = uniform(K + o);
                            v0 = uniform(V + o);
                        }
                        load_to_lds16(k0, off[i], &kv[buf][0][u * 512]);
                        load_to_lds16(v0, off[i], &kv[buf][1][u * 512]);
                    }
                }
            } else {
#pragma unroll 1
                for (int u = wave; u < L::C; u += WAVES) {
                    const int s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
                    // rows past the last: that one
                    const int r = min(s * L::RPL + p / L::C, klen - 1 - first);
                    const int64_t at = row_at(k, one, r, a.row_stride) + 8 * (p % L::C);
                    load_to_lds16(K + at, &kv[buf][0][u * 512]);
                    load_to_lds16(V + at, &kv[buf][1][u * 512]);
                }
            }
        };
        Entries entries = entries_of<PAGED>(a, w, KB * b0, klen);
        // The queries are asked for before the first block: loads return in order.
        const TX *qs =
            static_cast<const TX *>(a.q) + (int64_t)(w.rows.first + node) * a.ld_q + (int64_t)head * D + 8 * half;
        u32x4_t qf[ES][T];
        f32x4_t qx[EXACT ? ES : 1][2];
#pragma unroll
        for (int s = 0; s < ES; ++s) {
            if constexpr (EXACT) {
                qx[s][0] = load4(qs + 16 * s);
                qx[s][1] = load4(qs + 16 * s + 4);
            } else {
                qf[s][0] = *reinterpret_cast<const u32x4_t *>(qs + 16 * s);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        Groups k = groups_of<PAGED>(a, w, entries, KB * b0, klen);
        if (b0 < b1)
            load_block(k, KB * b0, 0);
        entries = entries_of<PAGED>(a, w, KB * (b0 + 1), klen);
        // Rows past the last are zeros, which draw less power than copies of it.
        const bool mine = r0 + col < rows;
#pragma unroll
        for (int s = 0; s < ES; ++s) {
            if constexpr (EXACT) {
                const float scale = mine ? a.scale : 0.0f;
                query_terms(qx[s][0] * scale, qx[s][1] * scale, qf[s]);
            } else {
                // (a negative scale as one of q, so that the largest score stays the largest)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    qf[s][0][j] = mine ? qf[s][0][j] ^ (a.scale < 0.0f ? 0x80008000u : 0u) : 0u;
            }
        }
        // (a scale that float32 products would take for zero would make NaN of a masked score)
        const float factor = EXACT ? 1.0f : fmaxf(fabsf(a.scale), 1.17549435e-38f);
        // V^T reads: ds_read_b64_tr_b16 hands lane l of each 16-lane group element
        // l % 4 of the 8 bytes that lanes l / 4 + 4 k (k = 0..3) point at, so lane l
        // points at row 4 half + l / 4 % 4, columns 16 (l / 16 % 2) + 4 (l % 4) ...
        // (head_dim 16: columns past it repeat the first, in output rows that
        // nothing reads)
        const int v_lane = 2 * (KB * D + L::at(4 * half + ((lane >> 2) & 3), (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) % L::C) +
                                4 * (lane & 1));
        const char *lds = reinterpret_cast<const char *>(kv);
        float m_run = -INFINITY, l_run = 0.0f;
        f32x16_t o[ET];
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                o[et][v] = 0.0f;

        int buf = 0;
        for (int b = b0; b < b1; ++b, buf ^= 1) {
            const int first = KB * b;
            const Groups now = k;
            // this wave's loads of the block have landed, then everyone's; every
            // read of the other buffer has returned
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (b + 1 < b1) {
                k = groups_of<PAGED>(a, w, entries, first + KB, klen);
                load_block(k, first + KB, buf ^ 1);
                entries = entries_of<PAGED>(a, w, first + 2 * KB, klen);
            }
            const bool full = first + KB <= kall && now.ok == 15;  // every row sees every key
            bool odd = false;
            if (!full) {
                // A row must not add 0 times an infinity or NaN of a value that it
                // does not see: they are taken out here, and put where they belong
                // beside the products.
                uint16_t *vs = kv[buf][1];
                for (int c = threadIdx.x; c < KB * D / 8; c += 64 * WAVES) {
                    u32x4_t x = reinterpret_cast<const u32x4_t *>(vs)[c];
                    bool hit = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t y = without_odd(x[j]);
                        hit |= y != x[j];
                        x[j] = y;
                    }
                    if (hit)
                        reinterpret_cast<u32x4_t *>(vs)[c] = x;
                    odd |= hit;
                }
                odd = __syncthreads_or(odd);
            }
            const uint64_t visible = full ? ~0ull : seen_bits(see - first, now.ok);
#pragma unroll 1
            for (int h = wk; h < 2; h += NK) {
                const uint32_t bits = h ? (uint32_t)(visible >> 32) : (uint32_t)visible;
                if (!live || (!full && !__any(bits != 0)))
                    continue;  // uniform over the wave: no row of it sees these keys
                f32x16_t s;
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    s[v] = 0.0f;
                // byte addresses in LDS: rows 32 h + col, chunk 2 e + half at xk ^ 32 e.
                // (Hidden from the compiler, which would keep every address of the
                // loop in a register and spill.)
                int xk = 2 * (buf * 2 * KB * D + 32 * h * D + L::at(col, half));
                int xv = 2 * (buf * 2 * KB * D + 32 * h * D) + v_lane;
                asm volatile("" : "+v"(xk), "+v"(xv));
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int e = 0; e < ES; ++e) {
                    const u32x4_t kf = *reinterpret_cast<const u32x4_t *>(lds + (xk ^ (32 * e)));
#pragma unroll
                    for (int i = 0; i < T; ++i)
                        s = mfma32(kf, qf[e][i], s);
                }
                __builtin_amdgcn_s_setprio(0);
                if (!full) {
                    uint32_t own = bits >> (4 * half);
                    asm volatile("" : "+v"(own));  // (a branch, and not selects in every block)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        s[v] = (own >> (8 * (v >> 2) + (v & 3))) & 1 ? s[v] : -INFINITY;
                }
                float mx = s[0];
#pragma unroll
                for (int v = 1; v < 16; ++v)
                    mx = fmaxf(mx, s[v]);
                {
                    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                    mx = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
                }
                if constexpr (!EXACT)
                    mx *= factor;
                const bool grows = mx > m_run + SLACK;
                if (__any(grows)) {
                    // (a row that has seen no key yet keeps zeros)
                    const float m_new = grows ? mx : m_run;
                    const float sc = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
                    l_run *= sc;
#pragma unroll
                    for (int et = 0; et < ET; ++et)
                        o[et] *= sc;
                    m_run = m_new;
                }
                const float m_use = m_run == -INFINITY ? 0.0f : m_run;
                // (the running sum is rounded once for the 16 weights)
                float p[16], sum = 0.0f;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    p[v] = __builtin_amdgcn_exp2f(EXACT ? s[v] - m_use : fmaf(s[v], factor, -m_use));
                    sum += p[v];
                }
                l_run += sum;
                if (odd) {
                    // what was taken out, from memory: lane (col, half) holds
                    // elements 32 et + 8 (v / 4) + 4 half + v % 4 of row col
#pragma unroll 1
                    for (int key = 0; key < 32; ++key) {
                        float pk = 0.0f;
                        const int own = 4 * (key >> 3) + (key & 3);
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            pk = v == own ? p[v] : pk;
                        pk = __shfl(pk, col + 32 * ((key >> 2) & 1), 64);
                        const uint16_t *vr = V + row_at(now, one, min(32 * h + key, klen - 1 - first), a.row_stride);
#pragma unroll
                        for (int et = 0; et < ET; ++et)
#pragma unroll
                            for (int v = 0; v < 16; ++v) {
                                const int e = 32 * et + 8 * (v >> 2) + 4 * half + (v & 3);
                                const float x = e < D ? load1(vr + e) : 0.0f;
                                if (pk != 0.0f && !finite(x))
                                    o[et][v] = fmaf(pk, x, o[et][v]);
                            }
                    }
                }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    u32x4_t pf[T];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        if constexpr (EXACT) {
                            uint32_t t[T];
                            terms2(p[8 * j + 2 * u], p[8 * j + 2 * u + 1], t);
#pragma unroll
                            for (int i = 0; i < T; ++i)
                                pf[i][u] = t[i];
                        } else {
                            pf[0][u] = cvt_pk(p[8 * j + 2 * u], p[8 * j + 2 * u + 1]);
                        }
                    }
                    // A operand V^T: column 32 et + col of keys 16 j + 8 I + 4 half +
                    // 0..3, the row's chunks of et and I one exclusive or away
#pragma unroll
                    for (int et = 0; et < ET; ++et) {
                        u32x4_t vf;
#pragma unroll
                        for (int I = 0; I < 2; ++I) {
                            const char *src = lds + (xv ^ (64 * et) ^ (I ? (D == 16 ? 16 : 32) : 0)) + 2 * (16 * j + 8 * I) * D;
                            const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)src);
                            const u32x2_t y = __builtin_bit_cast(u32x2_t, x);
                            vf[2 * I] = y[0];
                            vf[2 * I + 1] = y[1];
                        }
#pragma unroll
                        for (int i = 0; i < T; ++i)
                            o[et] = mfma32(vf, pf[i], o[et]);
                    }
                }
                __builtin_amdgcn_s_setprio(0);
            }
        }
        {
            const auto lr = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
            l_run = __uint_as_float(lr[0]) + __uint_as_float(lr[1]);
        }
        if constexpr (NK == 2) {
            // the second half of the keys joins the first: its states through LDS,
            // 16 ET + 2 words a lane
            static_assert(sizeof(kv) >= NQ * 64 * (16 * ET + 2) * 4 || D < 128, "LDS for the states");
            __shared__ float st[D == 128 ? 1 : NQ * 64 * (16 * ET + 2)];
            float *to = D == 128 ? reinterpret_cast<float *>(kv) : st;
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (wk == 1) {
#pragma unroll
                for (int et = 0; et < ET; ++et)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        to[((16 * et + v) * NQ + wq) * 64 + lane] = o[et][v];
                to[(16 * ET * NQ + wq) * 64 + lane] = m_run;
                to[((16 * ET + 1) * NQ + wq) * 64 + lane] = l_run;
            }
            __syncthreads();
            if (wk == 0) {
                const float m2 = to[(16 * ET * NQ + wq) * 64 + lane], l2 = to[((16 * ET + 1) * NQ + wq) * 64 + lane];
                const float m = fmaxf(m_run, m2), mu = m == -INFINITY ? 0.0f : m;
                const float w1 = __builtin_amdgcn_exp2f(m_run - mu), w2 = __builtin_amdgcn_exp2f(m2 - mu);
                m_run = m;
                l_run = l_run * w1 + l2 * w2;
#pragma unroll
                for (int et = 0; et < ET; ++et)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        o[et][v] = o[et][v] * w1 + to[((16 * et + v) * NQ + wq) * 64 + lane] * w2;
            }
        }
        if (mine && wk == 0) {
            const int64_t packed = w.rows.first + node;
            const int64_t slot = FROM == STREAM ? (int64_t)part * a.tile + 32 * wq + col
                                                : ((int64_t)part * a.n + packed) * a.n_heads + head;
            TX *out = static_cast<TX *>(a.out) + packed * a.ld_out + (int64_t)head * D;
            const float inv = part >= 0 ? 1.0f : l_run == 0.0f ? 0.0f : 1.0f / l_run;
#pragma unroll
            for (int et = 0; et < ET; ++et)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int e = 32 * et + 8 * q + 4 * half;
                    const f32x4_t y = f32x4_t{o[et][4 * q], o[et][4 * q + 1], o[et][4 * q + 2], o[et][4 * q + 3]} * inv;
                    if (e < D) {
                        if (part < 0)
                            store4(out + e, y);
                        else
                            store4(a.part_o + slot * D + e, y);
                    }
                }
            if (part >= 0 && half == 0)
                a.part_ml[slot] = make_float2(m_run, l_run);
        }
        if constexpr (FROM != STREAM) {
            return;
        } else {
            at += done;
            if (at >= end)
                return;
            // the next sequence that has spans
            do
                ++seq;
            while (stream.pre[seq + 1] <= at);
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------
// bfloat16 queries, tiles of 128 rows: four waves of 32, and steps of 32 keys.  Of
// heads of 128, a step of a wave is 16 products of 32 cycles (8 of K, 8 of V) and a
// softmax of about 90 vector operations, 16 of them exponentials of 8 cycles, which the
// matrix cores do not wait for: step t turns the scores of block t into weights while it
// takes the scores of block t + 1 and the values of block t - 1, a product of each and
// a part of the softmax at a time.  K comes four blocks ahead and V two, in rings
// of four.  The running maximum of block t rescales the sums when block t - 1 is in
// them.  Blocks that some row does not see whole take their parts one after another.
//
// Heads of 128, us: 8000 rows of 32 heads 534 (0.98 PFLOP/s), 1000 rows of 64 heads on 8
// behind 15111 positions 541 (0.94), 16 ragged prompts of 64 heads on 8 378 (0.70: 5 to 6 us of
// start and end a tile).  With k_batch_attn_mfma, whose blocks of 64 keys take their parts
// one after another, 579, 622 and 398.  Of the cycles of a SIMD the products take 57% and the vector operations
// 51%: its two waves nearly take turns.  Rows of zeros take as many cycles (907 thousand) in 383 us: power holds
// the clock, 1.74 GHz with random operands and 2.18 with zeros under the profiler (522 and 415 us).  Loads cost 13% of
// a step, its barrier 2 to 4.  64-key steps need more registers than there are.
struct Halves {  // where the 16-key halves of a block start (elements), and which have a page
    int64_t off[2];
    int ok;
};

template <int D, bool PAGED>
__global__ __launch_bounds__(256, 2) void k_batch_attn_wide(BatchAttnArgs a) {
    constexpr int ES = D / 16, ET = D < 32 ? 1 : D / 32, BE = KB_FEW * D;  // BE: elements of a block
    // A block lies in LDS as lines of 256 bytes; one of 128 elements a row as two blocks
    // of 64, so that all but a few of a lane's addresses differ by a constant.
    constexpr int LD = D < 64 ? D : 64;
    using L = Lines<LD>;
    __shared__ __attribute__((aligned(1024))) uint16_t kv[2][4][BE];  // [K, V][block % 4]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31,
              half = lane >> 5;
    const int g = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int split = rest / a.slots;
    // (from the last tile, which has the most keys, to the first)
    const Tile w = tile_of(a, a.slots - 1 - rest % a.slots);
    const int rows = w.rows.m * a.G;
    if (w.row0 >= rows)
        return;  // uniform
    auto sees = [&](int rr) { return seen_from(w.rows.past + rr / a.G, a.max_length); };
    const int klen = __builtin_amdgcn_readfirstlane(sees(min(w.row0 + 32 * NW, rows) - 1));
    const int kall = __builtin_amdgcn_readfirstlane(sees(w.row0));
    const int t0 = split * a.per_split, t1 = min(t0 + a.per_split, (klen + KB_FEW - 1) / KB_FEW);
    if (a.splits > 1 && t0 >= t1)
        return;
    const int r0 = w.row0 + wave * 32;
    const bool live = r0 < rows;  // uniform over the wave: a wave without rows loads and waits with the others
    const int row = min(r0 + col, rows - 1), node = row / a.G, head = g * a.G + row - node * a.G;
    const int see = seen_from(w.rows.past + node, a.max_length);
    const uint16_t *K = static_cast<const uint16_t *>(a.k) + (int64_t)g * a.head_stride;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + (int64_t)g * a.head_stride;

    // A wave takes every fourth KB of a block of K or of V.  Whole blocks: lane
    // offsets that do not change, from the block's first row where its rows follow one
    // another (packed, or pages of a block and more), else from a half's.
    constexpr int LOADS = D / 16, NU = (LOADS + NW - 1) / NW, ROWS = 4 * L::RPL;  // of a block; of a wave; rows of one
    constexpr int PER = LD / 16;                                                  // loads of LD columns
    const bool one = !PAGED || a.page_shift >= 5, near = (one || D > 16) && near_rows(a.row_stride);
    uint32_t off[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const int u = wave + NW * i, s = 4 * (u % PER) + (lane >> 4), p = (lane & 15) ^ L::swz(s);
        off[i] = (uint32_t)(2 * ((int64_t)((s * L::RPL + p / L::C) & (one ? 31 : 15)) * a.row_stride + 8 * (p % L::C) +
                                 u / PER * LD));
    }
    const int32_t *table = PAGED ? a.table + (int64_t)w.seq * a.ld_table : nullptr;
    // The entries of block t, asked for a step before they are needed.
    struct Pages {
        int32_t p[2];
    };
    auto pages_of = [&](int t) {
        Pages e{{-1, -1}};
        if constexpr (PAGED) {
            const int first = KB_FEW * t;
            if (first < klen)
                e.p[0] = table[first >> a.page_shift];
            if (!one && first + 16 < klen)
                e.p[1] = table[(first + 16) >> a.page_shift];
        }
        return e;
    };
    auto whole_pages_of = [&](int t) {  // the same without a branch
        const int first = KB_FEW * t;
        return Pages{{table[first >> a.page_shift], table[min(first + 16, klen - 1) >> a.page_shift]}};
    };
    auto halves_of = [&](const Pages &e, int t) {
        Halves h;
        const int first = KB_FEW * t;
        h.ok = 3;  // (keys past the last are masked by their number)
        h.off[1] = 0;
        if constexpr (!PAGED) {
            h.off[0] = (int64_t)(w.rows.first + first) * a.row_stride;
        } else {
            // (without a page: any rows, which are masked, and taken for finite)
            const int p = __builtin_amdgcn_readfirstlane(e.p[0]);
            const bool there = (uint32_t)p < (uint32_t)a.n_pages;
            h.off[0] = (there ? p * a.page_stride : 0) + (int64_t)(first & ((1 << a.page_shift) - 1)) * a.row_stride;
            h.ok = there ? 3 : one ? 0 : 2;
            if (!one) {
                const int q = __builtin_amdgcn_readfirstlane(e.p[1]);
                const bool too = (uint32_t)q < (uint32_t)a.n_pages;
                h.off[1] = (too ? q * a.page_stride : 0) + (int64_t)((first + 16) & ((1 << a.page_shift) - 1)) * a.row_stride;
                if (!too && first + 16 < klen)
                    h.ok &= 1;
            }
        }
        return h;
    };
    auto row_at = [&](const Halves &h, int r) {
        // (the two as values: chosen by address, they would lie in memory)
        const int64_t o0 = h.off[0], o1 = h.off[1];
        const bool low = one || r < 16;
        return (low ? o0 : o1) + (low ? r : r - 16) * a.row_stride;
    };
    auto load_block = [&](const uint16_t *m, const Halves &h, int t, uint16_t *to) {
        if (KB_FEW * t + KB_FEW <= klen && near) {
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int u = wave + NW * i;
                if (LOADS % NW == 0 || u < LOADS)  // uniform over the wave
                    load_to_lds16(uniform(m + row_at(h, one || ROWS * (u % PER) < 16 ? 0 : 16)), off[i], to + u * 512);
            }
        } else {
            int own = lane;
            asm volatile("" : "+v"(own));  // (nothing of this is kept in registers over the loop)
#pragma unroll 1
            for (int u = wave; u < LOADS; u += NW) {
                const int s = 4 * (u % PER) + (own >> 4), p = (own & 15) ^ L::swz(s);
                // rows past the last: that one
                const int r = min(s * L::RPL + p / L::C, klen - 1 - KB_FEW * t);
                load_to_lds16(m + row_at(h, r) + 8 * (p % L::C) + u / PER * LD, to + u * 512);
            }
        }
    };
    // The queries are asked for before the first block: loads return in order.
    const uint16_t *qs =
        static_cast<const uint16_t *>(a.q) + (int64_t)(w.rows.first + node) * a.ld_q + (int64_t)head * D + 8 * half;
    u32x4_t qf[ES];
#pragma unroll
    for (int s = 0; s < ES; ++s)
        qf[s] = *reinterpret_cast<const u32x4_t *>(qs + 16 * s);
    __builtin_amdgcn_sched_barrier(0);
    // Block t + 4 of K and t + 2 of V are asked for in step t (past the last block it
    // again, so that a wave has as many loads under way in every step).
    auto slot = [&](int t) { return (t - t0) & 3; };
    auto load_k = [&](const Pages &e, int t) {
        const int b = min(t, t1 - 1);
        load_block(K, halves_of(e, b), b, kv[0][slot(t)]);
    };
    // (and which halves of the blocks t, t + 1 and t + 2 of V have a page)
    int ok_now = 3, ok_next = 3, ok_after = 3;
    auto load_v = [&](const Pages &e, int t) {
        const int b = min(t, t1 - 1);
        const Halves h = halves_of(e, b);
        load_block(V, h, b, kv[1][slot(t)]);
        return h.ok;
    };
    Pages next_k{}, next_v{};
    if (t0 < t1) {
        load_k(pages_of(t0), t0);
        load_k(pages_of(min(t0 + 1, t1 - 1)), t0 + 1);
        load_k(pages_of(min(t0 + 2, t1 - 1)), t0 + 2);
        ok_next = load_v(pages_of(t0), t0);
        load_k(pages_of(min(t0 + 3, t1 - 1)), t0 + 3);
        ok_after = load_v(pages_of(min(t0 + 1, t1 - 1)), t0 + 1);
        next_k = pages_of(min(t0 + 4, t1 - 1));
        next_v = pages_of(min(t0 + 2, t1 - 1));
    }
    // Rows past the last are zeros, which draw less power than copies of it.  (A
    // negative scale as one of q, so that the largest score stays the largest.)
    const bool mine = r0 + col < rows;
#pragma unroll
    for (int s = 0; s < ES; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            qf[s][j] = mine ? qf[s][j] ^ (a.scale < 0.0f ? 0x80008000u : 0u) : 0u;
    // (a scale that float32 products would take for zero would make NaN of a masked score)
    const float factor = fmaxf(fabsf(a.scale), 1.17549435e-38f);
    // Where a lane reads K (row col, chunk 2 e + half) and V^T (as in k_batch_attn_mfma) in
    // slot 0: what changes them by an exclusive or, a register each.
    constexpr int KA = ES < 4 ? ES : 4;
    int ka[KA], va[2][2];
    const int k_lane = 2 * L::at(col, half);
    const int v_lane = 2 * (4 * BE + L::at(4 * half + ((lane >> 2) & 3), (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) % L::C) +
                            4 * (lane & 1));
#pragma unroll
    for (int e = 0; e < KA; ++e)
        ka[e] = k_lane ^ (32 * e);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int I = 0; I < 2; ++I)
            va[x][I] = v_lane ^ (64 * x) ^ (I ? (D == 16 ? 16 : 32) : 0);
    const char *lds = reinterpret_cast<const char *>(kv);
    float m_run = -INFINITY, l_run = 0.0f;
    f32x16_t o[ET], s0, s1;
    u32x4_t p0[2], p1[2];  // weights of keys 16 j .. of a block, in the slots of its value products
#pragma unroll
    for (int et = 0; et < ET; ++et)
#pragma unroll
        for (int v = 0; v < 16; ++v)
            o[et][v] = 0.0f;

    // of the block whose slot starts `at` bytes from where the addresses point
    auto read_k = [&](int at, int e) {
        return *reinterpret_cast<const u32x4_t *>(lds + ka[e % KA] + at + e / 4 * (2 * KB_FEW * LD));
    };
    auto read_v = [&](int at, int i) {
        const int j = i / ET, et = i % ET;
        u32x4_t vf;
#pragma unroll
        for (int I = 0; I < 2; ++I) {
            const char *src = lds + va[et & 1][I] + at + et / 2 * (2 * KB_FEW * LD) + 2 * (16 * j + 8 * I) * LD;
            const u32x2_t y = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)src));
            vf[2 * I] = y[0];
            vf[2 * I + 1] = y[1];
        }
        return vf;
    };
    constexpr int SLOT = 2 * BE;  // bytes
    // Moves the lane addresses on by two slots, of four.
    auto turn_k = [&]() {
#pragma unroll
        for (int e = 0; e < KA; ++e)
            asm volatile("v_xor_b32 %0, %1, %0" : "+v"(ka[e]) : "n"(2 * SLOT));
    };
    auto turn_v = [&]() {
#pragma unroll
        for (int x = 0; x < 4; ++x)
            asm volatile("v_xor_b32 %0, %1, %0" : "+v"(va[x >> 1][x & 1]) : "n"(2 * SLOT));
    };
    // The softmax of a block's scores in parts: the row's maximum of them, the new
    // running one, and weights v0 .. v1 - 1.
    struct Soft {
        float mx, m_use, sc, sum[2], x[16];
        bool grows;
    };
    auto soft_max = [&](const f32x16_t &s, Soft &f) {
        // (a tree: a chain of them would wait for each)
        const float m0 = fmaxf(fmaxf(s[0], s[1]), s[2]), m1 = fmaxf(fmaxf(s[3], s[4]), s[5]),
                    m2 = fmaxf(fmaxf(s[6], s[7]), s[8]), m3 = fmaxf(fmaxf(s[9], s[10]), s[11]),
                    m4 = fmaxf(fmaxf(s[12], s[13]), s[14]);
        f.mx = fmaxf(fmaxf(fmaxf(fmaxf(m0, m1), m2), fmaxf(m3, m4)), s[15]);
    };
    auto soft_grow = [&](Soft &f) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(f.mx), __float_as_uint(f.mx), false, false);
        const float mx = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) * factor;
        f.grows = mx > m_run + SLACK;
        const float m_new = f.grows ? mx : m_run;
        f.m_use = m_new == -INFINITY ? 0.0f : m_new;
        // (a row that has seen no key yet keeps zeros; one whose maximum stays, its sums)
        f.sc = __builtin_amdgcn_exp2f(m_run - f.m_use);
        m_run = m_new;
    };
    // Weights 4 g .. 4 g + 3: their exponents, powers, and sums and words.
    auto soft_exponents = [&](const f32x16_t &s, Soft &f, int g) {
#pragma unroll
        for (int v = 4 * g; v < 4 * g + 4; ++v)
            f.x[v] = fmaf(s[v], factor, -f.m_use);
    };
    auto soft_powers = [&](Soft &f, int g) {
#pragma unroll
        for (int v = 4 * g; v < 4 * g + 4; ++v) {
            f.x[v] = __builtin_amdgcn_exp2f(f.x[v]);
            asm volatile("" : "+v"(f.x[v]));  // (here, and not where it is used)
        }
    };
    auto soft_words = [&](Soft &f, u32x4_t (&p)[2], int g) {
#pragma unroll
        for (int v = 4 * g; v < 4 * g + 4; v += 2) {
            f.sum[0] = v ? f.sum[0] + f.x[v] : f.x[v];
            f.sum[1] = v ? f.sum[1] + f.x[v + 1] : f.x[v + 1];
            uint32_t word = cvt_pk(f.x[v], f.x[v + 1]);
            asm volatile("" : "+v"(word), "+v"(f.sum[0]), "+v"(f.sum[1]));
            p[v >> 3][(v >> 1) & 3] = word;
        }
    };
    auto soft_end = [&](const Soft &f) {
        l_run = fmaf(l_run, f.grows ? f.sc : 1.0f, f.sum[0] + f.sum[1]);
        if (__any(f.grows)) {
            const float by = f.grows ? f.sc : 1.0f;
#pragma unroll
            for (int et = 0; et < ET; ++et)
                o[et] *= by;
        }
    };
    // The loads of a step, when those it reads have landed, this wave's, then
    // everyone's, and every read of what they fill has returned.
    constexpr bool EVEN = NU * NW == LOADS;  // every wave has 4 NU loads that may be under way
    auto begin = [&](int t) {
        if constexpr (EVEN)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(4 * NU) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        load_k(next_k, t + 4);
        ok_now = ok_next;
        ok_next = ok_after;
        ok_after = load_v(next_v, t + 2);
        next_k = pages_of(min(t + 5, t1 - 1));
        next_v = pages_of(min(t + 3, t1 - 1));
    };
    // Whether every row sees every key of a block (with its halves' pages).
    auto is_full = [&](int t, int ok) { return KB_FEW * t + KB_FEW <= kall && ok == 3; };
    auto scores = [&](int at, f32x16_t &to) {
#pragma unroll
        for (int e = 0; e < ES; ++e)
            to = mfma32(read_k(at, e), qf[e], e == 0 ? f32x16_t{} : to);
    };
    auto values = [&](int at, const u32x4_t (&p)[2]) {
#pragma unroll
        for (int i = 0; i < 2 * ET; ++i)
            o[i % ET] = mfma32(read_v(at, i), p[i / ET], o[i % ET]);
    };
    // A step of whole blocks: weights of s into p_next, scores of the next block into
    // s_next, values of the one before with its weights p.
    // loads(i): what else part i does.
    constexpr int PARTS = 8;
    auto fast = [&](int at, const f32x16_t &s, f32x16_t &s_next, const u32x4_t (&p)[2], u32x4_t (&p_next)[2], auto loads) {
        constexpr int AHEAD = 2;
        u32x4_t kf[ES], vf[2 * ET];
        Soft f;
        // (the part in which product i of n is)
        auto part_of = [](int i, int n) { return i * PARTS / n; };
#pragma unroll
        for (int i = -AHEAD; i < PARTS; ++i) {
#pragma unroll
            for (int e = 0; e < ES; ++e)
                if (part_of(e, ES) == i + AHEAD)
                    kf[e] = read_k(at, e);
#pragma unroll
            for (int v = 0; v < 2 * ET; ++v)
                if (part_of(v, 2 * ET) == i + AHEAD)
                    vf[v] = read_v(at, v);
            if (i < 0)
                continue;
#pragma unroll
            for (int e = 0; e < ES; ++e)
                if (part_of(e, ES) == i)
                    s_next = mfma32(kf[e], qf[e], e == 0 ? f32x16_t{} : s_next);
#pragma unroll
            for (int v = 0; v < 2 * ET; ++v)
                if (part_of(v, 2 * ET) == i)
                    o[v % ET] = mfma32(vf[v], p[v / ET], o[v % ET]);
            loads(i);
            if (i == 0)
                soft_max(s, f);
            if (i == 1)
                soft_grow(f);
            // (each part's vector operations need none of the same part's)
            if (i >= 4)
                soft_words(f, p_next, i - 4);
            if (i >= 3 && i < 7)
                soft_powers(f, i - 3);
            if (i >= 2 && i < 6)
                soft_exponents(s, f, i - 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        soft_end(f);
    };
    // The values of a block that some row does not see whole: a row must not add 0 times
    // an infinity or NaN of a value that it does not see.  They are taken out in
    // LDS, and put where they belong from memory.
    auto values_apart = [&](int t, int at, const u32x4_t (&p)[2]) {
        uint16_t *vs = kv[1][slot(t)];
        bool odd = false;
        int own = threadIdx.x;
        asm volatile("" : "+v"(own));
#pragma unroll 1
        for (int c = own; c < BE / 8; c += 64 * NW) {
            u32x4_t x = reinterpret_cast<const u32x4_t *>(vs)[c];
            bool hit = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t y = without_odd(x[j]);
                hit |= y != x[j];
                x[j] = y;
            }
            if (hit)
                reinterpret_cast<u32x4_t *>(vs)[c] = x;
            odd |= hit;
        }
        odd = __syncthreads_or(odd);
        if (!live)
            return;
        if (odd) {
            const Halves h = halves_of(pages_of(t), t);
            const int col = own & 31, half = (own >> 5) & 1;
            // lane (col, half) holds elements 32 et + 8 (v / 4) + 4 half + v % 4 of row col
#pragma unroll 1
            for (int key = 0; key < KB_FEW; ++key) {
                // the weight of key 16 j + 8 I + 4 half + u: in word 2 I + u / 2 of j
                uint32_t word = 0;
                const int which = 4 * (key >> 4) + 2 * ((key >> 3) & 1) + ((key & 3) >> 1);
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    word = v == which ? p[v >> 2][v & 3] : word;
                word = __shfl(word, col + 32 * ((key >> 2) & 1), 64);
                const float pk = __uint_as_float(key & 1 ? word & 0xffff0000u : word << 16);
                const uint16_t *vr = V + row_at(h, min(key, klen - 1 - KB_FEW * t));
#pragma unroll
                for (int et = 0; et < ET; ++et)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int e = 32 * et + 8 * (v >> 2) + 4 * half + (v & 3);
                        const float x = e < D ? load1(vr + e) : 0.0f;
                        if (pk != 0.0f && !finite(x))
                            o[et][v] = fmaf(pk, x, o[et][v]);
                        __builtin_amdgcn_sched_barrier(0);  // a load at a time: registers
                    }
            }
        }
        values(at, p);
    };

    // One part after another: weights of s1 into p0, the next block's scores into s1.
    auto weigh = [&](int t, int at) {
        if (t + 1 < t1)
            scores(at, s0);
        Soft f;
        soft_max(s1, f);
        soft_grow(f);
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
            soft_exponents(s1, f, g4);
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
            soft_powers(f, g4);
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
            soft_words(f, p0, g4);
        soft_end(f);
        s1 = s0;
    };
    int t = t0;
    bool full = false;  // the block before
    if (t0 < t1) {
        // K of the first two blocks has landed
        if constexpr (EVEN)
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(4 * NU) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        scores(0, s1);
        if (is_full(t0, ok_next)) {
            begin(t0);
            weigh(t0, SLOT);
            full = true;
            ++t;
        }
    }
    // (two steps at a time, so that what they hand on stays in its registers: the first
    // reads K from slots 2 and 3 and V from 0 and 1, the next the other way around)
    bool second = false;
    if (full) {
        turn_k();
        // Where what is asked for lies within whole blocks, too, a step's loads stand
        // between its products.
        // (Rows past the last key, of its block: of its pages, or of rows of the call; not
        // past those.)
        const bool within = PAGED || w.rows.first + KB_FEW * t1 <= a.n;
        const int quick = EVEN && near ? min(within ? t1 - 2 : klen / KB_FEW - 5, kall / KB_FEW - 1) : t0;
        const auto quick_step = [&](int t, int at, const f32x16_t &s, f32x16_t &s_next, const u32x4_t (&p)[2],
                                    u32x4_t (&p_next)[2]) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(4 * NU) : "memory");
            const Halves hk = halves_of(next_k, min(t + 4, t1 - 1)), hv = halves_of(next_v, min(t + 2, t1 - 1));
            ok_next = ok_after;
            ok_after = hv.ok;
            uint16_t *to_k = kv[0][slot(t + 4)], *to_v = kv[1][slot(t + 2)];
            const auto loads = [&](int i) {
                constexpr int EACH = PARTS / 2 / NU;  // parts of a load
                const int j = i / EACH % NU, u = wave + NW * j, r = one || ROWS * (u % PER) < 16 ? 0 : 16;
                if (i % EACH == 0 && i < PARTS / 2)
                    load_to_lds16(uniform(K + row_at(hk, r)), off[j], to_k + u * 512);
                else if (i % EACH == 0)
                    load_to_lds16(uniform(V + row_at(hv, r)), off[j], to_v + u * 512);
                if (PAGED && i == PARTS - 1) {
                    next_k = whole_pages_of(min(t + 5, t1 - 1));
                    next_v = whole_pages_of(min(t + 3, t1 - 1));
                }
            };
            fast(at, s, s_next, p, p_next, loads);  // (a wave without rows, too, with queries of zero)
        };
        while (t < quick && ok_next == 3 && ok_after == 3) {
            quick_step(t, 0, s1, s0, p0, p1);
            quick_step(t + 1, SLOT, s0, s1, p1, p0);
            t += 2;
            turn_k();
            turn_v();
            second = !second;
        }
        if (second)
            turn_v();
        else
            turn_k();
    }
#pragma unroll 1
    for (; t < t1; ++t) {
        begin(t);
        const bool was = full;
        full = is_full(t, ok_now);
        if (live && !full) {
            const int count = see - KB_FEW * t;
            const uint32_t seen = (count >= 32 ? ~0u : count <= 0 ? 0u : (1u << count) - 1) &
                                  ((ok_now & 1 ? 0xffffu : 0u) | (ok_now & 2 ? 0xffff0000u : 0u));
            const uint32_t own = seen >> (4 * half);
#pragma unroll
            for (int v = 0; v < 16; ++v)
                s1[v] = (own >> (8 * (v >> 2) + (v & 3))) & 1 ? s1[v] : -INFINITY;
        }
        if (t > t0) {
            if (!was)
                values_apart(t - 1, SLOT * slot(t - 1), p0);
            else if (live)
                values(SLOT * slot(t - 1), p0);
        }
        if (live)
            weigh(t, SLOT * slot(t + 1));
    }
    if (t0 < t1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (!full)
            values_apart(t1 - 1, SLOT * slot(t1 - 1), p0);
        else if (live)
            values(SLOT * slot(t1 - 1), p0);
    }
    {
        const auto lr = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(lr[0]) + __uint_as_float(lr[1]);
    }
    if (!mine)
        return;
    const int64_t at = (int64_t)(w.rows.first + node), place = ((int64_t)split * a.n + at) * a.n_heads + head;
    uint16_t *out = static_cast<uint16_t *>(a.out) + at * a.ld_out + (int64_t)head * D;
    const float inv = a.splits > 1 ? 1.0f : l_run == 0.0f ? 0.0f : 1.0f / l_run;
#pragma unroll
    for (int et = 0; et < ET; ++et)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = 32 * et + 8 * q + 4 * half;
            const f32x4_t y = f32x4_t{o[et][4 * q], o[et][4 * q + 1], o[et][4 * q + 2], o[et][4 * q + 3]} * inv;
            if (e < D) {
                if (a.splits == 1)
                    store4(out + e, y);
                else
                    store4(a.part_o + place * D + e, y);
            }
        }
    if (a.splits > 1 && half == 0)
        a.part_ml[place] = make_float2(m_run, l_run);
}

// ---------------------------------------------------------------------------
// The same for up to 32 rows of a kv head (one token of up to 32 query heads, or a
// few), where the read of the cache counts and not the products: four waves, each
// with 32-key blocks of its own and no barrier until the end.  K goes straight
// into registers as the A operand of 16x16x32 score products, V straight into the
// wave's LDS, both one block ahead.  Lane (col, grp) receives the keys 16 t + 4 grp +
// v of row col, which are the slots u = 4 t + v that the value products take from it.
// LDS lines are permuted for the reads here: eight rows, two adjacent chunks each.
// A lane holds the table's entry for half a block of the wave, 32 blocks at a time.
// A work-group takes a sequence whole, or the chunk of a stream.
//
// Bound by the read, 6.15 TB/s at most for pages in any order: 64 sequences of 500 to 8000
// keys, 64 heads on 8, 193 us, 5.6 TB/s; one of 60002 49 us, 5.0 (55 in a captured graph of
// such calls).  So weights of bfloat16 calls are two bfloat16 terms, off by 2^-16,
// for products that wait for the read in any case (float32 three, off by less than the
// float32 sums).  Loads that bypass the caches: 229 -> 238 us, 56.7 -> 55.0.
template <typename TX, int D, int QT, int W, bool STREAMED>
__global__ __launch_bounds__(64 * W, W == 8 ? 1 : QT == 1 || D < 128 ? 2 : 1) void k_batch_attn_few(BatchAttnArgs a) {
    constexpr bool EXACT = sizeof(TX) == 4;
    constexpr int T = EXACT ? X_TERMS : 1, TP = EXACT ? X_TERMS : 2;  // of q and of the weights
    constexpr int ES = D < 32 ? 1 : D / 32, ET = D / 16, ROWS = 16 * QT, OP = D + 4;
    using L = FewLines<D>;
    constexpr int VB = KB_FEW * D;  // elements of a V block
    constexpr int WORDS = VB > ROWS * OP ? VB : ROWS * OP;
    __shared__ __attribute__((aligned(1024))) uint32_t tile[W][WORDS];  // two V blocks, or the outputs
    __shared__ float2 ml[W][ROWS];
    __shared__ typename std::conditional<STREAMED, Stream, int>::type stream;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15,
              grp = lane >> 4;
    const int g = blockIdx.x % a.n_kv_heads, chunk = blockIdx.x / a.n_kv_heads;
    int32_t seq = chunk, at = 0, end = 1;
    if constexpr (STREAMED) {
        const bool some = chunk_of<W>(a, stream, chunk, &at, &end, &seq);
        if (blockIdx.x == 0)
            keep_spans<W>(a, stream);
        if (!some)
            return;  // uniform
    }
    for (;;) {
        seq = __builtin_amdgcn_readfirstlane(seq);
        int32_t from = 0, to = 0, all = 0;  // spans
        if constexpr (STREAMED) {
            from = __builtin_amdgcn_readfirstlane(at - stream.pre[seq]);
            all = __builtin_amdgcn_readfirstlane(stream.pre[seq + 1] - stream.pre[seq]);
            to = min(all, from + end - at);
        }
        constexpr int BLOCKS = W;  // of a span
        const int b0 = BLOCKS * from + wave;
        // the entries of this wave's blocks b .., of groups past the table none
        const int32_t *table = a.table + (int64_t)seq * a.ld_table;
        auto entries_from = [&](int b) {
            const int64_t first = KB_FEW * ((int64_t)b + W * (lane >> 1)) + 16 * (lane & 1);
            return first < a.max_length ? table[first >> a.page_shift] : -1;
        };
        int entries = entries_from(b0);
        Tile w;
        w.seq = seq;
        w.row0 = 0;
        w.rows = rows_of(a, seq);
        const int rows = w.rows.m * a.G;
        if (rows == 0)
            return;  // uniform (no sequence of a stream's)
        const int klen = __builtin_amdgcn_readfirstlane(seen_from(w.rows.past + w.rows.m - 1, a.max_length));
        const int kall = __builtin_amdgcn_readfirstlane(seen_from(w.rows.past, a.max_length));
        const int blocks = (klen + KB_FEW - 1) / KB_FEW, b1 = STREAMED ? min(BLOCKS * to, blocks) : blocks;
        const uint16_t *K = static_cast<const uint16_t *>(a.k) + (int64_t)g * a.head_stride;
        const uint16_t *V = static_cast<const uint16_t *>(a.v) + (int64_t)g * a.head_stride;
        uint16_t *vt = reinterpret_cast<uint16_t *>(tile[wave]);

        // Where the halves of a block start (elements), and whether they have a page.
        struct Halves {
            int64_t off[2];
            int ok;
        };
        auto halves_of = [&](int b, int slot) {  // slot: among the entries
            Halves h;
            h.ok = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                // (without a page: any rows, which are masked, and taken for finite)
                const int page = __builtin_amdgcn_readlane(entries, 2 * slot + t);
                const bool there = (uint32_t)page < (uint32_t)a.n_pages;
                h.off[t] = (there ? page * a.page_stride : 0) +
                           (int64_t)((KB_FEW * b + 16 * t) & ((1 << a.page_shift) - 1)) * a.row_stride;
                h.ok |= there ? 1 << t : 0;
            }
            return h;
        };
        // Whole blocks: lane offsets that do not change, from a half's first row.
        // (Of V's loads u, only the lane's place in odd and even ones differs.)
        const bool near = D > 16 && near_rows(a.row_stride);
        const uint32_t koff = (uint32_t)(2 * ((int64_t)col * a.row_stride + (8 * grp) % D));
        uint32_t voff[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
            voff[u] = (uint32_t)(2 * ((int64_t)((lane >> 4) * L::RPL + p / L::C) * a.row_stride + 8 * (p % L::C)));
        }
        u32x4_t kf[2][ES];
        auto load_k = [&](const Halves &h, int first) {
            const bool whole = first + KB_FEW <= klen && near;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                // keys past the last: that one, masked; head_dim 16: the upper slots are zeros of q
                const int r = min(16 * t + col, klen - 1 - first);
                const char *kp = whole ? reinterpret_cast<const char *>(K + h.off[t]) + koff
                                       : reinterpret_cast<const char *>(K + (r < 16 ? h.off[0] : h.off[1]) +
                                                                        (r & 15) * a.row_stride + (8 * grp) % D);
#pragma unroll
                for (int s = 0; s < ES; ++s)
                    kf[t][s] = *reinterpret_cast<const u32x4_t *>(kp + 64 * s);
            }
        };
        auto load_v = [&](const Halves &h, int first, int buf) {
            constexpr int LOAD_ROWS = 4 * L::RPL;
            if (first + KB_FEW <= klen && near) {
#pragma unroll
                for (int u = 0; u < VB / 512; ++u)
                    load_to_lds16(V + h.off[LOAD_ROWS * u / 16] + (int64_t)(LOAD_ROWS * u % 16) * a.row_stride, voff[u & 1],
                                  vt + buf * VB + u * 512);
            } else {
#pragma unroll 1
                for (int u = 0; u < VB / 512; ++u) {
                    const int s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
                    const int r = min(s * L::RPL + p / L::C, klen - 1 - first);
                    load_to_lds16(V + (r < 16 ? h.off[0] : h.off[1]) + (r & 15) * a.row_stride + 8 * (p % L::C),
                                  vt + buf * VB + u * 512);
                }
            }
        };
        Halves k{};
        int b = b0, slot = 0;
        if (b < b1) {
            k = halves_of(b, 0);
            load_k(k, KB_FEW * b);
            load_v(k, KB_FEW * b, 0);
        }
        int see[QT];
        u32x4_t qf[QT][ES][T];
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            const int row = min(16 * i + col, rows - 1), node = row / a.G;
            see[i] = seen_from(w.rows.past + node, a.max_length);
            const TX *qs = static_cast<const TX *>(a.q) + (int64_t)(w.rows.first + node) * a.ld_q +
                           (int64_t)(g * a.G + row - node * a.G) * D + (8 * grp) % D;
            const bool none = (D < 32 && grp >= 2) || 16 * i + col >= rows;  // head_dim 16: the upper half of the reduction
#pragma unroll
            for (int s = 0; s < ES; ++s) {
                if constexpr (EXACT) {
                    const float scale = a.scale;
                    f32x4_t x0 = load4(qs + 32 * s) * scale, x1 = load4(qs + 32 * s + 4) * scale;
                    if (none)
                        x0 = x1 = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                    query_terms(x0, x1, qf[i][s]);
                } else {
                    // (a negative scale as one of q, so that the largest score stays the largest)
                    const u32x4_t x = *reinterpret_cast<const u32x4_t *>(qs + 32 * s);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        qf[i][s][0][j] = none ? 0u : x[j] ^ (a.scale < 0.0f ? 0x80008000u : 0u);
                }
            }
        }
        // (a scale that float32 products would take for zero would make NaN of a masked score)
        const float factor = EXACT ? 1.0f : fmaxf(fabsf(a.scale), 1.17549435e-38f);
        float m_run[QT], l_run[QT];
        f32x4_t o[QT][ET];
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            m_run[i] = -INFINITY;
            l_run[i] = 0.0f;
#pragma unroll
            for (int et = 0; et < ET; ++et)
                o[i][et] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int v_lane = 2 * L::at(4 * grp + (col >> 2), (col & 3) >> 1) + 8 * (col & 1);
        const char *vb = reinterpret_cast<const char *>(vt);

        int buf = 0;
        for (; b < b1; b += W, buf ^= 1) {
            const int first = KB_FEW * b;
            const Halves now = k;
            f32x4_t s[QT][2];
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    s[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int e = 0; e < ES; ++e)
#pragma unroll
                        for (int u = 0; u < T; ++u)
                            s[i][t] = mfma16(kf[t][e], qf[i][e][u], s[i][t]);
                }
            // this block's V has landed (it was asked for before this block's K, or
            // just after), then the next block's loads
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (b + W < b1) {
                if (++slot == 32) {
                    slot = 0;
                    entries = entries_from(b + W);
                }
                k = halves_of(b + W, slot);
                load_v(k, first + W * KB_FEW, buf ^ 1);
                load_k(k, first + W * KB_FEW);
            }
            const bool full = first + KB_FEW <= kall && now.ok == 3;  // every row sees every key
            // Infinities and NaN among values that some row does not see: it must not
            // add 0 times one.  They are taken out here, and put where they belong
            // beside the products.
            bool odd = false;
            if (!full) {
                u32x4_t *vw = reinterpret_cast<u32x4_t *>(vt + buf * VB);
                for (int c = lane; c < VB / 8; c += 64) {
                    u32x4_t x = vw[c];
                    bool hit = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t y = without_odd(x[j]);
                        hit |= y != x[j];
                        x[j] = y;
                    }
                    if (hit)
                        vw[c] = x;
                    odd |= hit;
                }
                odd = __any(odd);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            // (a tile's rows at a time: V again from LDS for the second costs less than
            // the registers of both)
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                float p[8], mx = -INFINITY;
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    p[u] = s[i][u >> 2][u & 3];
                if (!full) {
                    const int count = see[i] - first;
                    uint32_t own = count >= 32 ? ~0u : count <= 0 ? 0u : (1u << count) - 1;
                    own = (own & ((now.ok & 1 ? 0xffffu : 0u) | (now.ok & 2 ? 0xffff0000u : 0u))) >> (4 * grp);
                    asm volatile("" : "+v"(own));  // (a branch, and not selects in every block)
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        p[u] = (own >> (16 * (u >> 2) + (u & 3))) & 1 ? p[u] : -INFINITY;
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    mx = fmaxf(mx, p[u]);
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                if constexpr (!EXACT)
                    mx *= factor;
                const bool grows = mx > m_run[i] + SLACK;
                if (__any(grows)) {
                    const float m_new = grows ? mx : m_run[i];
                    const float sc = m_run[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[i] - m_new);
                    l_run[i] *= sc;
#pragma unroll
                    for (int et = 0; et < ET; ++et)
                        o[i][et] *= sc;
                    m_run[i] = m_new;
                }
                const float m_use = m_run[i] == -INFINITY ? 0.0f : m_run[i];
                float sum = 0.0f;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    p[u] = __builtin_amdgcn_exp2f(EXACT ? p[u] - m_use : fmaf(p[u], factor, -m_use));
                    sum += p[u];
                }
                l_run[i] += sum;
                if (odd) {
                    // lane (col, grp) holds elements 16 et + 4 grp + u of row col
#pragma unroll 1
                    for (int key = 0; key < KB_FEW; ++key) {
                        float pk = 0.0f;
                        const int own = 4 * (key >> 4) + (key & 3);
#pragma unroll
                        for (int u = 0; u < 8; ++u)
                            pk = u == own ? p[u] : pk;
                        pk = __shfl(pk, col + 16 * ((key >> 2) & 3), 64);
                        const int r = min(key, klen - 1 - first);
                        const uint16_t *vr = V + (r < 16 ? now.off[0] : now.off[1]) + (r & 15) * a.row_stride + 4 * grp;
#pragma unroll
                        for (int et = 0; et < ET; ++et) {
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const float x = load1(vr + 16 * et + u);
                                if (pk != 0.0f && !finite(x))
                                    o[i][et][u] = fmaf(pk, x, o[i][et][u]);
                            }
                            __builtin_amdgcn_sched_barrier(0);  // a few loads at a time: registers
                        }
                    }
                }
                u32x4_t pf[TP];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (EXACT) {
                        uint32_t t[T];
                        terms2(p[2 * j], p[2 * j + 1], t);
#pragma unroll
                        for (int u = 0; u < T; ++u)
                            pf[u][j] = t[u];
                    } else {
                        pf[0][j] = cvt_pk(p[2 * j], p[2 * j + 1]);
                        pf[1][j] = cvt_pk(p[2 * j] - __uint_as_float(pf[0][j] << 16),
                                          p[2 * j + 1] - __uint_as_float(pf[0][j] & 0xffff0000u));
                    }
                }
                // A operand V^T: column 16 et + col of keys 16 I + 4 grp + 0..3
                int xv = v_lane + 2 * buf * VB;
                asm volatile("" : "+v"(xv));
#pragma unroll
                for (int et = 0; et < ET; ++et) {
                    u32x4_t vf;
#pragma unroll
                    for (int I = 0; I < 2; ++I) {
                        const char *src = vb + (xv ^ (32 * et)) + 2 * 16 * I * D;
                        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)src);
                        const u32x2_t y = __builtin_bit_cast(u32x2_t, x);
                        vf[2 * I] = y[0];
                        vf[2 * I + 1] = y[1];
                    }
#pragma unroll
                    for (int u = 0; u < TP; ++u)
                        o[i][et] = mfma16(vf, pf[u], o[i][et]);
                }
            }
            // (every read of this block has returned before its buffer is filled again)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        // the waves' states, merged in wave order
        float *mine = reinterpret_cast<float *>(tile[wave]);
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            l_run[i] += __shfl_xor(l_run[i], 16, 64);
            l_run[i] += __shfl_xor(l_run[i], 32, 64);
#pragma unroll
            for (int et = 0; et < ET; ++et)
                *reinterpret_cast<f32x4_t *>(mine + (16 * i + col) * OP + 16 * et + 4 * grp) = o[i][et];
            if (grp == 0)
                ml[wave][16 * i + col] = make_float2(m_run[i], l_run[i]);
        }
        __syncthreads();
        int part = -1;
        if constexpr (STREAMED)
            part = from == 0 && to == all ? -1 : 2 * (g * a.chunks + chunk) + (from == 0);
        merge_waves<TX, D, ROWS, W>(a, w, reinterpret_cast<const float *>(tile), WORDS, &ml[0][0], g, part);
        if constexpr (!STREAMED) {
            return;
        } else {
            at += to - from;
            if (at >= end)
                return;
            // the next sequence that has spans
            do
                ++seq;
            while (stream.pre[seq + 1] <= at);
            __syncthreads();
        }
    }
}

// The shares of a (row, head) joined: a work-group each.  D / 4 lanes hold a row, the
// groups of lanes take the shares in turn and add up in order.  One wave where there are at
// most eight shares: 12800 rows of four joined with attention 58 us, 68 with four waves.
template <typename TX, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void k_batch_join(BatchAttnArgs a) {
    constexpr int LANES = D / 4, NG = THREADS / LANES;
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

// The parts of a sequence joined, of a stream's chunks: a work-group a row of a
// (sequence, kv head).  4 to 5 us, of which about 2.5 are a launch's.
template <typename TX, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void k_batch_join_stream(BatchAttnArgs a, int rows_most) {
    constexpr int LANES = D / 4, NG = THREADS / LANES;
    __shared__ f32x4_t red[NG][LANES];
    const int lane = threadIdx.x & 63, e = threadIdx.x % LANES, gi = threadIdx.x / LANES;
    const int rr = blockIdx.x % rows_most, unit = blockIdx.x / rows_most, g = unit % a.n_kv_heads,
              s = unit / a.n_kv_heads;
    const int32_t at = a.spans[s], end = a.spans[s + 1], len = a.spans[a.n_seqs + 1];
    const SeqRows rows = rows_of(a, s);
    if (rr >= rows.m * a.G || at == end)
        return;  // uniform
    const int c0 = at / len, parts = (end - 1) / len - c0 + 1;
    if (parts == 1)
        return;
    // the first is part 1 of its chunk, the others are part 0
    auto slot_of = [&](int j) { return (int64_t)(2 * (g * a.chunks + c0 + j) + (j == 0)) * a.tile + rr; };
    constexpr int J = 4;
    f32x4_t x[J];
#pragma unroll
    for (int j = 0; j < J; ++j)
        x[j] = load4(a.part_o + slot_of(min(gi + j * NG, parts - 1)) * D + 4 * e);
    const float2 first = a.part_ml[slot_of(min(lane, parts - 1))];
    float m = first.x;
    for (int j = lane + 64; j < parts; j += 64)
        m = fmaxf(m, a.part_ml[slot_of(j)].x);
    m = wave_max_all(m);
    const float mu = m == -INFINITY ? 0.0f : m;
    const float w0 = __builtin_amdgcn_exp2f(first.x - mu);  // of part `lane`
    float sum = lane < parts ? w0 * first.y : 0.0f;
    for (int j = lane + 64; j < parts; j += 64) {
        const float2 v = a.part_ml[slot_of(j)];
        sum = fmaf(__builtin_amdgcn_exp2f(v.x - mu), v.y, sum);
    }
    const float total = wave_sum_all(sum);
    f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int p = gi + j * NG;
        const float wt = __shfl(w0, p & 63, 64);
        if (p < parts)
            O += (p < 64 ? wt : __builtin_amdgcn_exp2f(a.part_ml[slot_of(p)].x - mu)) * x[j];
    }
#pragma unroll 4
    for (int p = gi + J * NG; p < parts; p += NG)
        O += __builtin_amdgcn_exp2f(a.part_ml[slot_of(p)].x - mu) * load4(a.part_o + slot_of(p) * D + 4 * e);
    red[gi][e] = O;
    __syncthreads();
    if (gi > 0)
        return;
#pragma unroll
    for (int j = 1; j < NG; ++j)
        O += red[j][e];
    const int node = rr / a.G, head = g * a.G + rr - node * a.G;
    store4(static_cast<TX *>(a.out) + (int64_t)(rows.first + node) * a.ld_out + (int64_t)head * D + 4 * e,
           total == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / total);
}

// Tiles, and how the keys are shared out, from the sizes alone (what lies in device
// memory is not known here).
//   Streams (sequences of one tile) where work-groups of whole sequences would end
// unevenly, or be too few: contexts past 512, past 1024 with a tile for every
// CU, past 2048 with two.  us, streams and whole, a token of 250 .. 500 keys (40
// heads, 8 sequences) 23.1 and 18.5, of 750 .. 1500 46.3 and 49.2; 64 heads on 8, 4
// sequences of up to 700 11.5 and 13.1, 32 24.5 and 17.9, 128 72.6 and 61.2; chains of
// 13, 16 sequences of up to 700 35.6 and 43.3, 8 of 40 heads 29.2 and 24.9.
//   Eight waves a work-group for long ones: 60000 keys 57.7 -> 55.2 us, 64 sequences of
// 500 .. 8000 197 -> 193; 8 sequences of 750 .. 1500 (40 heads) 46.6 -> 48.7.
//   Packed tiles of 64 or 128 rows, us: 1023 rows of 40 heads (320 tiles) float32 51
// and 68, bfloat16 31.8 and 35.5; 1000 of 64 heads on 8 (504) 72 and 71, 43 and 35.
//   Over pages, where tiles of 128 rows are too many for shares (more than 256) and too few
// to fill the last round (at most 450): 15 chains of 26 rows, 64 heads on 8, 26.9 and 36.3,
// float32 39.6 and 56.9; five chunks of up to 358 rows of 32 heads 40.7 and 55.5, 58.8 and 76.4; 1000
// rows of 40 heads behind 2000 positions 126 and 96, 187 and 187; six of 100 rows, 64 heads
// on 8, behind up to 8000 264 and 258, 367 and 497: float32 always, bfloat16 where
// sequences are short, whose last tiles are a large part.
//   k_batch_attn_wide for bfloat16 queries, or k_batch_attn_mfma where blocks that a row sees
// in part, which the first takes without overlap, and the start are much of it: 39 chunks
// of up to 77 rows over up to 96 positions, 32 heads, 42.3 and 28.7; 20 of up to 128 over 428 52.3 and
// 42.9, over 728 96.3 and 93.7, over 1128 123 and 127; 10 of 100 of 64 heads on 8 over 700 55.8 and
// 61.6.  Prompts of 32 heads, 16 of 400 rows 94 and 79, 1200 343 and 315, one of 3001 108 and
// 105, of 8000 534 and 579; of 64 heads on 8, 8 of 400 61.6 and 60.3, 800 145 and 151.
//   Shares for two work-groups a CU (three, four): 200 rows of 64 heads on 8 behind 4000 positions
// 58 (64, 78) us, 1000 of 40 heads behind 2000 97 (121, 122), 13 of 64 heads on 8 behind 2000,
// float32, 46 (40, 40).
//   One wave a work-group for short ones, where more than four times as many then run
// at once (four waves and one): a token of 32 sequences (40 heads, float32) of up to 30
// keys 18.7 and 9.8 us, 100 22.4 and 16.9, 250 34.0 and 32.5, 500 55.3 and 55.0; 64
// sequences of 500 93 and 101; 256 (64 heads on 8, bfloat16) of 100 29.2 and 20.7, 500 77.9 and
// 79.8; 16 of 30 11.8 and 6.9, 8 of 100 9.6 and 11.7.  27 rows each of 14 sequences, 100 keys
// 30.7 and 23.7, 400 48.8 and 43.9; 2 to 4 rows of 64 heads on 8, 40 sequences of 100 (320
// work-groups) 19.0 and 21.9.
constexpr int FEW_ROWS = 32, CUS = 256, SHORT = 256, LONG = 2048, NARROW = 450;
void plan(BatchAttnArgs *a, bool x_bf16, bool bf16, int D) {
    const int64_t most = (int64_t)a->max_rows * a->G;
    const bool few = bf16 && a->paged && most <= FEW_ROWS;
    const auto slots_of = [&](int tile) {
        return most <= tile ? (int64_t)a->n_seqs : (int64_t)a->n * a->G / tile + a->n_seqs;
    };
    const int64_t tiles = slots_of(128) * a->n_kv_heads;
    const bool brief = !x_bf16 || (int64_t)a->n * a->G <= 512 * (int64_t)a->n_seqs;
    const bool narrow = most <= 64 || (tiles <= NARROW && (!a->paged || (tiles > CUS && brief)));
    a->tile = !bf16 ? 16 : few ? (most <= 16 ? 16 : 32) : narrow ? 64 : 128;
    a->one_tile = most <= a->tile;
    a->slots = (int32_t)slots_of(a->tile);
    const int64_t units = (int64_t)a->slots * a->n_kv_heads;
    a->splits = 1;
    a->chunks = 0;
    a->waves = NW;
    if (bf16 && a->paged && a->one_tile) {
        const int whole = 512 * (int)std::max<int64_t>(1, std::min<int64_t>(4, units / (CUS / 2)));
        const int waves = few && a->tile == 16 && a->max_length > LONG ? 8 : NW, span = few ? waves * KB_FEW : KB;
        const int64_t spans = (int64_t)a->n_seqs * ((a->max_length + span - 1) / span);
        // (the join has a work-group a row, and a launch at most 2^32 threads)
        const int64_t joins = units * std::min<int64_t>(most, a->tile);
        if (a->max_length > whole && a->n_seqs <= MAX_STREAM && spans <= 1 << 30 && joins <= 1 << 23) {
            // as many work-groups as run at once
            const int at_once = waves == 8 || (a->tile == 32 && D == 128) ? CUS : 2 * CUS;
            a->waves = waves;
            a->span = span;
            a->block = few ? KB_FEW : KB;
            a->chunks = (int32_t)std::min<int64_t>(spans, std::max(1, at_once / a->n_kv_heads));
            return;
        }
    }
    if (few && units > 2 * CUS && a->max_length <= (a->tile == 16 ? SHORT : 2 * SHORT))
        a->waves = 1;
    a->wide = x_bf16 && bf16 && a->tile == 128 &&
              (a->paged ? a->max_length > 512 : (int64_t)a->n * a->G > 4096 * (int64_t)a->n_seqs);
    a->block = few || a->wide ? KB_FEW : KB;
    const int blocks = (a->max_length + a->block - 1) / a->block;
    a->per_split = blocks;
    if (a->paged && !few) {
        // (shares of all n rows, also those of no sequence: at most 2^22 in all)
        const int64_t most_shares = std::min<int64_t>(2 * CUS / units, (1 << 22) / ((int64_t)a->n * a->n_heads));
        const int want = (int)std::max<int64_t>(1, std::min<int64_t>((blocks + 7) / 8, most_shares));
        a->per_split = (blocks + want - 1) / want;
        a->splits = (blocks + a->per_split - 1) / a->per_split;
    }
}

// What the workspace holds: outputs and states of the parts, and the spans.
struct Space {
    size_t o, ml, spans;
    size_t bytes() const { return o + ml + spans; }
};
Space space_of(const BatchAttnArgs &a, int D) {
    const size_t rows = a.chunks       ? (size_t)2 * a.n_kv_heads * a.chunks * a.tile
                        : a.splits > 1 ? (size_t)a.splits * a.n * a.n_heads
                                       : 0;
    return {rows * D * sizeof(float), rows * sizeof(float2), a.chunks ? sizeof(int32_t) * ((size_t)a.n_seqs + 2) : 0};
}

template <typename TX>
void launch_f32(const BatchAttnArgs &a, int D, hipStream_t s) {
    const dim3 grid((unsigned)(a.slots * a.n_kv_heads), (unsigned)a.splits), block(NW * 64);
    if (D == 16)
        hipLaunchKernelGGL((k_batch_attn_f32<TX, 16>), grid, block, 0, s, a);
    else if (D == 32)
        hipLaunchKernelGGL((k_batch_attn_f32<TX, 32>), grid, block, 0, s, a);
    else if (D == 64)
        hipLaunchKernelGGL((k_batch_attn_f32<TX, 64>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_batch_attn_f32<TX, 128>), grid, block, 0, s, a);
}

template <typename TX, int D>
void launch_mfma(const BatchAttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.chunks ? a.chunks * a.n_kv_heads : a.slots * a.n_kv_heads * a.splits)), block(256);
    if (a.tile == 16) {
        if (a.waves == 8)
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 1, 8, true>), grid, dim3(512), 0, s, a);
        else if (a.chunks)
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 1, NW, true>), grid, block, 0, s, a);
        else if (a.waves == 1)
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 1, 1, false>), grid, dim3(64), 0, s, a);
        else
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 1, NW, false>), grid, block, 0, s, a);
    } else if (a.tile == 32) {
        if (a.chunks)
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 2, NW, true>), grid, block, 0, s, a);
        else if (a.waves == 1)
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 2, 1, false>), grid, dim3(64), 0, s, a);
        else
            hipLaunchKernelGGL((k_batch_attn_few<TX, D, 2, NW, false>), grid, block, 0, s, a);
    } else if (a.tile == 64) {
        if (a.chunks)
            hipLaunchKernelGGL((k_batch_attn_mfma<TX, D, 2, 2, STREAM>), grid, block, 0, s, a);
        else if (a.paged)
            hipLaunchKernelGGL((k_batch_attn_mfma<TX, D, 2, 2, PAGES>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((k_batch_attn_mfma<TX, D, 2, 2, PACKED>), grid, block, 0, s, a);
    } else if (a.chunks) {
        hipLaunchKernelGGL((k_batch_attn_mfma<TX, D, 4, 1, STREAM>), grid, block, 0, s, a);
    } else if (a.wide) {
        if (a.paged)
            hipLaunchKernelGGL((k_batch_attn_wide<D, true>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((k_batch_attn_wide<D, false>), grid, block, 0, s, a);
    } else {
        if (a.paged)
            hipLaunchKernelGGL((k_batch_attn_mfma<TX, D, 4, 1, PAGES>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((k_batch_attn_mfma<TX, D, 4, 1, PACKED>), grid, block, 0, s, a);
    }
}
template <typename TX>
void launch_bf16(const BatchAttnArgs &a, int D, hipStream_t s) {
    if (D == 16)
        launch_mfma<TX, 16>(a, s);
    else if (D == 32)
        launch_mfma<TX, 32>(a, s);
    else if (D == 64)
        launch_mfma<TX, 64>(a, s);
    else
        launch_mfma<TX, 128>(a, s);
}

template <typename TX, int D>
void launch_join_stream(const BatchAttnArgs &a, hipStream_t s) {
    const int rows = std::min(a.max_rows * a.G, a.tile);
    const dim3 grid((unsigned)(a.n_seqs * a.n_kv_heads * rows));
    // (parts of a sequence: one or two of many, or all of one)
    if (a.chunks <= 8 * a.n_seqs)
        hipLaunchKernelGGL((k_batch_join_stream<TX, D, 64>), grid, dim3(64), 0, s, a, rows);
    else
        hipLaunchKernelGGL((k_batch_join_stream<TX, D, 256>), grid, dim3(256), 0, s, a, rows);
}

template <typename TX, int D>
void launch_join_shares(const BatchAttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.n * a.n_heads));
    if (a.splits <= 8)
        hipLaunchKernelGGL((k_batch_join<TX, D, 64>), grid, dim3(64), 0, s, a);
    else
        hipLaunchKernelGGL((k_batch_join<TX, D, 256>), grid, dim3(256), 0, s, a);
}

template <typename TX, int D>
void launch_join(const BatchAttnArgs &a, hipStream_t s) {
    if (a.chunks)
        launch_join_stream<TX, D>(a, s);
    else
        launch_join_shares<TX, D>(a, s);
}
template <typename TX>
void launch_join(const BatchAttnArgs &a, int D, hipStream_t s) {
    if (D == 16)
        launch_join<TX, 16>(a, s);
    else if (D == 32)
        launch_join<TX, 32>(a, s);
    else if (D == 64)
        launch_join<TX, 64>(a, s);
    else
        launch_join<TX, 128>(a, s);
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
            launch_bf16<uint16_t>(a, D, s);
        else
            launch_f32<uint16_t>(a, D, s);
    } else if (dtype == SD_BF16) {
        launch_bf16<float>(a, D, s);
    } else {
        launch_f32<float>(a, D, s);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && (a.splits > 1 || a.chunks)) {
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
    a->paged = 1;
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

// The plan of a call over pages, from its sizes alone.
sd_status paged_plan(const sd_kv_pages *kv, const sd_batch *batch, int32_t x_dtype, int32_t n_heads, int32_t n,
                     BatchAttnArgs *a) {
    sd_status st = paged_sizes(kv, batch, n_heads, n, false, a);
    if (st != SD_OK || (st = check_call(nullptr, 0, x_dtype, n_heads, n, a->n_seqs, a->n_kv_heads, kv->head_dim, nullptr, 0,
                                        nullptr)) != SD_OK)
        return st;
    plan(a, x_dtype == SD_BF16, kv->dtype == SD_BF16, kv->head_dim);
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
    plan(&a, x_dtype == SD_BF16, kv->dtype == SD_BF16, kv->head_dim);
    const Space space = space_of(a, kv->head_dim);
    const size_t need = space.bytes();
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
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + space.o);
        a.spans = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + space.o + space.ml);
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
    plan(&a, x_dtype == SD_BF16, kv->dtype == SD_BF16, kv->head_dim);
    return launch(a, x_dtype, kv->dtype, kv->head_dim, s);
}

}  // namespace

extern "C" {

size_t sd_paged_attention_workspace(const sd_kv_pages *kv, const sd_batch *batch, int32_t x_dtype, int32_t n_heads,
                                    int32_t n) try {
    BatchAttnArgs a{};
    return paged_plan(kv, batch, x_dtype, n_heads, n, &a) == SD_OK ? space_of(a, kv->head_dim).bytes() : 0;
} catch (...) {  // (a refusal's message is allocated)
    return 0;
}

sd_status sd_paged_attention(const sd_kv_pages *kv, const sd_batch *batch, const void *q, int64_t ld_q, int32_t x_dtype,
                             int32_t n_heads, int32_t n, float scale, void *out, int64_t ld_out, void *workspace,
                             size_t workspace_bytes, void *hip_stream) {
    SD_GUARD(return paged_attention(kv, batch, q, ld_q, x_dtype, n_heads, n, scale, out, ld_out, workspace,
                                    workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));)
}

// For the tests: how a call over pages is shared out: rows of a tile and how many tiles at
// most, chunks of the streams and keys of a span, shares of the keys, waves of a work-group, and whether
// k_batch_attn_wide takes it.
sd_status sdk_paged_plan(const sd_kv_pages *kv, const sd_batch *batch, int32_t x_dtype, int32_t n_heads, int32_t n,
                         int32_t out[7]) {
    SD_GUARD(BatchAttnArgs a{};
             const sd_status st = paged_plan(kv, batch, x_dtype, n_heads, n, &a);
             if (st != SD_OK) return st;
             const int32_t of[7] = {a.tile, a.slots, a.chunks, a.span, a.splits, a.waves, a.wide};
             std::copy(of, of + 7, out); return SD_OK;)
}

sd_status sd_prompt_attention(const sd_kv_layer *kv, const int32_t *starts, int32_t n_seqs, const void *q, int64_t ld_q,
                              int32_t x_dtype, int32_t n_heads, int32_t n, float scale, void *out, int64_t ld_out,
                              void *hip_stream) {
    SD_GUARD(return prompt_attention(kv, starts, n_seqs, q, ld_q, x_dtype, n_heads, n, scale, out, ld_out,
                                     reinterpret_cast<hipStream_t>(hip_stream));)
}

}  // extern "C"
