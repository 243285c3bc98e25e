// Attention of a tree's nodes over a cached prefix and their own ancestors.
//
// Row r of head h: o = sum_k p_k v_k / sum_k p_k, p_k = exp(scale q.k - max),
// over every prefix key and the nodes whose bit is set in row r of the mask.
// The query heads of a kv head and the nodes share its keys: the n G rows of a kv
// head (G query heads each, row = node G + head) are one matrix of queries.
//
// Keys come in blocks of 32 or 64: first the prefix, its last block cut off, then
// the nodes in blocks of their own, so that a block's visible keys are one word,
// or half a word, of the mask a row.  The blocks are split over work-groups,
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
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

constexpr int KB = 64;       // keys of a block
constexpr int KB_FEW = 32;   // of the kernel for few rows

struct TreeAttnArgs {
    const float *q;
    int64_t ld_q;
    const void *k, *v;
    int64_t head_stride, row_stride;
    const uint64_t *mask;  // [n][words], or null: row r sees nodes 0 .. row0 + r
    float *out;
    int64_t ld_out;
    float *part_o;    // [splits][n H][D] unnormalised outputs
    float2 *part_ml;  // [splits][n H]: (maximum, sum), in units of log2
    float scale;      // of the scores, times log2(e)
    int32_t row0, nodes;  // the n rows are nodes row0 .. of that many
    int32_t n, words, prefix, n_heads, n_kv_heads, G, rows, q_tiles;  // rows = n G
    int32_t q_rows;                                                   // of a tile
    int32_t prefix_blocks, blocks, splits, per_split;                 // per_split: blocks of a share
};

// Block b of B keys: its first key, how many keys it has, and whether they are nodes.
struct Block {
    int first, len, node0;  // node0: the first node, or -1
};
template <int B>
__device__ __forceinline__ Block block_of(const TreeAttnArgs &a, int b) {
    Block k;
    if (b < a.prefix_blocks) {
        k.first = B * b;
        k.len = min(B, a.prefix - k.first);
        k.node0 = -1;
    } else {
        k.node0 = B * (b - a.prefix_blocks);
        k.first = a.prefix + k.node0;
        k.len = min(B, a.nodes - k.node0);
    }
    return k;
}
// The keys of a block that a node sees, as bits.
__device__ __forceinline__ uint64_t visible(const TreeAttnArgs &a, const Block &k, int node) {
    const uint64_t all = k.len >= 64 ? ~0ull : (1ull << k.len) - 1;
    if (k.node0 < 0)
        return all;
    if (a.mask)
        return (a.mask[(int64_t)node * a.words + (k.node0 >> 6)] >> (k.node0 & 63)) & all;
    const int last = a.row0 + node - k.node0;
    return last < 0 ? 0 : (last >= 63 ? ~0ull : (2ull << last) - 1) & all;
}

__device__ __forceinline__ f32x4_t load4(const float *p) { return *reinterpret_cast<const f32x4_t *>(p); }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Two packed bfloat16 values, zero for those that are infinite or NaN.
__device__ __forceinline__ uint32_t without_odd(uint32_t x) {
    const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
    return x & (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
}

// The NW waves' states of ROWS rows from row0 on (o [wave][row][D + 4], waves
// `pitch` floats apart; (maximum, sum) [wave][row]) merged in wave order: the
// result of a single share, or its part of several.
template <int D, int NW, int ROWS>
__device__ __forceinline__ void merge_waves(const TreeAttnArgs &a, const float *o, int pitch, const float2 *ml, int row0,
                                            int g, int split) {
#pragma unroll
    for (int i = threadIdx.x; i < ROWS * D / 4; i += NW * 64) {
        const int rc = i / (D / 4), e = 4 * (i % (D / 4)), rr = row0 + rc;
        if (rr >= a.rows)
            break;  // i only grows
        float m = -INFINITY, L = 0.0f;
        f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < NW; ++w)
            m = fmaxf(m, ml[w * ROWS + rc].x);
        const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            // (a wave without keys has weight zero, output zero)
            const float wt = __builtin_amdgcn_exp2f(ml[w * ROWS + rc].x - mu);
            L = fmaf(wt, ml[w * ROWS + rc].y, L);
            O += wt * load4(o + w * pitch + rc * (D + 4) + e);
        }
        const int nd = rr / a.G, hd = g * a.G + rr - nd * a.G;
        if (a.splits == 1) {
            *reinterpret_cast<f32x4_t *>(a.out + (int64_t)nd * a.ld_out + (int64_t)hd * D + e) =
                L == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / L;
        } else {
            const int64_t slot = ((int64_t)split * a.n + nd) * a.n_heads + hd;
            *reinterpret_cast<f32x4_t *>(a.part_o + slot * D + e) = O;
            if (e == 0)
                a.part_ml[slot] = make_float2(m, L);
        }
    }
}

// ---------------------------------------------------------------------------
// In float32: a work-group of four waves takes 16 rows of a kv head, each wave
// 16 keys of every block of its share.  Scores S^T[key][row] = K q are
// 16x16x4 float32 matrix products: lane (c = lane % 16, g = lane / 16) gives
// elements 16 j + 4 g + u of key c and of row c in step (j, u), so both come by
// 16-byte loads straight from memory, and receives the keys 4 g + v, v = 0..3,
// of row c.  The value products O^T[e][row] += V^T P^T take the reduction slots
// (step v, slot g) as key 4 g + v, so weights stay in their lanes; tile t's row i is
// element 64 (t / 4) + 4 i + t % 4, so 16 bytes of row 4 g + v are a lane's operands
// of four tiles.  V is asked for before the scores and the next block's K after
// them.  The waves keep states of their own and merge at the end.
//
// Bound by the read of the cache, 4 rows over 4000 keys, 40 heads of 128: 32.3 us
// with the join, 5.1 TB/s (43 with V by single elements and no load ahead); by the
// chain of loads, products and softmax of a block where there are few, 5 rows over
// 30 keys, 4 heads of 64: 4.5 us; for more rows by every tile's own read of the
// context and that chain, 64 rows over 4000 keys, 40 heads: 105 us.
constexpr int TA_WAVES = 4;

template <int D>
__global__ __launch_bounds__(TA_WAVES * 64, 2) void k_tree_attn_f32(TreeAttnArgs a) {
    constexpr int ES = D / 16, OP = D + 4, W = ES < 4 ? ES : 4;  // W: elements of a load of V
    typedef float vec_t __attribute__((ext_vector_type(W)));
    __shared__ __attribute__((aligned(16))) float tile[TA_WAVES][16 * OP];
    __shared__ float2 ml[TA_WAVES][16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g4 = lane >> 4;
    const int qt = blockIdx.x % a.q_tiles, g = blockIdx.x / a.q_tiles, split = blockIdx.y;
    const int b0 = split * a.per_split, b1 = min(a.blocks, b0 + a.per_split);
    const float *K = static_cast<const float *>(a.k) + (int64_t)g * a.head_stride;
    const float *V = static_cast<const float *>(a.v) + (int64_t)g * a.head_stride;
    const int row = min(qt * 16 + c, a.rows - 1), node = row / a.G, head = g * a.G + row - node * a.G;

    f32x4_t qx[ES];
#pragma unroll
    for (int j = 0; j < ES; ++j)
        qx[j] = load4(a.q + (int64_t)node * a.ld_q + (int64_t)head * D + 16 * j + 4 * g4) * a.scale;
    // o[t][u]: this element of row c
    auto element = [&](int t, int u) { return 16 * W * (t / W) + W * (4 * g4 + u) + t % W; };
    float m_run = -INFINITY, l_run = 0.0f;
    f32x4_t o[ES];
#pragma unroll
    for (int t = 0; t < ES; ++t)
        o[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    // keys past a block read its last one; their scores are masked
    f32x4_t kx[ES];
    auto load_k = [&](const Block &k) {
        const float *kp = K + (int64_t)(k.first + min(16 * wave + c, k.len - 1)) * a.row_stride + 4 * g4;
#pragma unroll
        for (int j = 0; j < ES; ++j)
            kx[j] = load4(kp + 16 * j);
    };
    if (b0 < b1)
        load_k(block_of<KB>(a, b0));
    for (int b = b0; b < b1; ++b) {
        const Block k = block_of<KB>(a, b);
        const bool some = 16 * wave < k.len;  // uniform over the wave
        f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
        vec_t vx[4][ES / W];
        if (some) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float *vp = V + (int64_t)(k.first + min(16 * wave + 4 * g4 + v, k.len - 1)) * a.row_stride + W * c;
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
        if (b + 1 < b1)
            load_k(block_of<KB>(a, b + 1));
        if (!some)
            continue;
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
#pragma unroll
        for (int t = 0; t < ES; ++t)
            o[t] *= sc;
        bool odd = false;
        if (k.node0 >= 0) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int t = 0; t < ES; ++t)
                    odd |= !finite(vx[v][t / W][t % W]);
        }
        if (__any(odd)) {
            // An infinity or NaN among the nodes' values: a row that does not
            // see it must not add 0 times it.  They are taken out of the
            // operands, and added here, from memory, where they belong.
            for (int key = 0; key < 16; ++key) {
                const float *vr = V + (int64_t)(k.first + min(16 * wave + key, k.len - 1)) * a.row_stride;
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
    merge_waves<D, TA_WAVES, 16>(a, &tile[0][0], 16 * OP, &ml[0][0], qt * 16, g, split);
}

// ---------------------------------------------------------------------------
// bfloat16 caches: matrix cores.  q (times scale log2(e)) and the weights are
// float32; each is held as three bfloat16 terms that add up to it exactly, so that
// only the float32 sums round.  That issues three times the flops: 1.5 matrix
// cycles a score and SIMD, next to about as many for its softmax and terms.
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
//
// Heads of 128, with their join: 64 rows of 8 over 16000 keys, 8 kv heads (tiles
// of 128) 90 + 8 us, 1.1 PFLOP/s issued; 9 rows of 8 over 60000 keys, 8 kv heads
// 79 + 6 us (74 to 85 over runs), 3.1 TB/s (the read alone takes 50, and power holds
// the clock at 1.7 GHz); 61 rows over 3001 keys, 32 heads (64) 21 + 4 us.

// A maximum that grows by no more than this (in log2) does not rescale the sums:
// weights then reach 2^8 and not 1, which float32 sums do not mind.  A row decides
// by its own scores, so that its bits do not follow from what other rows of its
// wave see; the wave passes over the rescale where no row asks for it.
constexpr float SLACK = 8.0f;

__device__ __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}
__device__ __forceinline__ uint32_t cvt_pk(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
// The three terms of two values, packed.
__device__ __forceinline__ void terms2(float a, float b, uint32_t (&t)[X_TERMS]) {
    t[0] = cvt_pk(a, b);
    const float a1 = a - __uint_as_float(t[0] << 16), b1 = b - __uint_as_float(t[0] & 0xffff0000u);
    t[1] = cvt_pk(a1, b1);
    t[2] = cvt_pk(a1 - __uint_as_float(t[1] << 16), b1 - __uint_as_float(t[1] & 0xffff0000u));
}

// The terms of eight values as MFMA operands.
__device__ __forceinline__ void query_terms(f32x4_t x0, f32x4_t x1, u32x4_t (&q)[X_TERMS]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint32_t t0[X_TERMS], t1[X_TERMS];
        terms2(x0[2 * j], x0[2 * j + 1], t0);
        terms2(x1[2 * j], x1[2 * j + 1], t1);
#pragma unroll
        for (int i = 0; i < X_TERMS; ++i) {
            q[i][j] = t0[i];
            q[i][2 + j] = t1[i];
        }
    }
}

// Sixteen bytes per lane from g to LDS at l + 16 lane (l the same in every lane).
// The compiler does not see these loads; the kernel waits for them itself.  They
// have no register result; M0 holds the LDS address and needs one wait state.
__device__ __forceinline__ void load_to_lds16(const uint16_t *g, uint16_t *l) {
    const uint32_t off = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)l;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(
                     __builtin_amdgcn_readfirstlane(off)),
                 "v"(g)
                 : "memory", "m0");
}

// The same from base (the same in every lane) + off bytes.
__device__ __forceinline__ void load_to_lds16(const uint16_t *base, uint32_t off, uint16_t *l) {
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)l;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(
                     __builtin_amdgcn_readfirstlane(to)),
                 "v"(off), "s"(base)
                 : "memory", "m0");
}
// Whether a block's offsets in bytes fit 32 bits.
__device__ __forceinline__ bool near_rows(int64_t row_stride) { return row_stride < (int64_t)1 << 24; }

template <int D>
struct Lines {  // where a block's rows lie in LDS
    static constexpr int C = D / 8, RPL = 16 / C;  // chunks of a row, rows of a line
    __device__ static int swz(int s) {
        return C == 16 ? ((s & 3) << 2) | ((s >> 2) & 3) : C == 8 ? ((s & 1) << 2) | ((s >> 1) & 3) : s & (RPL == 4 ? 3 : 1);
    }
    // element offset of chunk c of row r
    __device__ static int at(int r, int c) {
        const int s = r / RPL;
        return s * 128 + 8 * (((r % RPL) * C + c) ^ swz(s));
    }
};

template <int D, int NQ, int NK>
__global__ __launch_bounds__(64 * NQ * NK, 2) void k_tree_attn_mfma(TreeAttnArgs a) {
    constexpr int T = X_TERMS, NW = NQ * NK, ES = D / 16, ET = D < 32 ? 1 : D / 32;
    constexpr int LOADS = 2 * (D / 8);  // 1 KB loads of a block's K and V
    using L = Lines<D>;
    __shared__ __attribute__((aligned(1024))) uint16_t kv[2][2][KB * D];  // [block % 2][K, V]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31,
              half = lane >> 5;
    const int wq = wave % NQ, wk = wave / NQ;
    const int g = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int qt = rest % a.q_tiles, split = rest / a.q_tiles;
    const int b0 = split * a.per_split, b1 = min(a.blocks, b0 + a.per_split);
    const int r0 = (qt * NQ + wq) * 32;
    const bool live = r0 < a.rows;  // uniform over the wave: a wave without rows loads and waits with the others
    const int row = min(r0 + col, a.rows - 1), node = row / a.G, head = g * a.G + row - node * a.G;
    const uint16_t *K = static_cast<const uint16_t *>(a.k) + (int64_t)g * a.head_stride;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + (int64_t)g * a.head_stride;

    // A wave takes every NW-th KB of K's and of V's rows.  Whole blocks: lane
    // offsets that do not change, from the block's first row (with the addresses
    // taken load by load, issuing them was a quarter of a block's time).
    constexpr int NU = (L::C + NW - 1) / NW;
    uint32_t off[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const int s = 4 * (wave + NW * i) + (lane >> 4), p = (lane & 15) ^ L::swz(s);
        off[i] = (uint32_t)(2 * ((int64_t)(s * L::RPL + p / L::C) * a.row_stride + 8 * (p % L::C)));
    }
    const bool near = near_rows(a.row_stride);
    auto load_block = [&](int b, int buf) {
        const Block k = block_of<KB>(a, b);
        if (k.len == KB && near) {
            const int64_t first = (int64_t)k.first * a.row_stride;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int i = 0; i < NU; ++i)
                    if (L::C % NW == 0 || wave + NW * i < L::C)  // uniform over the wave
                        load_to_lds16((m ? V : K) + first, off[i], &kv[buf][m][(wave + NW * i) * 512]);
        } else {
#pragma unroll 1
            for (int t = wave; t < LOADS; t += NW) {
                const int m = t / L::C, u = t % L::C;  // matrix, and 1 KB of it
                const int s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
                const int r = min(s * L::RPL + p / L::C, k.len - 1);  // rows past the block: its last
                load_to_lds16((m ? V : K) + (int64_t)(k.first + r) * a.row_stride + 8 * (p % L::C), &kv[buf][m][u * 512]);
            }
        }
    };
    // The queries are asked for before the first block: loads return in order
    // (100 rows over 2000 keys, 40 heads: 27.2 -> 26.4 us).
    f32x4_t qx[ES][2];
    {
        const float *qs = a.q + (int64_t)node * a.ld_q + (int64_t)head * D + 8 * half;
#pragma unroll
        for (int s = 0; s < ES; ++s) {
            qx[s][0] = load4(qs + 16 * s);
            qx[s][1] = load4(qs + 16 * s + 4);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    load_block(b0, 0);
    // Rows past the last are zeros, which draw less power than copies of it (9 rows
    // of 8 over 60000 keys: 80.3 -> 79.8 us with the join).
    const float scale = r0 + col < a.rows ? a.scale : 0.0f;
    u32x4_t qf[ES][T];
#pragma unroll
    for (int s = 0; s < ES; ++s)
        query_terms(qx[s][0] * scale, qx[s][1] * scale, qf[s]);
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
        const Block k = block_of<KB>(a, b);
        // this wave's loads of the block have landed, then everyone's; every
        // read of the other buffer has returned
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (b + 1 < b1)
            load_block(b + 1, buf ^ 1);
        uint16_t *vs = kv[buf][1];
        bool odd = false;
        if (k.node0 >= 0) {
            // A row must not add 0 times an infinity or NaN of a node that it
            // does not see: they are taken out of the nodes' values, and put
            // where they belong beside the products.
            for (int c = threadIdx.x; c < KB * D / 8; c += 64 * NW) {
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
        const bool full = k.node0 < 0 && k.len == KB;  // every row sees every key
        const uint64_t see = full ? ~0ull : visible(a, k, node);
#pragma unroll 1
        for (int h = wk; h < 2; h += NK) {
            const uint32_t bits = h ? (uint32_t)(see >> 32) : (uint32_t)see;
            if (!live || (!full && !__any(bits != 0)))
                continue;  // uniform over the wave: no row of it sees these keys
            f32x16_t s;
#pragma unroll
            for (int v = 0; v < 16; ++v)
                s[v] = 0.0f;
            // byte addresses in LDS: rows 32 h + col, chunk 2 e + half at xk ^ 32 e.
            // (Hidden from the compiler, which would keep every address of the
            // loop in a register and spill.)
            int xk = 2 * (buf * 2 * KB * D + 32 * h * D + L::at(col, half)), xv = 2 * (buf * 2 * KB * D + 32 * h * D) + v_lane;
            asm volatile("" : "+v"(xk), "+v"(xv));
            // (the wave in its products before the one in its softmax: 4% less time
            // where the products bound it)
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
                uint32_t mine = bits >> (4 * half);
                asm volatile("" : "+v"(mine));  // (a branch, and not selects in every block)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    s[v] = (mine >> (8 * (v >> 2) + (v & 3))) & 1 ? s[v] : -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int v = 1; v < 16; ++v)
                mx = fmaxf(mx, s[v]);
            {
                const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                mx = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
            }
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
                p[v] = __builtin_amdgcn_exp2f(s[v] - m_use);
                sum += p[v];
            }
            l_run += sum;
            if (odd) {
                // what was taken out, from memory: lane (col, half) holds
                // elements 32 et + 8 (v / 4) + 4 half + v % 4 of row col
#pragma unroll 1
                for (int key = 0; key < 32; ++key) {
                    float pk = 0.0f;
                    const int mine = 4 * (key >> 3) + (key & 3);
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        pk = v == mine ? p[v] : pk;
                    pk = __shfl(pk, col + 32 * ((key >> 2) & 1), 64);
                    const uint16_t *vr = V + (int64_t)(k.first + min(32 * h + key, k.len - 1)) * a.row_stride;
#pragma unroll
                    for (int et = 0; et < ET; ++et)
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const int e = 32 * et + 8 * (v >> 2) + 4 * half + (v & 3);
                            const float x = e < D ? __uint_as_float((uint32_t)vr[e] << 16) : 0.0f;
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
                    uint32_t t[T];
                    terms2(p[8 * j + 2 * u], p[8 * j + 2 * u + 1], t);
#pragma unroll
                    for (int i = 0; i < T; ++i)
                        pf[i][u] = t[i];
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
        if (wk == 1)
            return;
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
    if (r0 + col >= a.rows)
        return;
    const int64_t slot = ((int64_t)split * a.n + node) * a.n_heads + head;
    float *to = a.splits == 1 ? a.out + (int64_t)node * a.ld_out + (int64_t)head * D : a.part_o + slot * D;
    const float inv = a.splits > 1 ? 1.0f : l_run == 0.0f ? 0.0f : 1.0f / l_run;
#pragma unroll
    for (int et = 0; et < ET; ++et)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = 32 * et + 8 * q + 4 * half;
            if (e < D)
                *reinterpret_cast<f32x4_t *>(to + e) =
                    f32x4_t{o[et][4 * q], o[et][4 * q + 1], o[et][4 * q + 2], o[et][4 * q + 3]} * inv;
        }
    if (a.splits > 1 && half == 0)
        a.part_ml[slot] = make_float2(m_run, l_run);
}

// ---------------------------------------------------------------------------
// The same for up to 32 rows of a kv head, where the read of the cache counts and
// not the products: four waves, each with 32-key blocks of its own and no barrier
// until the end.  K goes straight into registers as the A operand of 16x16x32
// score products, V straight into the wave's LDS, both one block ahead.  Lane
// (col, grp) receives the keys 16 t + 4 grp + v of row col, which are the slots
// u = 4 t + v that the value products take from it.  LDS lines are permuted for
// the reads here: eight rows, two adjacent chunks each.  13 rows over 1200 keys, 40
// heads of 128: 10.6 us (2.4 TB/s) and the join's 3.9, most of which is a
// launch's; one row over 60000 keys, 8 heads: 43 us, 5.7 TB/s.
__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}

// Rows r .. of a wave's V block in LDS.
template <int D>
struct FewLines {
    static constexpr int C = D / 8, RPL = 16 / C;
    __device__ static int swz(int s) {
        return C == 16 ? ((s & 3) << 2) | ((s >> 1) & 2) : C == 8 ? (s & 3) << 1 : C == 4 ? (s & 1) << 1 : 0;
    }
    __device__ static int at(int r, int c) {
        const int s = r / RPL;
        return s * 128 + 8 * (((r % RPL) * C + c) ^ swz(s));
    }
};

template <int D, int QT>
__global__ __launch_bounds__(256, QT == 1 || D < 128 ? 2 : 1) void k_tree_attn_few(TreeAttnArgs a) {
    constexpr int T = X_TERMS, NW = 4, ES = D < 32 ? 1 : D / 32, ET = D / 16, ROWS = 16 * QT, OP = D + 4;
    using L = FewLines<D>;
    constexpr int VB = KB_FEW * D;  // elements of a V block
    constexpr int WORDS = VB > ROWS * OP ? VB : ROWS * OP;
    __shared__ __attribute__((aligned(1024))) uint32_t tile[NW][WORDS];  // two V blocks, or the outputs
    __shared__ float2 ml[NW][ROWS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15,
              grp = lane >> 4;
    const int g = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int r0 = rest % a.q_tiles * ROWS, split = rest / a.q_tiles;
    const int b1 = min(a.blocks, (split + 1) * a.per_split);
    const uint16_t *K = static_cast<const uint16_t *>(a.k) + (int64_t)g * a.head_stride;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + (int64_t)g * a.head_stride;
    uint16_t *vt = reinterpret_cast<uint16_t *>(tile[wave]);

    // Whole blocks: lane offsets that do not change, from the block's first row.
    // (Of V's loads u, only the lane's place in odd and even ones differs.)
    const bool near = near_rows(a.row_stride);
    const uint32_t koff = (uint32_t)(2 * ((int64_t)col * a.row_stride + (8 * grp) % D));
    uint32_t voff[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
        voff[u] = (uint32_t)(2 * ((int64_t)((lane >> 4) * L::RPL + p / L::C) * a.row_stride + 8 * (p % L::C)));
    }
    u32x4_t kf[2][ES];
    auto load_k = [&](const Block &k) {
        const bool whole = k.len == KB_FEW && near;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            // keys past the block: its last, masked; head_dim 16: the upper slots are zeros of q
            const char *kp = whole ? reinterpret_cast<const char *>(K + (int64_t)(k.first + 16 * t) * a.row_stride) + koff
                                   : reinterpret_cast<const char *>(
                                         K + (int64_t)(k.first + min(16 * t + col, k.len - 1)) * a.row_stride + (8 * grp) % D);
#pragma unroll
            for (int s = 0; s < ES; ++s)
                kf[t][s] = *reinterpret_cast<const u32x4_t *>(kp + 64 * s);
        }
    };
    auto load_v = [&](const Block &k, int buf) {
        if (k.len == KB_FEW && near) {
#pragma unroll
            for (int u = 0; u < VB / 512; ++u)
                load_to_lds16(V + (int64_t)(k.first + 4 * u * L::RPL) * a.row_stride, voff[u & 1], vt + buf * VB + u * 512);
        } else {
#pragma unroll 1
            for (int u = 0; u < VB / 512; ++u) {
                const int s = 4 * u + (lane >> 4), p = (lane & 15) ^ L::swz(s);
                const int r = min(s * L::RPL + p / L::C, k.len - 1);
                load_to_lds16(V + (int64_t)(k.first + r) * a.row_stride + 8 * (p % L::C), vt + buf * VB + u * 512);
            }
        }
    };
    int b = split * a.per_split + wave;
    if (b < b1) {
        const Block k = block_of<KB_FEW>(a, b);
        load_k(k);
        load_v(k, 0);
    }
    int node[QT];
    u32x4_t qf[QT][ES][T];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int row = min(r0 + 16 * i + col, a.rows - 1);
        node[i] = row / a.G;
        const float *qs = a.q + (int64_t)node[i] * a.ld_q + (int64_t)(g * a.G + row - node[i] * a.G) * D + (8 * grp) % D;
#pragma unroll
        for (int s = 0; s < ES; ++s) {
            f32x4_t x0 = load4(qs + 32 * s) * a.scale, x1 = load4(qs + 32 * s + 4) * a.scale;
            if (D < 32 && grp >= 2)  // head_dim 16: the upper half of the reduction
                x0 = x1 = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            query_terms(x0, x1, qf[i][s]);
        }
    }
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
    for (; b < b1; b += NW, buf ^= 1) {
        const Block k = block_of<KB_FEW>(a, b);
        f32x4_t s[QT][2];
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int e = 0; e < ES; ++e)
#pragma unroll
                    for (int w = 0; w < T; ++w)
                        s[i][t] = mfma16(kf[t][e], qf[i][e][w], s[i][t]);
            }
        // this block's V has landed (it was asked for before this block's K, or
        // just after), then the next block's loads
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (b + NW < b1) {
            const Block next = block_of<KB_FEW>(a, b + NW);
            load_v(next, buf ^ 1);
            load_k(next);
        }
        // Infinities and NaN among the nodes' values: a row must not add 0 times
        // one that it does not see.  They are taken out here, and put where they
        // belong beside the products.
        bool odd = false;
        if (k.node0 >= 0) {
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
            if (k.node0 >= 0 || k.len < KB_FEW) {
                uint32_t mine = (uint32_t)visible(a, k, node[i]) >> (4 * grp);
                asm volatile("" : "+v"(mine));  // (a branch, and not selects in every block)
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    p[u] = (mine >> (16 * (u >> 2) + (u & 3))) & 1 ? p[u] : -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                mx = fmaxf(mx, p[u]);
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
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
                p[u] = __builtin_amdgcn_exp2f(p[u] - m_use);
                sum += p[u];
            }
            l_run[i] += sum;
            if (odd) {
                // lane (col, grp) holds elements 16 et + 4 grp + u of row col
#pragma unroll 1
                for (int key = 0; key < KB_FEW; ++key) {
                    float pk = 0.0f;
                    const int mine = 4 * (key >> 4) + (key & 3);
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        pk = u == mine ? p[u] : pk;
                    pk = __shfl(pk, col + 16 * ((key >> 2) & 3), 64);
                    const uint16_t *vr = V + (int64_t)(k.first + min(key, k.len - 1)) * a.row_stride + 4 * grp;
#pragma unroll
                    for (int et = 0; et < ET; ++et) {
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const float x = __uint_as_float((uint32_t)vr[16 * et + u] << 16);
                            if (pk != 0.0f && !finite(x))
                                o[i][et][u] = fmaf(pk, x, o[i][et][u]);
                        }
                        __builtin_amdgcn_sched_barrier(0);  // a few loads at a time: registers
                    }
                }
            }
            u32x4_t pf[T];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t t[T];
                terms2(p[2 * j], p[2 * j + 1], t);
#pragma unroll
                for (int w = 0; w < T; ++w)
                    pf[w][j] = t[w];
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
                for (int w = 0; w < T; ++w)
                    o[i][et] = mfma16(vf, pf[w], o[i][et]);
            }
        }
        // (every read of this block has returned before its buffer is filled again)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    // the waves' states, merged in wave order
    float *to = reinterpret_cast<float *>(tile[wave]);
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        l_run[i] += __shfl_xor(l_run[i], 16, 64);
        l_run[i] += __shfl_xor(l_run[i], 32, 64);
#pragma unroll
        for (int et = 0; et < ET; ++et)
            *reinterpret_cast<f32x4_t *>(to + (16 * i + col) * OP + 16 * et + 4 * grp) = o[i][et];
        if (grp == 0)
            ml[wave][16 * i + col] = make_float2(m_run[i], l_run[i]);
    }
    __syncthreads();
    merge_waves<D, NW, ROWS>(a, reinterpret_cast<const float *>(tile), WORDS, &ml[0][0], r0, g, split);
}

// The shares of a (node, head) joined: a work-group each.  Every wave takes the
// shares' maxima and sums by itself; D / 4 lanes hold a row, the groups of lanes
// take the shares in turn and add up in order.  The first J shares of a group
// and the first 64 maxima are asked for at once.  (One thread per element walking
// over the shares: 6.7 us for 520 rows of 10 shares, 33 us for 576 of 63.)
constexpr int JOIN_THREADS = 256;
template <int D, int J>
__global__ __launch_bounds__(JOIN_THREADS) void k_tree_join(TreeAttnArgs a) {
    constexpr int LANES = D / 4, NG = JOIN_THREADS / LANES;
    __shared__ f32x4_t red[NG][LANES];
    const int64_t slots = (int64_t)a.n * a.n_heads, slot = blockIdx.x;
    const int lane = threadIdx.x & 63, e = threadIdx.x % LANES, gi = threadIdx.x / LANES;
    const float *po = a.part_o + slot * D + 4 * e;
    const float2 *pm = a.part_ml + slot;
    f32x4_t x[J];
#pragma unroll
    for (int j = 0; j < J; ++j)
        x[j] = load4(po + min(gi + j * NG, a.splits - 1) * slots * D);
    const float2 first = pm[min(lane, a.splits - 1) * slots];
    float m = first.x;
    for (int s = lane + 64; s < a.splits; s += 64)
        m = fmaxf(m, pm[s * slots].x);
    m = wave_max_all(m);
    const float mu = m == -INFINITY ? 0.0f : m;
    const float w0 = __builtin_amdgcn_exp2f(first.x - mu);  // of share `lane`
    float sum = lane < a.splits ? w0 * first.y : 0.0f;
    for (int s = lane + 64; s < a.splits; s += 64) {
        const float2 v = pm[s * slots];
        sum = fmaf(__builtin_amdgcn_exp2f(v.x - mu), v.y, sum);
    }
    const float total = wave_sum_all(sum);
    f32x4_t O = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int s = gi + j * NG;
        const float w = s < 64 ? __shfl(w0, s & 63, 64) : __builtin_amdgcn_exp2f(pm[min(s, a.splits - 1) * slots].x - mu);
        if (s < a.splits)
            O += w * x[j];
    }
#pragma unroll 4
    for (int s = gi + J * NG; s < a.splits; s += NG)
        O += __builtin_amdgcn_exp2f(pm[s * slots].x - mu) * load4(po + s * slots * D);
    red[gi][e] = O;
    __syncthreads();
    if (gi > 0)
        return;
#pragma unroll
    for (int i = 1; i < NG; ++i)
        O += red[i][e];
    const int nd = (int)(slot / a.n_heads), hd = (int)(slot - (int64_t)nd * a.n_heads);
    *reinterpret_cast<f32x4_t *>(a.out + (int64_t)nd * a.ld_out + (int64_t)hd * D + 4 * e) =
        total == 0.0f ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : O / total;
}

template <int D>
void launch_join(const TreeAttnArgs &a, hipStream_t s) {
    constexpr int NG = JOIN_THREADS / (D / 4);
    auto join = a.splits <= NG ? k_tree_join<D, 1> : a.splits <= 2 * NG ? k_tree_join<D, 2> : k_tree_join<D, 4>;
    hipLaunchKernelGGL(join, dim3((unsigned)(a.n * a.n_heads)), dim3(JOIN_THREADS), 0, s, a);
}

// Rows of a tile and shares of the keys.
//   float32: tiles of 16 rows, shares by their cost (f32_shares).
//   bfloat16, up to 32 rows of a kv head: the kernel for few, at most one work-group
//   per CU, four blocks (one a wave) a share at least (13 rows over 1200 keys, 40
//   heads: 10.3 us, 11.3 with two per CU, which halves the keys of a share; one
//   row over 60000 keys, 8 heads: 43 and 46; with a seventh share of 40 heads, 280
//   work-groups, 9 rows over 2500 take 17.7 in place of 15.7).
//   More rows: tiles of 64, or of 128 above that (for 72 rows a tile of three waves
//   took 82.4 us where four, one of which only loads, take 80.3), and one or two
//   work-groups per CU (mfma_shares).
// A single share needs no join, whose launch takes a caller 2.4 us: the few-row and
// float32 kernels keep short contexts whole.  us on the GPU, whole and split: 5 rows
// over 300 keys (40 heads) 8.9 and 8.6, over 500 11.6 and 8.8; 32 rows over 150 (8
// heads) 12.1 and 11.2, over 300 14.2 and 11.4; float32, 13 rows, 40 heads of 128 over
// 100 8.9 and 8.8, over 300 13.0 and 9.1; 4 of 64 over 300 8.5 and 7.0, over 1000
// 18.2 and 7.2; 8 of 16 over 700 9.4 and 7.9, over 1400 15.6 and 7.9.
constexpr int TA_CUS = 256, FEW_ROWS = 32;
constexpr int whole_blocks(int q_rows) { return q_rows == 16 ? 12 : 6; }  // few rows: blocks of 32 keys
constexpr int WHOLE_F32 = 6 * 64;  // float32: blocks of 64 times head_dim, which counts as 32 at least

// Shares of the tiles of more rows.  Two work-groups per CU hide a part of each
// other's softmax, about a seventh of a long share; every work-group costs its
// start and its end, about two blocks' time, and a join is about 1.7.  us, kernel
// and join, with one and two per CU: 61 rows over 3001 keys (32 heads, 6 and 3
// blocks a share) 24.2 and 27.5; 64 over 8000 (8 heads, 4 and 2) 19 and 24.8; 512
// over 16000 (8 heads, 32 and 16) 112 and 105.  Three per CU do not fit.
int mfma_shares(int units, int blocks) {
    int best = 1;
    double least = INFINITY;
    for (int groups = 0; groups <= 2 * TA_CUS; groups += TA_CUS) {
        const int shares = std::max(1, std::min(blocks, groups / units));
        const int per = (blocks + shares - 1) / shares, w = (units * shares + TA_CUS - 1) / TA_CUS;
        const double cost = w * (per * (w == 1 ? 7.0 / 6.0 : 1.0) + 2.0) + (shares > 1 ? 1.7 : 0.0);
        if (cost < least) {
            least = cost;
            best = shares;
        }
    }
    return best;
}

// Shares of float32 tiles, in us: a block takes 0.45 + 0.0115 D; another
// work-group on the busiest CU costs more than the first did, since every tile reads
// the whole share by itself; a join costs its start and the partial results.  us
// with the join, by shares: 160 tiles over 4000 keys (heads of 128) one 109-117,
// two 126, three 106, six 102; 136 113, 121, 93, 97; 280 over 4000 233, 205, 188,
// 179; 160 over 1000 31.4, 40.7, 34.7, 37.9; 240 over 4000 137, 154, 176, 151; 40
// over 4000, six 32.3, 13 37.4; heads of 16, 160 over 4000, one 50.7, three 28.0.
int f32_shares(int units, int blocks, int D) {
    const double block = 0.45 + 0.0115 * D;
    int best = 1;
    double least = INFINITY;
    for (int c : {1, TA_CUS / units, 2 * TA_CUS / units, (2 * TA_CUS + units - 1) / units}) {
        const int want = std::max(1, std::min(blocks, c)), per = (blocks + want - 1) / want;
        const int shares = (blocks + per - 1) / per;
        const int64_t groups = (int64_t)units * shares, w = (groups + TA_CUS - 1) / TA_CUS;
        const double cost = block * per * (1.0 + 1.2 * (double)(w - 1)) +
                            (shares > 1 ? 1.0 + 6.0 * (double)groups * D / (TA_CUS * 128) : 0.0);
        if (cost < least) {
            least = cost;
            best = shares;
        }
    }
    return best;
}

void plan(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t nodes, int32_t prefix, TreeAttnArgs *a) {
    const bool bf16 = kv->dtype == SD_BF16;
    a->n = n;
    a->nodes = nodes;
    a->row0 = nodes - n;
    a->words = (nodes + 63) / 64;
    a->prefix = prefix;
    a->n_heads = n_heads;
    a->n_kv_heads = kv->n_kv_heads;
    a->G = n_heads / kv->n_kv_heads;
    a->rows = n * a->G;
    const bool few = bf16 && a->rows <= FEW_ROWS;
    a->q_rows = few ? (a->rows <= 16 ? 16 : 32) : bf16 ? (a->rows <= 64 ? 64 : 128) : 16;
    a->q_tiles = (a->rows + a->q_rows - 1) / a->q_rows;
    const int kb = few ? KB_FEW : KB, step = few ? 4 : 1;
    a->prefix_blocks = (prefix + kb - 1) / kb;
    a->blocks = a->prefix_blocks + (nodes + kb - 1) / kb;
    const int units = a->q_tiles * a->n_kv_heads;
    int want;
    if (few ? a->blocks <= whole_blocks(a->q_rows)
            : !bf16 && (int64_t)a->blocks * std::max(32, kv->head_dim) <= WHOLE_F32)
        want = 1;
    else if (!bf16)
        want = f32_shares(units, a->blocks, kv->head_dim);
    else if (!few)
        want = mfma_shares(units, a->blocks);
    else
        want = std::max(1, std::min((a->blocks + step - 1) / step, TA_CUS / units));
    a->per_split = ((a->blocks + want - 1) / want + step - 1) / step * step;
    a->splits = (a->blocks + a->per_split - 1) / a->per_split;
}

size_t o_bytes(const TreeAttnArgs &a, int D) { return sizeof(float) * (size_t)a.splits * a.n * a.n_heads * D; }
size_t workspace_of(const TreeAttnArgs &a, int D) {
    return a.splits == 1 ? 0 : o_bytes(a, D) + sizeof(float2) * (size_t)a.splits * a.n * a.n_heads;
}

sd_status check_sizes(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t nodes, int32_t prefix) {
    const sd_status st = check_layer(kv);
    if (st != SD_OK)
        return st;
    if (n < 1 || nodes < n || nodes > SD_TREE_MAX || n_heads < 1 || n_heads > 4096 || n_heads % kv->n_kv_heads)
        return report(SD_ERR_INVALID_ARG, "a tree has 1 to " + std::to_string(SD_TREE_MAX) +
                                              " nodes; n_heads is a multiple of n_kv_heads, at most 4096");
    if (prefix < 0 || (int64_t)prefix + nodes > kv->capacity)
        return report(SD_ERR_CAPACITY, "a layer of capacity " + std::to_string(kv->capacity) + " does not hold " +
                                           std::to_string(nodes) + " nodes after " + std::to_string(prefix) +
                                           " positions");
    return SD_OK;
}

void launch_f32(const TreeAttnArgs &a, int D, hipStream_t s) {
    const dim3 grid((unsigned)(a.q_tiles * a.n_kv_heads), (unsigned)a.splits), block(TA_WAVES * 64);
    if (D == 16)
        hipLaunchKernelGGL(k_tree_attn_f32<16>, grid, block, 0, s, a);
    else if (D == 32)
        hipLaunchKernelGGL(k_tree_attn_f32<32>, grid, block, 0, s, a);
    else if (D == 64)
        hipLaunchKernelGGL(k_tree_attn_f32<64>, grid, block, 0, s, a);
    else
        hipLaunchKernelGGL(k_tree_attn_f32<128>, grid, block, 0, s, a);
}

template <int D>
void launch_mfma(const TreeAttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.q_tiles * a.n_kv_heads * a.splits));
    if (a.q_rows == 16)
        hipLaunchKernelGGL((k_tree_attn_few<D, 1>), grid, dim3(256), 0, s, a);
    else if (a.q_rows == 32)
        hipLaunchKernelGGL((k_tree_attn_few<D, 2>), grid, dim3(256), 0, s, a);
    else if (a.q_rows == 64)
        hipLaunchKernelGGL((k_tree_attn_mfma<D, 2, 2>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((k_tree_attn_mfma<D, 4, 1>), grid, dim3(256), 0, s, a);
}

}  // namespace

namespace sdk {

sd_status tree_attention(const sd_kv_layer *kv, const float *q, int64_t ld_q, int32_t n_heads, int32_t n,
                         int32_t nodes, int32_t prefix, const uint64_t *mask, float scale, float *out, int64_t ld_out,
                         void *workspace, size_t workspace_bytes, hipStream_t s) {
    const sd_status st = check_sizes(kv, n_heads, n, nodes, prefix);
    if (st != SD_OK)
        return st;
    const int D = kv->head_dim;
    auto aligned = [](const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; };
    if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(mask, 8))
        return report(SD_ERR_INVALID_ARG, "q and out must be set and 16-byte aligned, mask 8-byte aligned");
    if (ld_q % 4 || ld_out % 4 || ld_q < (int64_t)n_heads * D || ld_out < (int64_t)n_heads * D)
        return report(SD_ERR_INVALID_ARG, "ld_q and ld_out must hold a row and be multiples of 4");
    // (the scores are taken in units of log2)
    const float in_log2 = (scale == 0.0f ? 1.0f / std::sqrt((float)D) : scale) * 1.4426950408889634f;
    if (!std::isfinite(in_log2))
        return report(SD_ERR_INVALID_ARG, "scale, and scale log2(e), must be finite");
    TreeAttnArgs a{};
    plan(kv, n_heads, n, nodes, prefix, &a);
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
    if (need) {
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + o_bytes(a, D));
    }
    a.scale = in_log2;
    if (kv->dtype != SD_BF16)
        launch_f32(a, D, s);
    else if (D == 16)
        launch_mfma<16>(a, s);
    else if (D == 32)
        launch_mfma<32>(a, s);
    else if (D == 64)
        launch_mfma<64>(a, s);
    else
        launch_mfma<128>(a, s);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        if (D == 16)
            launch_join<16>(a, s);
        else if (D == 32)
            launch_join<32>(a, s);
        else if (D == 64)
            launch_join<64>(a, s);
        else
            launch_join<128>(a, s);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SD_OK : report(SD_ERR_DEVICE, std::string("tree attention: ") + hipGetErrorString(e));
}

size_t tree_attention_bytes(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t nodes, int32_t prefix) {
    if (check_sizes(kv, n_heads, n, nodes, prefix) != SD_OK)
        return 0;
    TreeAttnArgs a{};
    plan(kv, n_heads, n, nodes, prefix, &a);
    return workspace_of(a, kv->head_dim);
}

}  // namespace sdk

extern "C" {

size_t sd_tree_attention_workspace(const sd_kv_layer *kv, int32_t n_heads, int32_t n, int32_t prefix) {
    return tree_attention_bytes(kv, n_heads, n, n, prefix);
}

sd_status sd_tree_attention(const sd_kv_layer *kv, const float *q, int64_t ld_q, int32_t n_heads, int32_t n,
                            int32_t prefix, const uint64_t *mask, float scale, float *out, int64_t ld_out,
                            void *workspace, size_t workspace_bytes, void *hip_stream) {
    SD_GUARD(return tree_attention(kv, q, ld_q, n_heads, n, n, prefix, mask, scale, out, ld_out, workspace,
                                   workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));)
}

}  // extern "C"
