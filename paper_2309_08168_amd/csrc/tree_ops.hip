// Operators of token trees besides the attention: the layout of a tree, rotary
// embedding with the append to the cache, the greedy walk, and the move of the
// accepted path's cache rows.
//
// A verification (Algorithm 2) scores a chain; a tree holds several chains
// after one prefix.  Its nodes lie in the cache in their own order, while a
// node's position follows its depth, so rotary positions come apart from cache
// positions, and what is accepted is a path through the nodes instead of their
// first few.
#include "tree.h"

#include <algorithm>
#include <cmath>
#include <string>

#include "host_api.h"

using namespace sdk;

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

sd_status launched(const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SD_OK : report(SD_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

// ---------------------------------------------------------------------------
// Rotary embedding and append.  Reads 4 (H + 2 KVH) D bytes a row, writes 4 H D
// and the cache's 2 KVH D elements; three flops an element: bound by memory
// for many rows and by the launch for a few.
//
// A work-group of 256 threads takes a row, or a share of one where there are few
// rows.  Its first lanes take the row's angles (float64: at position 60000 a
// float32 angle is off by up to 0.002) into LDS, while the first
// loads are under way; a thread then handles units of eight elements: four pairs of a
// rotated head, or eight elements that pass.  1000 rows of 64 + 16 heads of 128
// into a bfloat16 cache: 12.4 us, 6.3 TB/s (from the last-level cache); 13 rows of
// 40 + 80: 3.2 us, most of it the kernel's start and the angles.

struct RopeArgs {
    // frequency of pair i: f = exp2(i * step), weighed for YARN, else times inv_factor
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

double scaled_base(const sd_rope &r) {
    return r.scaling == SD_ROPE_NTK ? r.base * std::pow(r.factor, (double)r.rotary_dim / (r.rotary_dim - 2)) : r.base;
}

// The rotary part of the arguments, for a checked form.
void rope_form(const sd_rope &r, RopeArgs *out) {
    out->step = -2.0 * std::log2(scaled_base(r)) / r.rotary_dim;
    out->yarn = r.scaling == SD_ROPE_YARN;
    out->inv_factor = r.scaling == SD_ROPE_LINEAR || out->yarn ? 1.0 / r.factor : 1.0;
    out->turns = r.original_context / 6.28318530717958647693;
    out->beta_slow = r.beta_slow;
    out->inv_beta = out->yarn ? 1.0 / (r.beta_fast - r.beta_slow) : 0.0;
    out->gain = (float)rope_gain(r);
    out->half = r.rotary_dim / 2;
    out->interleaved = r.layout == SD_ROPE_INTERLEAVED;
}

__device__ __forceinline__ float2 rope_turn(const RopeArgs &a, int i, int pos) {
    double f = exp2(a.step * (double)i);
    if (a.yarn) {
        const double g = fmin(1.0, fmax(0.0, (f * a.turns - a.beta_slow) * a.inv_beta));
        f *= g + (1.0 - g) * a.inv_factor;
    } else {
        f *= a.inv_factor;
    }
    // quarter turns, then the rest of at most an eighth turn in float32
    const double y = (double)pos * f * 0.63661977236758134308;
    const double k = rint(y);
    float s, c;
    sincosf((float)((y - k) * 1.57079632679489661923), &s, &c);
    const int q = (int)((long long)k & 3);
    const float cq = (q & 1) ? s : c, sq = (q & 1) ? c : s;
    return make_float2((q == 1 || q == 2 ? -cq : cq) * a.gain, (q >= 2 ? -sq : sq) * a.gain);
}

// (the conversion rounds to nearest even and keeps a NaN one)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
__device__ __forceinline__ f32x4_t load4(const float *p) { return *reinterpret_cast<const f32x4_t *>(p); }
__device__ __forceinline__ void store4(float *p, f32x4_t x) { *reinterpret_cast<f32x4_t *>(p) = x; }
__device__ __forceinline__ void store4(uint16_t *p, f32x4_t x) {
    *reinterpret_cast<u32x2_t *>(p) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
}
__device__ __forceinline__ void store1(float *p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t *p, float x) { *p = (uint16_t)pack_bf16(x, 0.0f); }

constexpr int ROPE_THREADS = 256;

// UNITS: rotary_dim is a multiple of eight, so every unit is four pairs or
// passes; otherwise a thread takes one element at a time.
template <typename TK, bool UNITS>
__global__ __launch_bounds__(ROPE_THREADS) void k_rope_append(RopeArgs a) {
    __shared__ __attribute__((aligned(16))) float2 turn[MAX_HEAD_DIM / 2];
    const int r = blockIdx.x, D = a.head_dim, H = a.n_heads, KVH = a.n_kv_heads, R = 2 * a.half;
    const int per = UNITS ? D / 8 : D, units = (H + 2 * KVH) * per;
    const int stride = gridDim.y * ROPE_THREADS;
    const float *x = a.qkv + (int64_t)r * a.ld_qkv;
    const int u0 = blockIdx.y * ROPE_THREADS + threadIdx.x;
    // unit w of a head: its two groups of four elements
    auto first_of = [&](int head, int w, int &e1) {
        if (head < H + KVH && 8 * w < R && !a.interleaved) {
            e1 = 4 * w + a.half;
            return 4 * w;
        }
        e1 = 8 * w + 4;
        return 8 * w;
    };
    f32x4_t p = {}, q = {};
    auto load = [&](int u) {
        const int head = u / per, w = u - head * per;
        int e1;
        const int e0 = first_of(head, w, e1);
        p = load4(x + (int64_t)head * D + e0);
        q = load4(x + (int64_t)head * D + e1);
    };
    if (UNITS && u0 < units)
        load(u0);
    if ((int)threadIdx.x < a.half)
        turn[threadIdx.x] = rope_turn(a, threadIdx.x, a.positions ? a.positions[r] : a.pos0 + r);
    __syncthreads();
    for (int u = u0; u < units; u += stride) {
        const int head = u / per, w = u - head * per;
        // where the head goes: queries to q, keys and values to the cache row
        float *qh = head < H ? a.q + (int64_t)r * a.ld_q + (int64_t)head * D : nullptr;
        TK *ch = nullptr;
        if (head >= H) {
            const int g = (head - H) % KVH;
            ch = static_cast<TK *>(head < H + KVH ? a.k : a.v) + (int64_t)g * a.head_stride +
                 (int64_t)(a.slot + r) * a.row_stride;
        }
        const bool turned = head < H + KVH;
        if constexpr (UNITS) {
            int e1;
            const int e0 = first_of(head, w, e1);
            f32x4_t np = p, nq = q;
            if (turned && 8 * w < R) {
                const f32x4_t t0 = *reinterpret_cast<const f32x4_t *>(turn + 4 * w),
                              t1 = *reinterpret_cast<const f32x4_t *>(turn + 4 * w + 2);
                const float c[4] = {t0[0], t0[2], t1[0], t1[2]}, s[4] = {t0[1], t0[3], t1[1], t1[3]};
                if (a.interleaved) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        np[2 * j] = p[2 * j] * c[j] - p[2 * j + 1] * s[j];
                        np[2 * j + 1] = p[2 * j + 1] * c[j] + p[2 * j] * s[j];
                        nq[2 * j] = q[2 * j] * c[2 + j] - q[2 * j + 1] * s[2 + j];
                        nq[2 * j + 1] = q[2 * j + 1] * c[2 + j] + q[2 * j] * s[2 + j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        np[j] = p[j] * c[j] - q[j] * s[j];
                        nq[j] = q[j] * c[j] + p[j] * s[j];
                    }
                }
            }
            if (u + stride < units)
                load(u + stride);
            if (qh) {
                store4(qh + e0, np);
                store4(qh + e1, nq);
            } else {
                store4(ch + e0, np);
                store4(ch + e1, nq);
            }
        } else {
            const float *xh = x + (int64_t)head * D;
            float y = xh[w];
            if (turned && w < R) {
                const bool second = a.interleaved ? (w & 1) : w >= a.half;
                const int i = a.interleaved ? w >> 1 : (second ? w - a.half : w);
                const float z = xh[a.interleaved ? w ^ 1 : (second ? w - a.half : w + a.half)];
                const float2 t = turn[i];
                y = second ? y * t.x + z * t.y : y * t.x - z * t.y;
            }
            if (qh)
                qh[w] = y;
            else
                store1(ch + w, y);
        }
    }
}

// ---------------------------------------------------------------------------
// The greedy walk.  4 n vocab bytes of logits are read once: bound by memory for
// many nodes, by two launches for a few.  A row is cut into slices of the
// vocabulary so that a few rows fill the CUs; a slice leaves (largest logit,
// lowest id) as one 64-bit key that orders like the pair, and one work-group
// then takes the rows' maxima and walks.  32000 logits a row: 13 rows 3.0 + 2.9 us,
// 700 rows 17.1 us (5.2 TB/s) and 3.9.

constexpr int ACC_THREADS = 256;
constexpr int WALK_THREADS = 1024;

// A (logit, id) pair as a key that orders like it: larger logits above, then
// lower ids; 0 is below every pair.  (The zeros are equal.)
__device__ __forceinline__ uint64_t best_key(float x, int id) {
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return ((uint64_t)o << 32) | (uint32_t)(0x7fffffff - id);
}
// Slice `s` of a vocabulary cut into slices of `slice` ids: ids [first, end).
// (The last slice's first id plus a slice can be past 2^31 - 1.)
struct Slice {
    int32_t first, end;
};
__host__ __device__ __forceinline__ Slice vocab_slice(int32_t vocab, int32_t slice, int32_t s) {
    const int32_t first = s * slice, left = vocab - first;
    return {first, first + (slice < left ? slice : left)};
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint32_t lo = __shfl_xor((uint32_t)v, o, 64), hi = __shfl_xor((uint32_t)(v >> 32), o, 64);
        v = max64(v, ((uint64_t)hi << 32) | lo);
    }
    return v;
}

struct AcceptArgs {
    const float *logits;
    int64_t ld;
    const int32_t *tokens, *parents;
    int32_t *walk;
    uint64_t *keys;  // [n][slices]
    int32_t vocab, n, slices, slice;
};

// A thread's ids ascend, so a logit wins only where it is larger than the one
// before, which a NaN never is: a comparison and two selects a logit.  Four
// loads of a thread are in flight (a load at a time: 21.3 us for 700 rows of
// 32000, 4.2 TB/s).  A slice without a logit above minus infinity, which no
// thread then reports, is looked through once more for its first one.
constexpr int BEST_LOADS = 4;
__global__ __launch_bounds__(ACC_THREADS) void k_row_best(AcceptArgs a) {
    __shared__ uint64_t red[ACC_THREADS / 64];
    const int r = blockIdx.y, tid = threadIdx.x;
    const Slice ids = vocab_slice(a.vocab, a.slice, blockIdx.x);
    const int i0 = ids.first, i1 = ids.end;
    const float *x = a.logits + (int64_t)r * a.ld;
    float top = -INFINITY;
    int id = -1;
    auto take = [&](float v, int i) {
        const bool wins = v > top;
        top = wins ? v : top;
        id = wins ? i : id;
    };
    // (the head and the tail that are not whole 16-byte words one by one)
    const int lead = min(i1 - i0, (int)((4 - (((uintptr_t)(x + i0) >> 2) & 3)) & 3));
    if (tid < lead)
        take(x[i0 + tid], i0 + tid);
    const int w0 = i0 + lead, words = (i1 - w0) / 4, tail = w0 + 4 * words;
    const f32x4_t *xw = reinterpret_cast<const f32x4_t *>(x + w0);
    int w = tid;
    for (; w + (BEST_LOADS - 1) * ACC_THREADS < words; w += BEST_LOADS * ACC_THREADS) {
        f32x4_t v[BEST_LOADS];
#pragma unroll
        for (int u = 0; u < BEST_LOADS; ++u)
            v[u] = __builtin_nontemporal_load(xw + w + u * ACC_THREADS);
#pragma unroll
        for (int u = 0; u < BEST_LOADS; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                take(v[u][j], w0 + 4 * (w + u * ACC_THREADS) + j);
    }
    for (; w < words; w += ACC_THREADS) {
        const f32x4_t v = __builtin_nontemporal_load(xw + w);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            take(v[j], w0 + 4 * w + j);
    }
    if (tid < i1 - tail)
        take(x[tail + tid], tail + tid);
    uint64_t best = wave_max64(id >= 0 ? best_key(top, id) : 0);
    if ((tid & 63) == 0)
        red[tid >> 6] = best;
    __syncthreads();
    best = red[0];
#pragma unroll
    for (int v = 1; v < ACC_THREADS / 64; ++v)
        best = max64(best, red[v]);
    if (best == 0) {  // uniform
        for (int i = i0 + tid; i < i1 && id < 0; i += ACC_THREADS)
            if (x[i] == -INFINITY)
                id = i;
        best = wave_max64(id >= 0 ? best_key(-INFINITY, id) : 0);
        __syncthreads();
        if ((tid & 63) == 0)
            red[tid >> 6] = best;
        __syncthreads();
        best = red[0];
#pragma unroll
        for (int v = 1; v < ACC_THREADS / 64; ++v)
            best = max64(best, red[v]);
    }
    if (tid == 0)
        a.keys[(int64_t)r * a.slices + blockIdx.x] = best;
}

// One work-group, a thread per node: best tokens, then the lowest matching child
// of every node by an LDS minimum, then the walk itself (at most n steps: a
// child's number is above its parent's).
__global__ __launch_bounds__(WALK_THREADS) void k_walk(AcceptArgs a) {
    __shared__ int32_t best[SD_TREE_MAX], child[SD_TREE_MAX];
    const int i = threadIdx.x;
    int p = -1, tok = 0;
    if (i < a.n) {
        p = a.parents[i];
        tok = a.tokens[i];
        uint64_t k = 0;
        for (int s = 0; s < a.slices; ++s)
            k = max64(k, a.keys[(int64_t)i * a.slices + s]);
        best[i] = k ? 0x7fffffff - (int32_t)(uint32_t)k : 0;
        child[i] = a.n;
    }
    __syncthreads();
    if (i > 0 && i < a.n) {
        if (p >= 0 && p < i && tok == best[p])
            atomicMin(&child[p], i);
    }
    if (i < a.n) {
        a.walk[2 + i] = -1;
        a.walk[2 + a.n + i] = best[i];
    }
    __syncthreads();
    if (i == 0) {
        int cur = 0, count = 0;
        for (;;) {
            a.walk[2 + count++] = cur;
            const int next = child[cur];
            if (next >= a.n)
                break;
            cur = next;
        }
        a.walk[0] = count;
        a.walk[1] = best[cur];
    }
}

// Slices of the vocabulary per row: enough work-groups for eight on every CU,
// slices of at least 2048 logits (two words a thread).  64 bits: the sums pass
// 2^31 - 1 at the largest vocabularies.
constexpr int32_t ACC_VOCAB = INT32_MAX - 4096;  // the largest
int accept_slices(int32_t n, int64_t vocab, int32_t *slice) {
    const int64_t most = (vocab + 2047) / 2048, want = (2048 + n - 1) / n;
    const int64_t slices = std::max<int64_t>(1, std::min(most, want));
    *slice = (int32_t)(((vocab + slices - 1) / slices + 3) / 4 * 4);
    return (int)((vocab + *slice - 1) / *slice);
}

// ---------------------------------------------------------------------------
// The move of a path's rows.  A wave takes one plane; its lanes hold whole
// rows of 16-byte words.  The path ascends, so path[i] >= i, and row i is
// written after every row path[j], j <= i, has been read and is no later row's
// source (path[j] >= j > i): batches of rows may follow one another in place,
// each read whole before it is written.  17 rows of 256 bytes in 3200 planes
// 7.3 us (3.7 TB/s: a wave's reads, then its writes), 4 rows in 1280 planes 3.3
// (7.6 and 3.7 with half the words in flight and none passed over).

struct KeepArgs {
    char *kv;
    int64_t planes, plane_stride;
    int32_t row_bytes, base, n;
    const int32_t *walk;
};
constexpr int KEEP_THREADS = 256;
constexpr int KEEP_WORDS = 8;  // 16-byte words in flight per lane

__global__ __launch_bounds__(KEEP_THREADS) void k_kv_keep(KeepArgs a) {
    __shared__ int32_t path[SD_TREE_MAX];
    __shared__ int32_t first;  // of the path's rows that move
    const int tid = threadIdx.x, lane = tid & 63;
    // the count and the path in one round trip
    if (tid == 0)
        first = a.n;
    const int count = a.walk[0];
    bool bad = count < 1 || count > a.n;
    int below = -1;
    for (int i = tid; i < a.n; i += KEEP_THREADS) {
        const int p = a.walk[2 + i], before = i > 0 ? a.walk[1 + i] : -1;
        path[i] = p;
        bad |= i < count && (p < 0 || p >= a.n || (i > 0 && p <= before));
        if (i < count && p != i && below < 0)
            below = i;
    }
    bad = __syncthreads_or(bad);
    if (bad)
        return;  // uniform
    if (below >= 0)
        atomicMin(&first, below);
    __syncthreads();
    const int64_t plane = (int64_t)blockIdx.x * (KEEP_THREADS / 64) + (tid >> 6);
    if (plane >= a.planes)
        return;
    char *rows = a.kv + plane * a.plane_stride + (int64_t)a.base * a.row_bytes;
    const int wpr = a.row_bytes >> 4;
    // the path leaves its nodes' numbers once: the rows before stay where they are
    const int words = count * wpr;
    for (int w0 = first * wpr; w0 < words; w0 += 64 * KEEP_WORDS) {
        u32x4_t v[KEEP_WORDS];
#pragma unroll
        for (int j = 0; j < KEEP_WORDS; ++j) {
            if (w0 + 64 * j >= words)  // uniform
                break;
            const int w = min(w0 + 64 * j + lane, words - 1), i = w / wpr;
            v[j] = *reinterpret_cast<const u32x4_t *>(rows + (int64_t)path[i] * a.row_bytes + 16 * (w - i * wpr));
        }
        // (every load of the batch has returned before its first store is issued)
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < KEEP_WORDS; ++j) {
            const int w = w0 + 64 * j + lane, i = w / wpr;
            if (w < words)
                *reinterpret_cast<u32x4_t *>(rows + (int64_t)i * a.row_bytes + 16 * (w - i * wpr)) = v[j];
        }
    }
}

sd_status tree_layout(const int32_t *parents, int32_t n, int32_t *depths, uint64_t *mask) {
    if (!parents || n < 1 || n > SD_TREE_MAX)
        return report(SD_ERR_INVALID_ARG, "a tree has 1 to " + std::to_string(SD_TREE_MAX) + " nodes, and parents");
    for (int32_t i = 0; i < n; ++i)
        if (i == 0 ? parents[0] != -1 : (parents[i] < 0 || parents[i] >= i))
            return report(SD_ERR_INVALID_ARG, "parents[" + std::to_string(i) + "] = " + std::to_string(parents[i]) +
                                                  ": the root has -1, every other node a node before it");
    const int words = (n + 63) / 64;
    for (int32_t i = 0; i < n; ++i) {
        const int32_t p = parents[i];
        if (depths)
            depths[i] = p < 0 ? 0 : depths[p] + 1;
        if (mask) {
            for (int w = 0; w < words; ++w)
                mask[(size_t)i * words + w] = p < 0 ? 0 : mask[(size_t)p * words + w];
            mask[(size_t)i * words + i / 64] |= (uint64_t)1 << (i % 64);
        }
    }
    return SD_OK;
}

sd_status rope_append(const sd_rope *rope, const float *qkv, int64_t ld_qkv, int32_t n, int32_t n_heads,
                      const int32_t *positions, int32_t pos0, float *q_out, int64_t ld_q, const sd_kv_layer *kv,
                      int32_t slot, hipStream_t s) {
    const sd_status st = check_layer(kv);
    if (st != SD_OK)
        return st;
    RopeArgs a{};
    const sd_status rt = check_rope(rope, kv->head_dim);
    if (rt != SD_OK)
        return rt;
    rope_form(*rope, &a);
    const int64_t D = kv->head_dim, KVH = kv->n_kv_heads;
    if (!qkv || !q_out || !aligned16(qkv) || !aligned16(q_out) || ((uintptr_t)positions & 3))
        return report(SD_ERR_INVALID_ARG, "qkv and q_out must be set and 16-byte aligned");
    if (n < 1 || n > 1 << 20 || n_heads < 1 || n_heads > 4096 || n_heads % KVH)
        return report(SD_ERR_INVALID_ARG, "n must be in [1, 2^20], n_heads a multiple of n_kv_heads and at most 4096");
    if (ld_qkv % 4 || ld_q % 4 || ld_qkv < (n_heads + 2 * KVH) * D || ld_q < n_heads * D)
        return report(SD_ERR_INVALID_ARG, "ld_qkv and ld_q must hold a row and be multiples of 4");
    if (!positions && (int64_t)pos0 + n - 1 > INT32_MAX)
        return report(SD_ERR_INVALID_ARG, "pos0 + n is past the last position");
    if (slot < 0 || (int64_t)slot + n > kv->capacity)
        return report(SD_ERR_CAPACITY, "a layer of capacity " + std::to_string(kv->capacity) + " does not hold " +
                                           std::to_string(n) + " rows from " + std::to_string(slot));
    a.qkv = qkv;
    a.ld_qkv = ld_qkv;
    a.positions = positions;
    a.pos0 = pos0;
    a.n = n;
    a.n_heads = n_heads;
    a.n_kv_heads = (int32_t)KVH;
    a.head_dim = (int32_t)D;
    a.q = q_out;
    a.ld_q = ld_q;
    a.k = kv->k;
    a.v = kv->v;
    a.head_stride = kv->head_stride;
    a.row_stride = kv->row_stride;
    a.slot = slot;
    const bool units = a.half % 4 == 0, bf16 = kv->dtype == SD_BF16;
    const int64_t work = (n_heads + 2 * KVH) * (units ? D / 8 : D);
    // shares of a row: about four work-groups per CU
    const int64_t most = (work + ROPE_THREADS - 1) / ROPE_THREADS, want = std::max(1, 1024 / n);
    const dim3 grid((unsigned)n, (unsigned)std::min(most, want)), block(ROPE_THREADS);
    if (bf16 && units)
        hipLaunchKernelGGL((k_rope_append<uint16_t, true>), grid, block, 0, s, a);
    else if (bf16)
        hipLaunchKernelGGL((k_rope_append<uint16_t, false>), grid, block, 0, s, a);
    else if (units)
        hipLaunchKernelGGL((k_rope_append<float, true>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_rope_append<float, false>), grid, block, 0, s, a);
    return launched("rotary embedding");
}

}  // namespace

namespace sdk {

sd_status check_layer(const sd_kv_layer *kv) {
    if (!kv || !kv->k || !kv->v || !aligned16(kv->k) || !aligned16(kv->v))
        return report(SD_ERR_INVALID_ARG, "the layer's k and v must be set and 16-byte aligned");
    if (kv->dtype != SD_F32 && kv->dtype != SD_BF16)
        return report(SD_ERR_INVALID_ARG, "dtype must be SD_F32 or SD_BF16");
    const int32_t D = kv->head_dim, unit = kv->dtype == SD_BF16 ? 8 : 4;
    if (D < 16 || D > MAX_HEAD_DIM || (D & (D - 1)) || kv->n_kv_heads < 1 || kv->capacity < 1 ||
        kv->capacity > 1 << 30)
        return report(SD_ERR_INVALID_ARG, "head_dim must be a power of two in [16, 128], n_kv_heads >= 1 and capacity in "
                                          "[1, 2^30]");
    const int64_t hs = kv->head_stride, rs = kv->row_stride, most = (int64_t)1 << 40;
    if (rs < D || rs % unit || hs < 0 || hs % unit || rs > most || hs > most)
        return report(SD_ERR_INVALID_ARG, "strides must be multiples of 16 bytes, row_stride at least head_dim");
    const auto reach = [](int64_t count, int64_t stride, int64_t width) {
        return count <= 1 ? 0.0 : (double)(count - 1) * (double)stride + (double)width;
    };
    if ((double)hs < reach(kv->capacity, rs, D) && (double)rs < reach(kv->n_kv_heads, hs, D) &&
        kv->n_kv_heads > 1 && kv->capacity > 1)
        return report(SD_ERR_INVALID_ARG, "rows of the layer overlap");
    if (kv->n_kv_heads > 1 && hs < D)
        return report(SD_ERR_INVALID_ARG, "rows of the layer overlap");
    return SD_OK;
}

sd_status check_rope(const sd_rope *r, int32_t head_dim) {
    if (!r)
        return report(SD_ERR_INVALID_ARG, "rope is null");
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > head_dim)
        return report(SD_ERR_INVALID_ARG, "rotary_dim must be even and in [2, head_dim]");
    if ((r->layout != SD_ROPE_HALF && r->layout != SD_ROPE_INTERLEAVED) || r->scaling < SD_ROPE_UNSCALED ||
        r->scaling > SD_ROPE_YARN)
        return report(SD_ERR_INVALID_ARG, "unknown rotary layout or scaling");
    // (positions reach 2^31: with a frequency of at most 1e9 an angle's quarter turns fit 64 bits)
    if (!(r->base >= 1e-9) || !std::isfinite(r->base) || !std::isfinite((float)r->gain))
        return report(SD_ERR_INVALID_ARG, "base must be at least 1e-9, base and gain finite (gain in float32)");
    const bool scaled = r->scaling != SD_ROPE_UNSCALED;
    if (scaled && (!(r->factor >= 1.0) || !std::isfinite(r->factor)))
        return report(SD_ERR_INVALID_ARG, "the factor of a scaled rotary embedding must be >= 1 and finite");
    if (r->scaling == SD_ROPE_NTK && (r->rotary_dim < 4 || !std::isfinite(scaled_base(*r))))
        return report(SD_ERR_INVALID_ARG, "NTK scaling needs rotary_dim >= 4 and a finite scaled base");
    if (r->scaling == SD_ROPE_YARN && (!(r->beta_slow >= 0.0) || !(r->beta_fast > r->beta_slow) ||
                                       !std::isfinite(r->beta_fast) || r->original_context < 1))
        return report(SD_ERR_INVALID_ARG, "YARN needs beta_fast > beta_slow >= 0 and original_context >= 1");
    return SD_OK;
}

double rope_frequency(const sd_rope &r, int32_t i) {
    const double f = std::pow(scaled_base(r), -2.0 * (double)i / (double)r.rotary_dim);
    if (r.scaling == SD_ROPE_LINEAR)
        return f / r.factor;
    if (r.scaling == SD_ROPE_YARN) {
        const double turns = f * r.original_context / 6.28318530717958647693;
        const double g = std::min(1.0, std::max(0.0, (turns - r.beta_slow) / (r.beta_fast - r.beta_slow)));
        return f * (g + (1.0 - g) / r.factor);
    }
    return f;
}

double rope_gain(const sd_rope &r) {
    return r.gain != 0.0 ? r.gain : r.scaling == SD_ROPE_YARN ? 0.1 * std::log(r.factor) + 1.0 : 1.0;
}

}  // namespace sdk

extern "C" {

sd_status sd_tree_layout(const int32_t *parents, int32_t n, int32_t *depths, uint64_t *mask) {
    SD_GUARD(return tree_layout(parents, n, depths, mask);)
}

sd_status sd_rope_append(const sd_rope *rope, const float *qkv, int64_t ld_qkv, int32_t n, int32_t n_heads,
                         const int32_t *positions, int32_t pos0, float *q_out, int64_t ld_q, const sd_kv_layer *kv,
                         int32_t slot, void *hip_stream) {
    SD_GUARD(return rope_append(rope, qkv, ld_qkv, n, n_heads, positions, pos0, q_out, ld_q, kv, slot,
                                reinterpret_cast<hipStream_t>(hip_stream));)
}

size_t sd_tree_accept_workspace(int32_t n, int32_t vocab) {
    if (n < 1 || n > SD_TREE_MAX || vocab < 1 || vocab > ACC_VOCAB)
        return 0;
    int32_t slice;
    return sizeof(uint64_t) * (size_t)n * accept_slices(n, vocab, &slice);
}

sd_status sd_tree_accept(const float *logits, int64_t ld, int32_t vocab, const int32_t *tokens, const int32_t *parents,
                         int32_t n, int32_t *walk, void *workspace, size_t workspace_bytes, void *hip_stream) {
    SD_GUARD(
        if (!logits || !tokens || !parents || !walk || (((uintptr_t)logits | (uintptr_t)tokens | (uintptr_t)parents |
                                                         (uintptr_t)walk) & 3))
            return report(SD_ERR_INVALID_ARG, "logits, tokens, parents and walk must be set and aligned");
        if (n < 1 || n > SD_TREE_MAX || vocab < 1 || vocab > ACC_VOCAB || ld < vocab)
            return report(SD_ERR_INVALID_ARG, "a tree has 1 to " + std::to_string(SD_TREE_MAX) +
                                                  " nodes, a row of logits at least one entry and at most ld");
        if (!workspace || !aligned16(workspace) || workspace_bytes < sd_tree_accept_workspace(n, vocab))
            return report(SD_ERR_INVALID_ARG, "the walk needs " + std::to_string(sd_tree_accept_workspace(n, vocab)) +
                                                  " bytes of 16-byte aligned workspace");
        AcceptArgs a{};
        a.logits = logits; a.ld = ld; a.tokens = tokens; a.parents = parents; a.walk = walk;
        a.keys = static_cast<uint64_t *>(workspace); a.vocab = vocab; a.n = n;
        a.slices = accept_slices(n, vocab, &a.slice);
        hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
        hipLaunchKernelGGL(k_row_best, dim3(a.slices, n), dim3(ACC_THREADS), 0, s, a);
        const sd_status st = launched("row maxima");
        if (st != SD_OK) return st;
        hipLaunchKernelGGL(k_walk, dim3(1), dim3(WALK_THREADS), 0, s, a);
        return launched("greedy walk");)
}

sd_status sd_kv_keep(void *kv, int64_t planes, int64_t plane_stride, int32_t row_bytes, int32_t capacity, int32_t base,
                     const int32_t *walk, int32_t n, void *hip_stream) {
    SD_GUARD(
        if (!kv || !walk || !aligned16(kv) || ((uintptr_t)walk & 3))
            return report(SD_ERR_INVALID_ARG, "kv must be set and 16-byte aligned, and walk set");
        if (planes < 1 || planes > 1 << 24 || row_bytes < 16 || row_bytes % 16 || row_bytes > 65536 ||
            capacity < 1 || n < 1 || n > SD_TREE_MAX || plane_stride % 16 ||
            (planes > 1 && plane_stride < (int64_t)capacity * row_bytes))
            return report(SD_ERR_INVALID_ARG, "1 to 2^24 planes hold capacity rows of row_bytes (a multiple of 16, at most "
                                              "65536), plane_stride is a multiple of 16, a tree has 1 to " +
                                                  std::to_string(SD_TREE_MAX) + " nodes");
        if (base < 0 || (int64_t)base + n > capacity)
            return report(SD_ERR_CAPACITY, "planes of " + std::to_string(capacity) + " rows do not hold " +
                                               std::to_string(n) + " nodes from " + std::to_string(base));
        KeepArgs a{static_cast<char *>(kv), planes, plane_stride, row_bytes, base, n, walk};
        const int64_t groups = (planes + KEEP_THREADS / 64 - 1) / (KEEP_THREADS / 64);
        hipLaunchKernelGGL(k_kv_keep, dim3((unsigned)groups), dim3(KEEP_THREADS), 0,
                           reinterpret_cast<hipStream_t>(hip_stream), a);
        return launched("cache move");)
}

// For the tests: the ids of slice s of a row, as the row maxima take them; returns
// the number of slices (-1: refused sizes).
int32_t sdk_accept_slice(int32_t n, int32_t vocab, int32_t s, int32_t *first, int32_t *end) {
    int32_t slice;
    if (!sd_tree_accept_workspace(n, vocab))
        return -1;
    const int slices = accept_slices(n, vocab, &slice);
    const Slice ids = vocab_slice(vocab, slice, s);
    *first = ids.first;
    *end = ids.end;
    return slices;
}

}  // extern "C"
