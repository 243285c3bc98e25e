// Norms of the heads, rotary embedding, and the append of keys and values to the
// pages of a cache.
//
// Row r belongs to the sequence s with starts[s] <= r < starts[s + 1] and stands
// at position p = lengths[s] - m + i; its keys and values go to row p % page_size of
// page table[s][p / page_size].
#include "paged.h"

#include <algorithm>
#include <cmath>
#include <string>

#include "host_api.h"
#include "rope.h"
#include "sd_internal.h"

using namespace sdk;

namespace {

struct AppendArgs : RopeForm {
    const void *x;
    int64_t ld_x;
    const int32_t *positions;
    const void *q_norm, *k_norm;
    float eps;
    void *q;
    int64_t ld_q;
    void *k, *v;
    int64_t page_stride, head_stride, row_stride;
    const int32_t *table, *lengths, *starts;
    int64_t ld_table;
    int32_t n_seqs, max_rows, max_length, n_pages, page_shift;
    int32_t n, n_heads, n_kv_heads, head_dim;
};

constexpr int APPEND_THREADS = 256;

// A work-group takes a row, or a share of one where there are few rows; a thread
// units of eight elements of a head, and the head_dim / 8 threads of a head add up
// its squares.  FOURS: rotary_dim is a multiple of eight, so a unit is four pairs
// (of a head that is rotated in halves) or eight elements in a row; otherwise eight
// in a row whose partners are fetched one by one.
//
// Elements (x, y) of a pair become (x cos - y sin, y cos + x sin); angles in float64 once a
// row (one of 2^31 is off by 2^-22 then), squares and means in float32.  Bound by memory where
// there are many rows (1665 of 64 heads on 8, bfloat16, with norms, 17.9 us, 3.8 TB/s), else
// by the reads of starts, lengths and table, one after another, before the store (16
// rows 3.4 us); the first units are asked for before those.  Four or five units of a
// thread under way at once: 20 -> 22.5 us; frequencies from the host: no faster.  A
// head's squares are added by moves between its lanes.
template <typename TX, typename TK, bool FOURS>
__global__ __launch_bounds__(APPEND_THREADS) void k_paged_append(AppendArgs a) {
    __shared__ __attribute__((aligned(16))) float2 turn[MAX_HEAD_DIM / 2];
    const int r = blockIdx.x, D = a.head_dim, H = a.n_heads, KVH = a.n_kv_heads, R = 2 * a.half;
    const int per = D / 8, units = (H + 2 * KVH) * per, stride = gridDim.y * APPEND_THREADS;
    const TX *x = static_cast<const TX *>(a.x) + (int64_t)r * a.ld_x;
    const int u0 = blockIdx.y * APPEND_THREADS + threadIdx.x;
    // unit w of a head: its two groups of four elements
    auto first_of = [&](int head, int w, int &e1) {
        if (FOURS && head < H + KVH && 8 * w < R && !a.interleaved) {
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
    if (u0 < units)
        load(u0);
    // the row's sequence, and its place there
    int s;
    SeqRows rows;
    if (a.starts) {
        s = wave_count(a.n_seqs, r, [&](int j) { return (int64_t)a.starts[j]; });
        if (s >= a.n_seqs)
            return;  // uniform
        const int start = a.starts[s];
        if (start > r)
            return;
        rows = seq_rows(start, a.starts[s + 1], a.lengths[s], a.n, a.max_rows);
    } else {
        s = r / a.max_rows;
        rows = seq_rows(s * a.max_rows, (s + 1) * a.max_rows, a.lengths[s], a.n, a.max_rows);
    }
    const int i = r - rows.first;
    if (i < 0 || i >= rows.m)
        return;
    const int at = rows.past + i;
    int page = -1;
    if (at >= 0 && at < a.max_length)
        page = a.table[(int64_t)s * a.ld_table + (at >> a.page_shift)];
    const bool stored = (uint32_t)page < (uint32_t)a.n_pages;
    const int64_t to = (int64_t)page * a.page_stride + (int64_t)(at & ((1 << a.page_shift) - 1)) * a.row_stride;
    if ((int)threadIdx.x < a.half)
        turn[threadIdx.x] = rope_turn(a, threadIdx.x, a.positions ? a.positions[r] : at);
    __syncthreads();
    for (int u = u0; u < units; u += stride) {
        const int head = u / per, w = u - head * per;
        // where the head goes: queries to q, keys and values to the row of the page
        TX *qh = head < H ? static_cast<TX *>(a.q) + (int64_t)r * a.ld_q + (int64_t)head * D : nullptr;
        TK *ch = nullptr;
        if (head >= H) {
            const int g = (head - H) % KVH;
            ch = static_cast<TK *>(head < H + KVH ? a.k : a.v) + to + (int64_t)g * a.head_stride;
        }
        const bool key = head < H + KVH;  // a query or a key
        int e1;
        const int e0 = first_of(head, w, e1);
        const TK *norm = static_cast<const TK *>(head < H ? a.q_norm : a.k_norm);
        f32x4_t np = p, nq = q;
        float inv = 1.0f;
        if (a.q_norm) {
            // (every thread of the head takes part; values have no norm)
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum = fmaf(p[j], p[j], fmaf(q[j], q[j], sum));
            // over the 2, 4, 8 or 16 lanes of the head
            sum += dpp_mov<DPP_QUAD_XOR1>(sum);
            if (per >= 4)
                sum += dpp_mov<DPP_QUAD_XOR2>(sum);
            if (per >= 8)
                sum += dpp_mov<DPP_ROW_HALF_MIRROR>(sum);
            if (per >= 16)
                sum += dpp_mov<DPP_ROW_ROR8>(sum);
            inv = rsqrtf(sum / (float)D + a.eps);
            if (key) {
                np = np * inv * load4(norm + e0);
                nq = nq * inv * load4(norm + e1);
            }
        }
        if (key && 8 * w < R) {
            if constexpr (FOURS) {
                const f32x4_t t0 = *reinterpret_cast<const f32x4_t *>(turn + 4 * w),
                              t1 = *reinterpret_cast<const f32x4_t *>(turn + 4 * w + 2);
                const float c[4] = {t0[0], t0[2], t1[0], t1[2]}, n[4] = {t0[1], t0[3], t1[1], t1[3]};
                const f32x4_t y = np, z = nq;
                if (a.interleaved) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        np[2 * j] = y[2 * j] * c[j] - y[2 * j + 1] * n[j];
                        np[2 * j + 1] = y[2 * j + 1] * c[j] + y[2 * j] * n[j];
                        nq[2 * j] = z[2 * j] * c[2 + j] - z[2 * j + 1] * n[2 + j];
                        nq[2 * j + 1] = z[2 * j + 1] * c[2 + j] + z[2 * j] * n[2 + j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        np[j] = y[j] * c[j] - z[j] * n[j];
                        nq[j] = z[j] * c[j] + y[j] * n[j];
                    }
                }
            } else {
                const TX *xh = x + (int64_t)head * D;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int e = 8 * w + j;
                    if (e < R) {
                        const bool second = a.interleaved ? (e & 1) : e >= a.half;
                        const int pair = a.interleaved ? e >> 1 : (second ? e - a.half : e);
                        const int other = a.interleaved ? e ^ 1 : (second ? e - a.half : e + a.half);
                        const float y = j < 4 ? np[j & 3] : nq[j & 3];
                        float z = load1(xh + other);
                        if (a.q_norm)
                            z = z * inv * load1(norm + other);
                        const float2 t = turn[pair];
                        const float v = second ? y * t.x + z * t.y : y * t.x - z * t.y;
                        if (j < 4)
                            np[j & 3] = v;
                        else
                            nq[j & 3] = v;
                    }
                }
            }
        }
        if (u + stride < units)
            load(u + stride);
        if (qh) {
            store4(qh + e0, np);
            store4(qh + e1, nq);
        } else if (stored) {
            store4(ch + e0, np);
            store4(ch + e1, nq);
        }
    }
}

template <typename TX, typename TK>
void launch_append(const AppendArgs &a, bool fours, dim3 grid, hipStream_t s) {
    if (fours)
        hipLaunchKernelGGL((k_paged_append<TX, TK, true>), grid, dim3(APPEND_THREADS), 0, s, a);
    else
        hipLaunchKernelGGL((k_paged_append<TX, TK, false>), grid, dim3(APPEND_THREADS), 0, s, a);
}

sd_status paged_append(const sd_rope *rope, const void *qkv, int64_t ld_qkv, int32_t x_dtype, int32_t n, int32_t n_heads,
                       const int32_t *positions, const void *q_norm, const void *k_norm, float eps, void *q_out,
                       int64_t ld_q, const sd_kv_pages *kv, const sd_batch *batch, hipStream_t s) {
    sd_status st = check_pages(kv);
    if (st != SD_OK)
        return st;
    AppendArgs a{};
    if ((st = check_rope(rope, kv->head_dim)) != SD_OK || (st = check_rows(n, n_heads, kv->n_kv_heads)) != SD_OK ||
        (st = check_batch(batch, kv, n, true)) != SD_OK)
        return st;
    rope_form(*rope, &a);
    const int64_t D = kv->head_dim, KVH = kv->n_kv_heads;
    if (x_dtype != SD_F32 && x_dtype != SD_BF16)
        return report(SD_ERR_INVALID_ARG, "x_dtype must be SD_F32 or SD_BF16");
    if (!qkv || !q_out || !aligned16(qkv) || !aligned16(q_out) || ((uintptr_t)positions & 3))
        return report(SD_ERR_INVALID_ARG, "qkv and q_out must be set and 16-byte aligned, positions 4-byte aligned");
    const int unit = x_dtype == SD_BF16 ? 8 : 4;
    if (ld_qkv % unit || ld_q % unit || ld_qkv < (n_heads + 2 * KVH) * D || ld_q < n_heads * D)
        return report(SD_ERR_INVALID_ARG, "ld_qkv and ld_q must hold a row and be multiples of 16 bytes");
    if (!q_norm != !k_norm || !aligned16(q_norm) || !aligned16(k_norm))
        return report(SD_ERR_INVALID_ARG, "q_norm and k_norm are both set or both null, and 16-byte aligned");
    if (!(eps >= 0.0f) || !std::isfinite(eps))
        return report(SD_ERR_INVALID_ARG, "eps must be at least 0 and finite");
    a.x = qkv;
    a.ld_x = ld_qkv;
    a.positions = positions;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.eps = eps;
    a.q = q_out;
    a.ld_q = ld_q;
    a.k = kv->k;
    a.v = kv->v;
    a.page_stride = kv->page_stride;
    a.head_stride = kv->head_stride;
    a.row_stride = kv->row_stride;
    a.table = batch->table;
    a.lengths = batch->lengths;
    a.starts = batch->starts;
    a.ld_table = batch->ld_table;
    a.n_seqs = batch->n_seqs;
    a.max_rows = batch->max_rows;
    a.max_length = positions_of(*batch, *kv);
    a.n_pages = kv->n_pages;
    a.page_shift = log2_of(kv->page_size);
    a.n = n;
    a.n_heads = n_heads;
    a.n_kv_heads = (int32_t)KVH;
    a.head_dim = (int32_t)D;
    // shares of a row: about four work-groups per CU
    const int64_t most = ((n_heads + 2 * KVH) * (D / 8) + APPEND_THREADS - 1) / APPEND_THREADS, want = std::max(1, 1024 / n);
    const dim3 grid((unsigned)n, (unsigned)std::min(most, want));
    const bool fours = a.half % 4 == 0, bf16 = kv->dtype == SD_BF16;
    if (x_dtype == SD_BF16) {
        if (bf16)
            launch_append<uint16_t, uint16_t>(a, fours, grid, s);
        else
            launch_append<uint16_t, float>(a, fours, grid, s);
    } else if (bf16) {
        launch_append<float, uint16_t>(a, fours, grid, s);
    } else {
        launch_append<float, float>(a, fours, grid, s);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SD_OK : report(SD_ERR_DEVICE, std::string("paged append: ") + hipGetErrorString(e));
}

}  // namespace

namespace sdk {

sd_status check_pages(const sd_kv_pages *kv) {
    if (!kv || !kv->k || !kv->v || !aligned16(kv->k) || !aligned16(kv->v))
        return report(SD_ERR_INVALID_ARG, "the pages' k and v must be set and 16-byte aligned");
    if (kv->dtype != SD_F32 && kv->dtype != SD_BF16)
        return report(SD_ERR_INVALID_ARG, "dtype must be SD_F32 or SD_BF16");
    const int32_t D = kv->head_dim, P = kv->page_size, unit = kv->dtype == SD_BF16 ? 8 : 4;
    if (D < 16 || D > MAX_HEAD_DIM || (D & (D - 1)) || P < 16 || P > MAX_PAGE || (P & (P - 1)) || kv->n_kv_heads < 1 ||
        kv->n_kv_heads > MAX_QUERY_HEADS || kv->n_pages < 1)
        return report(SD_ERR_INVALID_ARG, "head_dim must be a power of two in [16, 128], page_size one in [16, 65536], "
                                          "n_kv_heads in [1, 4096] and n_pages >= 1");
    // rows do not overlap: by ascending stride, each level's stride holds the one inside it
    struct Level {
        int64_t count, stride;
    } level[3] = {{P, kv->row_stride}, {kv->n_kv_heads, kv->head_stride}, {kv->n_pages, kv->page_stride}};
    for (const Level &l : level)
        if (l.stride < 0 || l.stride % unit || l.stride > (int64_t)1 << 40)
            return report(SD_ERR_INVALID_ARG, "strides must be multiples of 16 bytes, and not negative");
    std::sort(level, level + 3, [](const Level &x, const Level &y) { return x.stride < y.stride; });
    double width = D;
    for (const Level &l : level) {
        if (l.count == 1)
            continue;
        if ((double)l.stride < width)
            return report(SD_ERR_INVALID_ARG, "rows of the pages overlap");
        width += (double)(l.count - 1) * (double)l.stride;
    }
    if (width > 4611686018427387904.0)
        return report(SD_ERR_INVALID_ARG, "the pages reach past 64 bits");
    return SD_OK;
}

sd_status check_batch(const sd_batch *b, const sd_kv_pages *kv, int32_t n, bool addresses) {
    if (!b)
        return report(SD_ERR_INVALID_ARG, "batch is null");
    if (addresses && (!b->table || !b->lengths || (((uintptr_t)b->table | (uintptr_t)b->lengths | (uintptr_t)b->starts) & 3)))
        return report(SD_ERR_INVALID_ARG, "the batch's table and lengths must be set, and its arrays 4-byte aligned");
    if (b->n_seqs < 1 || b->n_seqs > MAX_SEQS || b->table_pages < 1 || b->ld_table < b->table_pages ||
        b->ld_table > (int64_t)1 << 40 || (int64_t)b->table_pages * kv->page_size > MAX_POSITIONS)
        return report(SD_ERR_INVALID_ARG, "a batch has 1 to 65536 sequences, a table of at least one page and at most 2^30 "
                                          "positions a row, rows at most ld_table apart");
    if (b->max_rows < 1 || b->max_length < 0 || b->max_length > (int64_t)b->table_pages * kv->page_size)
        return report(SD_ERR_INVALID_ARG, "max_rows must be at least 1, max_length in [0, table_pages * page_size]");
    if (!b->starts && (int64_t)b->n_seqs * b->max_rows != n)
        return report(SD_ERR_INVALID_ARG, "without starts, n must be n_seqs * max_rows");
    return SD_OK;
}

sd_status check_rows(int32_t n, int32_t n_heads, int32_t n_kv_heads) {
    if (n < 1 || n > MAX_BATCH_ROWS || n_heads < 1 || n_heads > MAX_QUERY_HEADS || n_heads % n_kv_heads)
        return report(SD_ERR_INVALID_ARG, "n must be in [1, 2^20], n_heads a multiple of n_kv_heads and at most 4096");
    return SD_OK;
}

}  // namespace sdk

extern "C" {

sd_status sd_paged_append(const sd_rope *rope, const void *qkv, int64_t ld_qkv, int32_t x_dtype, int32_t n,
                          int32_t n_heads, const int32_t *positions, const void *q_norm, const void *k_norm, float eps,
                          void *q_out, int64_t ld_q, const sd_kv_pages *kv, const sd_batch *batch, void *hip_stream) {
    SD_GUARD(return paged_append(rope, qkv, ld_qkv, x_dtype, n, n_heads, positions, q_norm, k_norm, eps, q_out, ld_q, kv,
                                 batch, reinterpret_cast<hipStream_t>(hip_stream));)
}

// For the tests: where row i of a sequence stands, as the kernels take it.
void sdk_seq_rows(int32_t start, int32_t end, int32_t length, int32_t n, int32_t max_rows, int32_t *first, int32_t *m,
                  int32_t *past) {
    const SeqRows r = seq_rows(start, end, length, n, max_rows);
    *first = r.first;
    *m = r.m;
    *past = r.past;
}
int32_t sdk_seen_from(int32_t position, int32_t max_length) { return seen_from(position, max_length); }

}  // extern "C"
