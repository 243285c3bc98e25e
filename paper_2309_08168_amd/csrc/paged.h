// What the operators of batches (paged_append.hip, batch_attention.hip) share:
// where the rows of a call stand, and the checks of its arguments.
#pragma once

#include <hip/hip_runtime.h>

#include "sd.h"
#include "tree.h"

namespace sdk {

constexpr int32_t MAX_SEQS = 65536, MAX_BATCH_ROWS = 1 << 20, MAX_PAGE = 65536, MAX_POSITIONS = 1 << 30;
constexpr int32_t MAX_QUERY_HEADS = 4096;

// The rows of a sequence: row i is packed row `first` + i and stands at position
// past + i.  m counts those that the call takes (at most max_rows).
struct SeqRows {
    int32_t first, m, past;
};

// From what starts and lengths hold, whatever that is: rows within [0, n),
// positions within 32 bits.
__host__ __device__ inline SeqRows seq_rows(int32_t start, int32_t end, int32_t length, int32_t n, int32_t max_rows) {
    SeqRows r;
    r.first = start < 0 ? 0 : start > n ? n : start;
    const int32_t e = end < r.first ? r.first : end > n ? n : end;
    const int32_t len = length < 0 ? 0 : length > MAX_POSITIONS ? MAX_POSITIONS : length;
    r.past = len - (e - r.first);
    r.m = e - r.first < max_rows ? e - r.first : max_rows;
    return r;
}

// Positions 0 .. that the row at a position sees.
__host__ __device__ inline int32_t seen_from(int32_t position, int32_t max_length) {
    return position < 0 ? 0 : position < max_length ? position + 1 : max_length;
}

#ifdef __HIPCC__
// How many of j = 1 .. count have at(j) <= x, for at that does not fall: a wave
// looks at 64 of them at a time.  (Whatever at gives, it ends, within [0, count].)
template <typename F>
__device__ __forceinline__ int32_t wave_count(int32_t count, int64_t x, F at) {
    const int lane = threadIdx.x & 63;
    int32_t lo = 0, hi = count;
    while (lo < hi) {
        const int32_t step = (hi - lo + 63) >> 6, j = lo + (lane + 1) * step;
        const bool below = j <= hi && at(j) <= x;
        const int32_t t = __popcll(__ballot(below));
        lo += t * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}
#endif

// Refuses pages and batches that break the rules of sd_kv_pages and sd_batch.
sd_status check_pages(const sd_kv_pages *kv);
// addresses: whether the batch's pointers are checked too.
sd_status check_batch(const sd_batch *batch, const sd_kv_pages *kv, int32_t n, bool addresses);
// The rows and heads of a call on n_kv_heads.
sd_status check_rows(int32_t n, int32_t n_heads, int32_t n_kv_heads);

// Positions that a checked batch takes.
inline int32_t positions_of(const sd_batch &b, const sd_kv_pages &kv) {
    return b.max_length ? b.max_length : b.table_pages * kv.page_size;
}

inline int log2_of(int32_t x) {
    int s = 0;
    while ((1 << s) < x)
        ++s;
    return s;
}

}  // namespace sdk
