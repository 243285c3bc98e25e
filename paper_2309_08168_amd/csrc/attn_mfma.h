// What the attention kernels on matrix cores share (tree_attention.hip,
// batch_attention.hip): bfloat16 terms, products, loads to LDS and where rows lie there.
#pragma once

#include "rope.h"
#include "sd_internal.h"

namespace sdk {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Two packed bfloat16 values, zero for those that are infinite or NaN.
__device__ __forceinline__ uint32_t without_odd(uint32_t x) {
    const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
    return x & (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
}

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

}  // namespace sdk
