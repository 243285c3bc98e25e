// The rotary form on the device (tree_ops.hip, paged_append.hip), and loads and
// stores of float32 and bfloat16 elements, which the operators share.
#pragma once

#include <cmath>

#include "sd.h"
#include "tree.h"

namespace sdk {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct RopeForm {
    // frequency of pair i: f = exp2(i * step), weighed for YARN, else times inv_factor
    double step, inv_factor, turns, beta_slow, inv_beta;
    float gain;
    int32_t half, interleaved, yarn;  // half: pairs of a head
};

inline double scaled_base(const sd_rope &r) {
    return r.scaling == SD_ROPE_NTK ? r.base * std::pow(r.factor, (double)r.rotary_dim / (r.rotary_dim - 2)) : r.base;
}

// The rotary part of the arguments, for a checked form.
inline void rope_form(const sd_rope &r, RopeForm *out) {
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

__device__ __forceinline__ float2 rope_turn(const RopeForm &a, int i, int pos) {
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
__device__ __forceinline__ f32x4_t load4(const uint16_t *p) {
    const u32x2_t x = *reinterpret_cast<const u32x2_t *>(p);
    return f32x4_t{__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), __uint_as_float(x[1] << 16),
                   __uint_as_float(x[1] & 0xffff0000u)};
}
__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store4(float *p, f32x4_t x) { *reinterpret_cast<f32x4_t *>(p) = x; }
__device__ __forceinline__ void store4(uint16_t *p, f32x4_t x) {
    *reinterpret_cast<u32x2_t *>(p) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
}
__device__ __forceinline__ void store1(float *p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t *p, float x) { *p = (uint16_t)pack_bf16(x, 0.0f); }

}  // namespace sdk
