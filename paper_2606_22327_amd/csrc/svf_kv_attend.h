// svf_kv_attend.h -- what the attention kernels of the paged cache share.
#pragma once

#include "svf_kv_device.h"

namespace svfk {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Sixteen 16-bit elements' worth of a matrix product, and the type's constants.
// kShift: probabilities are scaled by 2^kShift, which cancels against their sum: float16's up, so that the
// small ones stay above its subnormal numbers, bfloat16's down, so that sums of values as large as the
// type has stay finite in 32 bits before they are divided (2^24 of them with kSlack).
// kSlack: powers of two by which a row's scores may pass the maximum that its
// probabilities are taken against before the row's sums are scaled down to a new one.
struct BF16M : BF16 {
    static constexpr float kShift = -32.f, kUnshift = 4294967296.f;
    static constexpr uint16_t kInf = 0x7f80;
    static constexpr float kSlack = 8.f;
    // Two numbers, each as the sum of two of the type, as words of two: the upper 16 bits of each, and what is left, rounded.
    static __device__ inline void split(float a, float b, uint32_t& hi, uint32_t& low) {
        typedef __bf16 V2 __attribute__((ext_vector_type(2)));
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        hi = __builtin_amdgcn_perm(y, x, 0x07060302u);
        low = __builtin_bit_cast(uint32_t, V2{(__bf16)(a - __uint_as_float(x & 0xffff0000u)), (__bf16)(b - __uint_as_float(y & 0xffff0000u))});
    }
    static __device__ inline f32x4 mfma16(V8 a, V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ inline f32x16 mfma32(V8 a, V8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F16M : F16 {
    static constexpr float kShift = 14.f, kUnshift = 1.f / 16384.f;
    static constexpr uint16_t kInf = 0x7c00;
    static constexpr float kSlack = 1.f;
    static __device__ inline void split(float a, float b, uint32_t& hi, uint32_t& low) {
        const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
        hi = __builtin_bit_cast(uint32_t, h);
        low = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a - (float)h.x, b - (float)h.y));
    }
    static __device__ inline f32x4 mfma16(V8 a, V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ inline f32x16 mfma32(V8 a, V8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// The largest of three (the compiler's own first quiets every operand).
__device__ inline float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two elements in a word: whether one of them is no finite number; the word with zeros in the place of such; and
// two bits for each, the first for +infinity, the second for -infinity, both for no number.
template <class E>
__device__ inline bool odd_pair(uint32_t w) {
    return (w & E::kInf) == E::kInf || (w >> 16 & E::kInf) == E::kInf;
}
template <class E>
__device__ inline uint32_t finite_pair(uint32_t w) {
    if ((w & E::kInf) == E::kInf) w &= 0xffff0000u;
    if ((w >> 16 & E::kInf) == E::kInf) w &= 0x0000ffffu;
    return w;
}
template <class E>
__device__ inline uint32_t odd_marks_of(uint32_t w) {
    uint32_t marks = 0;
    for (int i = 0; i < 2; i++) {
        const uint32_t b = w >> 16 * i & 0xffff;
        if ((b & E::kInf) == E::kInf) marks |= ((b & 0x7fff) != E::kInf ? 3u : b & 0x8000 ? 2u : 1u) << 2 * i;
    }
    return marks;
}
// n sums of which some have marks: what those are, whatever is added to it.
__device__ inline void set_marked(uint32_t marks, float* acc, int n) {
    if (marks == 0) return;
    for (int i = 0; i < n; i++) {
        const uint32_t m = marks >> 2 * i & 3;
        if (m) acc[i] = m == 1 ? INFINITY : m == 2 ? -INFINITY : __builtin_nanf("");
    }
}

// A part's sum by the part's factor.  One that marked values decide stays, also where the factor has become 0.
__device__ inline float scaled(float x, float f) { return fabsf(x) == INFINITY ? x : x * f; }

// The first slot that any row of the sequence sees, or one of the fifteen before it: pages of 16 slots and more
// are read from a multiple of 16.
__device__ inline int first_slot(const AttendArgs& p, const Seq& s) {
    return p.window > 0 ? max(0, s.len - s.n - p.window + 1) & ~15 : 0;
}

// The slots that some row sees, one behind the other: place x is slot x below ``head`` and slot x + skip from there on.
// With first tokens that stay visible (FIRST) ``head`` is their number rounded up to ``unit``, so that what takes
// ``unit`` places at a time never has slots of both sides; 0 where the window begins before its end.
struct Line {
    int head, skip, places;
};
template <bool FIRST>
__device__ inline Line line_of(const AttendArgs& p, const Seq& s, int unit) {
    Line x;
    x.head = FIRST ? (p.first + unit - 1) & ~(unit - 1) : 0;
    x.skip = first_slot(p, s) - x.head;
    if (FIRST && x.skip <= 0) x.head = x.skip = 0;
    x.places = s.len - x.skip;
    return x;
}
template <bool FIRST>
__device__ inline int slot_of(const Line& x, int place) {
    return FIRST && place < x.head ? place : place + x.skip;
}

// Where a lane reads a slot that is not there: a row of zeros, so that loads need no branch.
static __device__ __align__(16) const char kZeroRow[512] = {};
__device__ inline const char* zero_row() { return kZeroRow; }

// KS operands of a row's query: dimensions k * 32 + g * 8 and the seven behind.
template <class E, int KS>
__device__ inline void load_query(typename E::V8* q, const char* at, int g, bool valid, bool wide) {
    using T = typename E::T;
#pragma unroll
    for (int k = 0; k < KS; k++) {
        if (!valid) {
#pragma unroll
            for (int i = 0; i < 8; i++) q[k][i] = (T)0.f;
        } else if (wide) {
            q[k] = *(const typename E::V8*)(at + (k * 32 + g * 8) * 2);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) q[k][i] = *(const T*)(at + (k * 32 + g * 8 + i) * 2);
        }
    }
}

// N of a row's dimensions from d0: the sums over the softmax's denominator, rounded once, and with the
// first of them the row's statistic.  A row without a probability has zeros, whatever its values.
template <class E, int N>
__device__ inline void write_row(const AttendArgs& p, int token, int h, int d0, const float* acc, float den, float top) {
    using T = typename E::T;
    typedef T V __attribute__((ext_vector_type(N)));
    const float inv = 1.f / den;
    V v;
#pragma unroll
    for (int j = 0; j < N; j++) v[j] = (T)(den == 0.f ? 0.f : acc[j] * inv);
    *(V*)(p.out + token * p.o_tok + h * p.o_head + d0 * 2) = v;
    if (d0 == 0) p.lse[(int64_t)token * p.heads + h] = (top + __builtin_amdgcn_logf(den * E::kUnshift)) * 0.69314718055994531f;
}

// Rows of one key head of a sequence that has more new tokens than it may.
template <class T, int D>
__device__ inline void fill_nan(const AttendArgs& p, const Seq& s, int head, int G, int tid, int threads) {
    const T nan = (T)__builtin_nanf("");
    for (int64_t i = tid; i < (int64_t)s.n * G * D; i += threads) {
        const int row = (int)(i / D), d = (int)(i - (int64_t)row * D), t = row / G, h = head * G + row - t * G;
        *(T*)(p.out + (s.q0 + t) * p.o_tok + h * p.o_head + d * 2) = nan;
        if (d == 0) p.lse[(int64_t)(s.q0 + t) * p.heads + h] = __builtin_nanf("");
    }
}

}  // namespace svfk
