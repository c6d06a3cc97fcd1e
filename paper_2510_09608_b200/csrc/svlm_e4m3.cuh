// 8-bit floats (e4m3) in device code: conversions and the exponent of a block.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace {

constexpr int E8_MIN = -100, E8_MAX = 120;      // of a block's exponent: the lower end is all zeros', the upper bf16's largest value's
constexpr float E8_TOP = 240.f;                 // the largest value in units of 2^E8_MAX (the next one, 256, would be 2^128)

__device__ __forceinline__ float pow2i(int e) { return __int_as_float((127 + e) << 23); }      // -126 <= e <= 127

constexpr unsigned NO_EXPONENTS = (unsigned)(E8_MIN & 255) * 0x101u;     // of a block that holds nothing

// Of a block's keys (0) or values (1).
__device__ __forceinline__ int exponent_of(unsigned exps, int which) { return (int)(exps << (24 - 8 * which)) >> 24; }

// Magnitude of x as an ordered integer, 0 for what is not finite.
__device__ __forceinline__ unsigned finite_bits(float x) {
    const unsigned b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
// The least e with x <= 448 * 2^e, 448 = 1.75 * 2^8, of a magnitude given by its bits.
__device__ __forceinline__ int block_exponent(unsigned bits) {
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return bits == 0 ? E8_MIN : max(E8_MIN, min(E8_MAX, e));
}
// Two values as two bytes, lo in the lower one: round to nearest even, limit at most, NaN for what is not finite.
__device__ __forceinline__ uint16_t to_e4m3x2(float lo, float hi, float limit = 448.f) {
    const float nan = __int_as_float(0x7fffffff);
    lo = (__float_as_uint(lo) & 0x7fffffffu) < 0x7f800000u ? fminf(fmaxf(lo, -limit), limit) : nan;      // (the conversion would turn an infinity into 448)
    hi = (__float_as_uint(hi) & 0x7fffffffu) < 0x7f800000u ? fminf(fmaxf(hi, -limit), limit) : nan;
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Of a word's four bytes those that are NaN (0x7f, 0xff): their lowest bits.
__device__ __forceinline__ unsigned nan_bytes(unsigned w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7; }
// Two bytes as two halves (exact).
__device__ __forceinline__ unsigned e4m3x2_to_half2(uint16_t x) {
    unsigned r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(x));
    return r;
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint16_t x) {
    const unsigned h = e4m3x2_to_half2(x);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// (cos, sin)(c * theta) rounded to fp32 once, from a table in fp64 (svlm_rope.cuh's, not rounded), and a pair rotated by it, each
// operation rounded by itself.  What is rounded to three mantissa bits behind this jumps by a sixteenth where it lies on a boundary: a key that
// decides a row's softmax then changes the row visibly.  So the bytes do not hang on how the factors were put together.  (With fp32 products of
// table entries one output of a chunk of 28 layers was off by 0.88 once; this way none of twelve such chunks by more than 0.06.)
__device__ __forceinline__ float2 rope_cs_exact(const double2* tab, int half, int pair, long long c, double theta) {
    const unsigned long long a = c < 0 ? (unsigned long long)(-c) : (unsigned long long)c;
    double2 r;
    if (a < (1ull << 24)) {
        r = __ldg(tab + (size_t)(a & 255u) * half + pair);
        auto times = [&](const double2& f) { r = make_double2(r.x * f.x - r.y * f.y, r.x * f.y + r.y * f.x); };
        if (a >> 8) times(__ldg(tab + (size_t)(256 + ((a >> 8) & 255u)) * half + pair));
        if (a >> 16) times(__ldg(tab + (size_t)(512 + (a >> 16)) * half + pair));
    } else {
        sincos((double)a * theta, &r.y, &r.x);
    }
    return make_float2((float)r.x, c < 0 ? -(float)r.y : (float)r.y);
}
__device__ __forceinline__ void rotate_exact(float& lo, float& hi, const float2& f) {
    const float x = lo, y = hi;
    lo = __fsub_rn(__fmul_rn(x, f.x), __fmul_rn(y, f.y));
    hi = __fadd_rn(__fmul_rn(y, f.x), __fmul_rn(x, f.y));
}

}  // namespace
