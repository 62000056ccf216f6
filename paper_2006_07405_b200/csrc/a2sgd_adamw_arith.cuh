// The arithmetic of AdamW's step that is written out for pairs of elements: the codes of the 8-bit states, roots and
// quotients.  Apart from the kernels so that a test program can compare it with the single operations.
#pragma once

#include "a2sgd_train.cuh"

namespace a2sgd_train {

// The codes q of two s = (value / scale) * top^2, q in [0, top]: q = floor(sqrt(s)), plus one when s - q^2 > u (2q + 1), by
// the dither u in [0, 1).  Where the approximate root is an ulp off and picks the neighbour of the exact floor, s lies so close to a
// square that the second test gives the same sum: u ends at 4095/4096 (compared with the exact floor around every square, for
// every dither).  q^2, 2q + 1 and its product with u are exact.  u comes as 1 + u, 12 bits on top of a mantissa.
__device__ __forceinline__ void encode2(f32x2 s, uint32_t one_plus_u0, uint32_t one_plus_u1, float top, float least, float &q0, float &q1)
{
    float s0, s1, r0, r1;
    unpair(s, s0, s1);
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(s0));
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(s1));
    const f32x2 q = add2(add2_down(pair(r0, r1), pair(8388608.0f)), pair(-8388608.0f));
    const f32x2 over = fma2(mul2(q, pair(-1.0f)), q, s); // s - q^2
    const f32x2 u = add2(pair(__uint_as_float(one_plus_u0), __uint_as_float(one_plus_u1)), pair(-1.0f));
    const f32x2 limit = mul2(u, fma2(pair(2.0f), q, pair(1.0f)));
    float o0, o1, l0, l1;
    unpair(over, o0, o1);
    unpair(limit, l0, l1);
    unpair(q, q0, q1);
    if (o0 > l0) q0 += 1.0f;
    if (o1 > l1) q1 += 1.0f;
    q0 = fminf(q0, top);
    q1 = fminf(q1, top);
    if (least > 0.0f) {
        q0 = fmaxf(q0, least);
        q1 = fmaxf(q1, least);
    }
}

// sqrt(v) and m / d for two elements each, correctly rounded.  Within the range that `plain_range` tests this is
// Markstein's method (IBM J. Res. Dev. 34, 1990): an approximate root or reciprocal, and the exact residual by a fused
// multiply-add.  It has no special cases and runs on pairs; outside of the range the library functions are called.
// One correction alone does not prove the last bit (a root lies as close as 2^-26 of a unit to the middle between two numbers, the
// error is of the order of 2^-22): it rests on the device's approximations, and tests/test_gpu_adamw_arithmetic.py compares
// all mantissas of the roots, and the quotients nearest the middle for every divisor's mantissa, with the single operations: no difference.
__device__ __forceinline__ f32x2 root2(f32x2 v)
{
    float a, b, x, y;
    unpair(v, a, b);
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(a));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(b));
    const f32x2 y2 = pair(x, y), g = mul2(v, y2), h = mul2(y2, pair(0.5f));
    const f32x2 left = fma2(mul2(g, pair(-1.0f)), g, v); // v - g^2
    return fma2(left, h, g);
}
__device__ __forceinline__ f32x2 quotient2(f32x2 m, f32x2 d)
{
    float a, b, x, y;
    unpair(d, a, b);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(a));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(b));
    const f32x2 minus = mul2(d, pair(-1.0f));
    f32x2 y2 = pair(x, y);
    y2 = fma2(y2, fma2(minus, y2, pair(1.0f)), y2);
    const f32x2 q = mul2(m, y2);
    return fma2(fma2(minus, q, m), y2, q);
}
// v of a lane within least..2^80 and |m| up to 2^80; least is 2^-80 for eps up to 2^60 and lets nothing through beyond.  With a
// root's factor below 2^27, d = sqrt(v) root + eps lies between 2^-40 and 2^68, its reciprocal is a normal number, and no
// residual leaves the normal range but that of an m below 2^-100 or of a quotient below 2^-125, which may be an ulp off.
constexpr uint32_t kLeastPlain = 0x17800000u;           // 2^-80
constexpr double kMostPlainEps = 1152921504606846976.0; // 2^60
__device__ __forceinline__ bool plain_range(uint32_t least_v, uint32_t least, uint32_t largest_v, uint32_t largest_m)
{
    return least_v >= least && largest_v <= 0x67800000u && largest_m <= 0x67800000u;
}

} // namespace a2sgd_train
