// Device helpers shared by the kernels that quantise activations (Sec. 3.4) and by the two forms of the
// SiLU(gate) * up step that follows the fused gate+up projection (Sec. 3.5, "Kernel Fusion"): every kernel that
// produces a code or an h value goes through these, so that the forms agree bit for bit.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace w4a8 {

// s_a = fp16_rne(min(amax / 127, 65504)) from the largest magnitude of a row, given as bf16 bits (15-bit pattern)
__device__ __forceinline__ __half row_scale_from_amax_bits(uint32_t amax_bf16_bits) {
    const float amax = __uint_as_float(amax_bf16_bits << 16);
    return __float2half_rn(fminf(__fdiv_rn(amax, 127.0f), 65504.0f));
}

// one code: rne(x / s) by IEEE division, clamped to [-127, 127]; x given as bf16 bits in the upper half of a word
__device__ __forceinline__ int quant1(uint32_t bf16_hi_bits, float s) {
    float q = __fdiv_rn(__uint_as_float(bf16_hi_bits), s);
    int r;
    asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(r) : "f"(q));   // ties to even, saturates to [-128,127]
    return max(r, -127);
}

// largest magnitudes of a 16-byte chunk (8 bf16), two lanes of a word at a time
__device__ __forceinline__ uint32_t absmax_bits_bf16x8(const uint4& v, uint32_t run) {
    // bf16 magnitudes order like their 15-bit patterns: keep a packed running max of two lanes
    run = __vmaxu2(run, v.x & 0x7FFF7FFFu);
    run = __vmaxu2(run, v.y & 0x7FFF7FFFu);
    run = __vmaxu2(run, v.z & 0x7FFF7FFFu);
    run = __vmaxu2(run, v.w & 0x7FFF7FFFu);
    return run;
}

__device__ __forceinline__ uint2 quant8(const uint4& v, float s, int& sum) {
    int q0 = quant1(v.x << 16, s), q1 = quant1(v.x & 0xFFFF0000u, s);
    int q2 = quant1(v.y << 16, s), q3 = quant1(v.y & 0xFFFF0000u, s);
    int q4 = quant1(v.z << 16, s), q5 = quant1(v.z & 0xFFFF0000u, s);
    int q6 = quant1(v.w << 16, s), q7 = quant1(v.w & 0xFFFF0000u, s);
    sum = q0 + q1 + q2 + q3 + q4 + q5 + q6 + q7;
    uint2 o;
    o.x = (q0 & 0xFF) | ((q1 & 0xFF) << 8) | ((q2 & 0xFF) << 16) | ((uint32_t)q3 << 24);
    o.y = (q4 & 0xFF) | ((q5 & 0xFF) << 8) | ((q6 & 0xFF) << 16) | ((uint32_t)q7 << 24);
    return o;
}

// The scales (fp16 bits) for which codes may be formed by the reciprocal, which has no clamp and so needs |x / s| < 127.5 - 2^-13 (products are
// within 2^-16 of their quotients).  From 2^-14 on s is amax / 127 but for a factor of 1 +- 2^-11: |x / s| < 127.1.  Below, s = n 2^-24 with amax / 127 at most
// (n + 1/2) 2^-24: |x / s| <= 127 + 63.5 / n, which is 127.4961 for n = 128 and more from there down to 190.5 for n = 1.  At the other end a scale
// that saturated at 65504 bounds nothing.  A scale taken from older values as well (the append's) is larger, its quotients smaller.
// (With the division 4096 rows of 5120 take the norm 31.1 instead of 25.7 us, one row of 4096 2.5 instead of 2.3.)
constexpr uint32_t FAST_SCALE_FIRST = 0x0080u, FAST_SCALE_END = 0x7BFFu;
__device__ __forceinline__ bool fast_scale(uint32_t fp16_bits) {
    return fp16_bits >= FAST_SCALE_FIRST && fp16_bits < FAST_SCALE_END;
}

// Fast path of a chunk (see quantize_act.cu): products with the row's reciprocal scale.  `worst` returns the largest
// distance of a product from the integer it was rounded to.  For rows whose scale satisfies fast_scale.
__device__ __forceinline__ uint32_t quant4_fast(uint32_t lo_pair, uint32_t hi_pair, float rinv, float& worst) {
    constexpr float MAGIC = 12582912.0f;                     // 1.5 * 2^23: adding it rounds to an integer, ties to even
    const float t0 = __fmul_rn(__uint_as_float(lo_pair << 16), rinv), t1 = __fmul_rn(__uint_as_float(lo_pair & 0xFFFF0000u), rinv);
    const float t2 = __fmul_rn(__uint_as_float(hi_pair << 16), rinv), t3 = __fmul_rn(__uint_as_float(hi_pair & 0xFFFF0000u), rinv);
    const float y0 = __fadd_rn(t0, MAGIC), y1 = __fadd_rn(t1, MAGIC), y2 = __fadd_rn(t2, MAGIC), y3 = __fadd_rn(t3, MAGIC);
    worst = fmaxf(worst, fmaxf(fmaxf(fabsf(__fsub_rn(t0, __fsub_rn(y0, MAGIC))), fabsf(__fsub_rn(t1, __fsub_rn(y1, MAGIC)))),
                               fmaxf(fabsf(__fsub_rn(t2, __fsub_rn(y2, MAGIC))), fabsf(__fsub_rn(t3, __fsub_rn(y3, MAGIC))))));
    // low mantissa bytes of y0..y3 -> one word
    const uint32_t a = __byte_perm(__float_as_uint(y0), __float_as_uint(y1), 0x0040);
    const uint32_t b = __byte_perm(__float_as_uint(y2), __float_as_uint(y3), 0x0040);
    return __byte_perm(a, b, 0x5410);
}

// h = bf16_rne(SiLU(g) * u) in fp32, g and u bf16 values: g / (1 + e^-g) * u with the fast exponential and
// division (a few fp32 ulps from the exact value: the rounded h equals the exactly computed one or its bf16
// neighbour; far out on the negative side, where e^-g overflows, the result is a signed zero like the limit).
__device__ __forceinline__ uint32_t silu_mul_bf16_bits(float g, float u) {
    const float h = __fmul_rn(__fdividef(g, 1.0f + __expf(-g)), u);
    return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(h));
}

// two h values from packed pairs of bf16 (low half = even element), result packed the same way
__device__ __forceinline__ uint32_t silu_mul_bf16x2(uint32_t g2, uint32_t u2) {
    const uint32_t lo = silu_mul_bf16_bits(__uint_as_float(g2 << 16), __uint_as_float(u2 << 16));
    const uint32_t hi = silu_mul_bf16_bits(__uint_as_float(g2 & 0xFFFF0000u), __uint_as_float(u2 & 0xFFFF0000u));
    return lo | (hi << 16);
}

}  // namespace w4a8
