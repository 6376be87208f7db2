// What the two attention kernels over the 8-bit cache share: arguments, the plan, the number formats.
//
//   out[t,h,:] = sum_j p_j sv_j v_j / sum_j p_j,   p_j = exp(scale q . (sk_j k_j)),  j < limit[t]
//
// with codes k_j, v_j in -127..127 and scales sk_j, sv_j of the block that holds position j.
//
// Codes become fp16 exactly (1024 + code + 128 is a byte under the exponent of 1024; one subtraction), so the products run as fp16
// tensor-core products with fp32 sums:
//   * a row of q is brought to fp16 by a power of two, its largest element to [2^14, 2^15): elements down to 2^-31 of the largest
//     keep all eight bits;
//   * the scores are worked in base 2:  x_j = (scale log2(e) 2^-e sk_j) (q' . k_j);
//   * the scale of a value's block goes into the exponent:  w_j = 2^(x_j + log2 sv_j - m + 7), an fp16 number of at most 2^15 whose
//     size is the key's weight in the OUTPUT relative to the largest so far; the sum of the p is sum_j w_j / sv_j in fp32 (of
//     the values before they are rounded to fp16).  m is a reference, not the maximum: it moves only when a weight
//     would pass 2^15 (256 times the reference), so sums are rescaled a few times per row, not per tile.
//     fp16 keeps 11 bits of weights down to 2^-21 of the reference, bf16 would keep 8 of all.
// A row of q with an infinity or not-a-number is one that both kernels mark where they form its power of two: its products alone may all be minus
// infinity, which is what masked positions have.
// A block of scale 0 holds zeros; 2^-80 stands for its scale (weights end at 2^-126, 2^-46 in the sum of the p, which is 2^7 / 65504 at least; and
// weights beside it are lost only below 2^-100 of its own).
#pragma once
#include <cuda_fp16.h>
#include <math.h>
#include "ptx_sm100.cuh"
#include "w4a8_internal.cuh"

namespace w4a8 {

struct AttendArgs {
    const int8_t *k_codes, *v_codes;
    const uint16_t *k_scales, *v_scales;
    const uint16_t* q;                  // bf16
    long long q_stride;                 // elements from one token to the next
    const int32_t *table, *limits;
    uint16_t* out;                      // bf16 [B T][q_heads dim]
    float* part_o;                      // partial sums of key slices: [unit][slice][row][dim], and [unit][slice][row] (m, l)
    float2* part_ml;
    uint32_t* status;
    int T, q_heads, kv_heads, rep;      // rep = q_heads / kv_heads; a row is (token, head of the group): row = token rep + r
    int table_width, num_blocks, log2_block;
    int tiles, slices;                  // row tiles per (sequence, key head); key slices per row tile
    float scale_log2;                   // scale log2(e)
};

constexpr float KV8_W_EXP = 7.0f;       // weights are 2^7 at the reference
constexpr float KV8_SLACK = 8.0f;       // ... and the reference moves when one is past 2^8 times that
constexpr float KV8_ZERO_LOG2 = -80.0f;

// two codes of a word (bytes `sel`) as fp16; w = four codes with their sign bits flipped
__device__ __forceinline__ uint32_t kv8_half2(uint32_t biased, uint32_t sel) {
    const uint32_t h = __byte_perm(biased, 0x64646464u, sel);
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(0x64806480u));      // 1024 + 128
    return r;
}

__device__ __forceinline__ float kv8_ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float kv8_lg2(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// log2 of a value scale and the reciprocal of the scale that this logarithm stands for
__device__ __forceinline__ void kv8_value_scale(uint32_t bits, float& lg, float& inv) {
    const float s = __half2float(__ushort_as_half((uint16_t)bits));
    lg = s > 0.0f ? kv8_lg2(s) : KV8_ZERO_LOG2;
    inv = kv8_ex2(-lg);
}
// exponent that brings a row whose largest magnitude has these bf16 bits to [2^14, 2^15); 0 for zero, infinity and NaN
__device__ __forceinline__ int kv8_row_exp(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 7);
    return e == 0 || e == 255 ? 0 : min(14 - (e - 127), 100);
}
__device__ __forceinline__ float kv8_pow2(int e) {           // e in -126..127
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ uint32_t kv8_pack_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Which kernel, how many rows per tile and how many slices of the keys.
struct Kv8Plan {
    int rows;                           // rows per tile: 16, 32, or TC_ROWS for the tensor-memory kernel
    int tiles, slices;
};
Kv8Plan kv8_plan(int B, int T, int q_heads, int kv_heads, long long max_keys, int sms);

cudaError_t launch_kv8_tiles(const AttendArgs& a, int B, int dim, cudaStream_t stream);      // 256 rows per tile

}  // namespace w4a8
