// The step in front of the QKV and the gate+up projection of a decoder layer: residual stream, root-mean-square norm, and
// the activation quantisation of the projection behind it (Sec. 3.5, "Kernel Fusion"), one pass over the row.
//
//   s = bf16(x + r)          the new residual stream (r optional), stored
//   h = bf16((s w) rstd),    rstd = 1 / sqrt(mean(s^2) + eps)
//   (qa, sa, asum)           h quantised as w4a8_quantize_act does it
//
// One CTA per row.  A thread keeps its 16-byte chunks of s in registers.  s w is exact in fp32 (two 8-bit significands), so
// h = bf16(fl((s w) rstd)) is monotone in |s w| and the row's largest |h| is bf16(fl(max|s w| rstd)): the sum of squares and
// the maximum that the scale needs travel through one block reduction instead of two, and the codes are still exactly those
// of the quantiser on h.  The sum of squares is fp32 (per thread, then a tree); the one rounding of h to bf16 is the
// quantiser's input format, as after SiLU * up.
// HBM-bound for many rows (7 B per element with a residual, 3 without): 4096 rows of 5120 with a residual 31 us, 4.7 TB/s, CTAs whose loads
// and stores follow one another; for few rows a latency chain of load, reduction, store (one row of 4096: 2.4 us a launch in a chain).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "ptx_sm100.cuh"
#include "quant_common.cuh"
#include "w4a8_internal.cuh"

namespace w4a8 {
namespace {

__device__ __forceinline__ float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// two bf16 sums; an fp32 sum of two bf16 is exact or too far from a tie for its own rounding to matter
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
    return ptx::pack_bf16x2(lo_f(a) + lo_f(b), hi_f(a) + hi_f(b));
}

// sum of squares of s and largest |s w| of two elements
__device__ __forceinline__ void tally2(uint32_t s, uint32_t w, float& sq, float& top) {
    const float a = lo_f(s), b = hi_f(s);
    sq = fmaf(a, a, sq);
    sq = fmaf(b, b, sq);
    top = fmaxf(top, fmaxf(fabsf(__fmul_rn(a, lo_f(w))), fabsf(__fmul_rn(b, hi_f(w)))));
}
__device__ __forceinline__ uint32_t norm2(uint32_t s, uint32_t w, float rstd) {
    return ptx::pack_bf16x2(__fmul_rn(__fmul_rn(lo_f(s), lo_f(w)), rstd), __fmul_rn(__fmul_rn(hi_f(s), hi_f(w)), rstd));
}

// T threads per row, CACHE chunks of 8 elements per thread in registers (a longer row's rest is read again: from sum_out, which
// may have overwritten x or r).  Codes by the quantiser's reciprocal form (see quantize_act.cu).
template <int T, int CACHE, bool ADD>
__global__ void __launch_bounds__(T, T == 256 ? (CACHE <= 3 ? 5 : 3) : 1)
add_rmsnorm_quantize_kernel(const uint4* x, const uint4* r, const uint4* __restrict__ w, float eps, int K, uint4* sum_out, uint4* h_out,
                            uint2* __restrict__ qa, uint16_t* __restrict__ sa, int32_t* __restrict__ asum) {
    ptx::pdl_launch_dependents();
    const int m = blockIdx.x, tid = threadIdx.x;
    const int chunks = K >> 3, G = K >> 7;
    const size_t row = (size_t)m * chunks;
    ptx::pdl_wait();
    uint4 cache[CACHE];
    float sq = 0.0f, top = 0.0f;
    auto take = [&](int c, uint4 v, const uint4& o) -> uint4 {            // first sight of chunk c
        if (ADD) {
            v = make_uint4(add_bf16x2(v.x, o.x), add_bf16x2(v.y, o.y), add_bf16x2(v.z, o.z), add_bf16x2(v.w, o.w));
            sum_out[row + c] = v;
        }
        const uint4 g = __ldg(w + c);
        tally2(v.x, g.x, sq, top);
        tally2(v.y, g.y, sq, top);
        tally2(v.z, g.z, sq, top);
        tally2(v.w, g.w, sq, top);
        return v;
    };
    // all loads ahead of the first store: sum_out may be x or r, so the compiler keeps loads and stores in order
    uint4 other[ADD ? CACHE : 1];
#pragma unroll
    for (int i = 0; i < CACHE; ++i) {
        const int c = tid + i * T;
        if (c < chunks) {
            cache[i] = __ldcg(x + row + c);
            if (ADD) other[i] = __ldcg(r + row + c);
        }
    }
#pragma unroll
    for (int i = 0; i < CACHE; ++i) {
        const int c = tid + i * T;
        if (c < chunks) cache[i] = take(c, cache[i], other[ADD ? i : 0]);
    }
    for (int c = tid + CACHE * T; c < chunks; c += T) {
        const uint4 v = __ldcg(x + row + c), o = ADD ? __ldcg(r + row + c) : v;
        take(c, v, o);
    }

    // |s w| is not negative, so its bits order like unsigned integers
#pragma unroll
    for (int o = 16; o; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
    uint32_t mx = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top));
    if (T > 32) {
        __shared__ float2 part[T / 32];
        if ((tid & 31) == 0) part[tid >> 5] = make_float2(sq, __uint_as_float(mx));
        __syncthreads();
        sq = 0.0f;
#pragma unroll
        for (int i = 0; i < T / 32; ++i) {
            sq += part[i].x;
            mx = max(mx, __float_as_uint(part[i].y));
        }
    }
    const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sq, (float)K), eps)));
    const uint32_t amax = __bfloat16_as_ushort(__float2bfloat16_rn(__fmul_rn(__uint_as_float(mx), rstd)));
    const __half sh = row_scale_from_amax_bits(amax);
    const float s = __half2float(sh);
    if (tid == 0) sa[m] = __half_as_ushort(sh);
    const bool fast_row = fast_scale(__half_as_ushort(sh));
    const float rinv = s != 0.0f ? __frcp_rn(s) : 0.0f;

    // sixteen neighbouring chunks are one group of 128 and sit in the 16 lanes of one half-warp (see quantize_act_kernel)
    const uint32_t seg_mask = (tid & 16) ? 0xFFFF0000u : 0x0000FFFFu;
    auto emit = [&](int c, const uint4& v) {
        const uint4 g = __ldg(w + c);
        const uint4 h = make_uint4(norm2(v.x, g.x, rstd), norm2(v.y, g.y, rstd), norm2(v.z, g.z, rstd), norm2(v.w, g.w, rstd));
        if (h_out) h_out[row + c] = h;
        int sum = 0;
        uint2 o = make_uint2(0u, 0u);
        if (s != 0.0f) {
            float worst = 1.0f;
            if (fast_row) {
                worst = 0.0f;
                o.x = quant4_fast(h.x, h.y, rinv, worst);
                o.y = quant4_fast(h.z, h.w, rinv, worst);
                sum = __dp4a((int)o.x, 0x01010101, __dp4a((int)o.y, 0x01010101, 0));
            }
            if (worst > 0.5f - 0.0001220703125f) o = quant8(h, s, sum);
        }
        qa[row + c] = o;
        sum += __shfl_xor_sync(seg_mask, sum, 8);
        sum += __shfl_xor_sync(seg_mask, sum, 4);
        sum += __shfl_xor_sync(seg_mask, sum, 2);
        sum += __shfl_xor_sync(seg_mask, sum, 1);
        if ((c & 15) == 0) asum[(size_t)m * G + (c >> 4)] = sum;
    };
#pragma unroll
    for (int i = 0; i < CACHE; ++i) {
        const int c = tid + i * T;
        if (c < chunks) emit(c, cache[i]);
    }
    for (int c = tid + CACHE * T; c < chunks; c += T) emit(c, __ldcg((ADD ? sum_out : x) + row + c));
}

template <int T, int CACHE>
cudaError_t launch_norm(cudaLaunchConfig_t cfg, const uint4* x, const uint4* r, const uint4* w, float eps, int K, uint4* sum, uint4* h,
                        uint2* qa, uint16_t* sa, int32_t* asum) {
    cfg.blockDim = dim3(T, 1, 1);
    if (r) return cudaLaunchKernelEx(&cfg, add_rmsnorm_quantize_kernel<T, CACHE, true>, x, r, w, eps, K, sum, h, qa, sa, asum);
    return cudaLaunchKernelEx(&cfg, add_rmsnorm_quantize_kernel<T, CACHE, false>, x, r, w, eps, K, sum, h, qa, sa, asum);
}

}  // namespace

cudaError_t launch_add_rmsnorm_quantize(const void* x, const void* residual, const void* weight, float eps, int M, int K, void* sum_out,
                                        void* h_out, int8_t* qa, uint16_t* sa, int32_t* asum, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)M, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const uint4 *xp = static_cast<const uint4*>(x), *rp = static_cast<const uint4*>(residual), *wp = static_cast<const uint4*>(weight);
    uint4 *sp = static_cast<uint4*>(sum_out), *hp = static_cast<uint4*>(h_out);
    uint2* qp = reinterpret_cast<uint2*>(qa);
    // Threads per row by the row's length, so that it fits their registers.  Up to 256 rows twice as many threads where 256 would hold more than one chunk of a
    // short row or three of a long one (200 rows of 4096: 3.7 against 4.4 us, of 8192 5.6 against 6.3; from 500 rows on the wider CTAs are slower,
    // 500 of 4096 6.6 against 6.0, 4096 of 5120 53 against 31).  Rows of 1024 with 256 threads: 4096 of them 12.5 instead of 8.5 us.
    if (K <= 1024) return launch_norm<128, 1>(cfg, xp, rp, wp, eps, K, sp, hp, qp, sa, asum);
    if (M <= 256 && K > 2048 && K <= 4096) return launch_norm<512, 1>(cfg, xp, rp, wp, eps, K, sp, hp, qp, sa, asum);
    if (M <= 256 && K > 6144) return launch_norm<512, 3>(cfg, xp, rp, wp, eps, K, sp, hp, qp, sa, asum);
    if (K <= 4096) return launch_norm<256, 2>(cfg, xp, rp, wp, eps, K, sp, hp, qp, sa, asum);
    if (K <= 6144) return launch_norm<256, 3>(cfg, xp, rp, wp, eps, K, sp, hp, qp, sa, asum);
    return launch_norm<256, 6>(cfg, xp, rp, wp, eps, K, sp, hp, qp, sa, asum);
}

}  // namespace w4a8
