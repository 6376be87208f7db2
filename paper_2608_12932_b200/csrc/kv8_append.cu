// Appends keys and values to a cache held in 8 bits with one scale per block of tokens and head (the decoder layer's step
// between the QKV projection and attention).
//
// A block's codes are value / scale, so tokens that join a block whose scale is too small for them raise it, and the codes
// that were there are rounded anew:  s' = max(s, fp16(amax_new / 127)),  q' = rne(q s / s').  q s is exact in fp32 (7 + 11 bits)
// and a quotient of it by an fp16 value is an exact tie or too far from one for fp32 division to matter (at least 2^-(12+d) with
// d the scales' distance in octaves, against half an fp32 step of at most 2^-(17+d)): the codes are those of exact arithmetic.
//
// One CTA per (sequence, touched block, head) and for K and V apart: it owns all that it reads and writes of the cache.
// For single tokens a latency chain (position, new values and table, scale, reduction, store): 2.0 us a launch in a chain.  A chunk moves 2 B in and 1 B
// out per element, but is over before the chain has paid for itself: 1391 tokens of 8 heads x 128 in blocks of 128 5.3 us, 1.6 TB/s.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "ptx_sm100.cuh"
#include "quant_common.cuh"
#include "w4a8_internal.cuh"

namespace w4a8 {
namespace {

constexpr int APPEND_FEW = 128, APPEND_MANY = 512;           // threads per CTA

struct AppendArgs {
    const uint4 *k, *v;
    long long k_stride, v_stride;       // 16-byte pieces from one token to the next
    int T, heads, pieces, log2_block;   // pieces: 16-byte pieces (8 elements) of a head's row
    const int32_t *table, *start, *count;
    int table_width, num_blocks;
    int8_t *k_codes, *v_codes;
    uint16_t *k_scales, *v_scales;
    uint32_t* status;
};

__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float s_old, float s_new) {
    uint32_t o = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float q = (float)(int8_t)(codes >> (8 * i));
        int r;
        asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(r) : "f"(__fdiv_rn(__fmul_rn(q, s_old), s_new)));
        o |= ((uint32_t)r & 0xFFu) << (8 * i);
    }
    return o;
}

// THREADS per CTA, CH 16-byte pieces of new values per thread
template <int THREADS, int CH>
__global__ void __launch_bounds__(THREADS)
kv8_append_kernel(const AppendArgs a) {
    ptx::pdl_launch_dependents();
    const int tid = threadIdx.x, seq = blockIdx.z, head = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const int block = 1 << a.log2_block;
    ptx::pdl_wait();
    const int start = __ldcg(a.start + seq);
    int count = a.T;
    if (a.count) count = min(max(__ldcg(a.count + seq), 0), a.T);
    if (start < 0) {
        if (count > 0 && tid == 0) flag_index(a.status);
        return;
    }
    const long long end = (long long)start + count;
    const long long index = (long long)(start >> a.log2_block) + blockIdx.x;          // the block's place in the table
    const long long first = index << a.log2_block;
    if (first >= end || count == 0) return;
    const int lo = (int)(max((long long)start, first) - first), hi = (int)(min(end, first + block) - first);     // slots of the new tokens
    const int number = index < a.table_width ? __ldcg(a.table + (size_t)seq * a.table_width + index) : -1;
    const long long stride = is_v ? a.v_stride : a.k_stride;
    // token of slot j: (seq T + first + j - start)
    const uint4* src = (is_v ? a.v : a.k) + ((long long)seq * a.T + first - start) * stride + (long long)head * a.pieces;
    const int n_lo = lo * a.pieces, n_hi = hi * a.pieces;
    const int log2_pieces = a.pieces == 16 ? 4 : 3;
    uint4 x[CH];
    uint32_t run = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int p = n_lo + tid + i * THREADS;
        if (p < n_hi) x[i] = __ldcg(src + (long long)(p >> log2_pieces) * stride + (p & (a.pieces - 1)));
    }
    // (the new values are on their way while the table is read, and the old scale)
    if ((unsigned)number >= (unsigned)a.num_blocks) {
        if (tid == 0) flag_index(a.status);
        return;
    }
    const size_t at = (size_t)number * a.heads + head;
    const size_t codes_at = at * (size_t)(block * a.pieces);                            // in pieces of 8 codes
    uint2* codes = reinterpret_cast<uint2*>(is_v ? a.v_codes : a.k_codes) + codes_at;
    uint16_t* scale = (is_v ? a.v_scales : a.k_scales) + at;
    const uint32_t old_bits = lo > 0 ? (uint32_t)__ldcg(scale) : 0u;
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (n_lo + tid + i * THREADS < n_hi) run = absmax_bits_bf16x8(x[i], run);
    uint32_t mx = __reduce_max_sync(0xFFFFFFFFu, max(run & 0xFFFFu, run >> 16));
    __shared__ uint32_t warp_max[THREADS / 32];
    if ((tid & 31) == 0) warp_max[tid >> 5] = mx;
    __syncthreads();                                         // every thread has read the old scale, too
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) mx = max(mx, warp_max[i]);
    // scales are not negative: their bits order like their values
    const uint32_t bits = max((uint32_t)__half_as_ushort(row_scale_from_amax_bits(mx)), old_bits);
    const float s = __half2float(__ushort_as_half((uint16_t)bits));
    if (bits != old_bits) {
        const float s_old = __half2float(__ushort_as_half((uint16_t)old_bits));
        for (int p = tid; p < n_lo; p += THREADS) {
            const uint2 q = codes[p];
            codes[p] = make_uint2(rescale4(q.x, s_old, s), rescale4(q.y, s_old, s));
        }
    }
    if (tid == 0) *scale = (uint16_t)bits;
    const bool fast = fast_scale(bits);
    const float rinv = s != 0.0f ? __frcp_rn(s) : 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int p = n_lo + tid + i * THREADS;
        if (p >= n_hi) continue;
        uint2 o = make_uint2(0u, 0u);
        if (s != 0.0f) {
            float worst = 1.0f;
            int sum;
            if (fast) {
                worst = 0.0f;
                o.x = quant4_fast(x[i].x, x[i].y, rinv, worst);
                o.y = quant4_fast(x[i].z, x[i].w, rinv, worst);
            }
            if (worst > 0.5f - 0.0001220703125f) o = quant8(x[i], s, sum);
        }
        codes[p] = o;
    }
}

}  // namespace

cudaError_t launch_kv8_append(const w4a8_kv8_cache& c, const void* k, const void* v, long long k_stride, long long v_stride, int B, int T,
                              const int32_t* table, int table_width, const int32_t* start, const int32_t* count, uint32_t* status,
                              cudaStream_t stream) {
    AppendArgs a;
    a.k = static_cast<const uint4*>(k);
    a.v = static_cast<const uint4*>(v);
    a.k_stride = k_stride / 8;
    a.v_stride = v_stride / 8;
    a.T = T;
    a.heads = c.heads;
    a.pieces = c.dim / 8;
    a.log2_block = kv8_log2(c.block);
    a.table = table;
    a.start = start;
    a.count = count;
    a.table_width = table_width;
    a.num_blocks = c.num_blocks;
    a.k_codes = c.k_codes;
    a.v_codes = c.v_codes;
    a.k_scales = c.k_scales;
    a.v_scales = c.v_scales;
    a.status = status;
    cudaLaunchConfig_t cfg = {};
    // a run of T tokens touches at most this many blocks, wherever it starts
    cfg.gridDim = dim3((unsigned)(((long long)T + c.block - 2) / c.block + 1), (unsigned)(2 * c.heads), (unsigned)B);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const int most = (T < c.block ? T : c.block) * a.pieces;                     // pieces of new values in one block
    // (128 threads for large blocks: 5.6 instead of 5.3 us above; 512 for few new tokens: 40 of them 3.2 instead of 2.0)
    const int threads = most > 2 * APPEND_FEW ? APPEND_MANY : APPEND_FEW;
    const int per = (most + threads - 1) / threads;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    if (threads == APPEND_FEW) return cudaLaunchKernelEx(&cfg, per == 1 ? kv8_append_kernel<APPEND_FEW, 1> : kv8_append_kernel<APPEND_FEW, 2>, a);
    return cudaLaunchKernelEx(&cfg, per == 1 ? kv8_append_kernel<APPEND_MANY, 1> : per == 2 ? kv8_append_kernel<APPEND_MANY, 2> : kv8_append_kernel<APPEND_MANY, 4>, a);
}

}  // namespace w4a8
