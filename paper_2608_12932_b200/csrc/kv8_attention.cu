// Attention over the 8-bit key/value cache for few rows: single tokens and draft blocks (definition and number formats in
// kv8_attention.cuh).
//
// kv8_attend_rows_kernel: one CTA per (sequence, key head, row tile, slice of the keys).  A row tile is 16 or 32 (token, head)
// rows of one key head's group, so a group's heads share what is read of the cache.  Each of the four warps walks its own chunks of 16
// positions with its own running sums: 16-byte asynchronous copies into a ring of its own (no block barrier in the loop),
// mma.m16n8k16 with the rows on the 16-row side.  The order of the contraction index is free as long as both operands agree,
// and so is the order of the output channels, so a lane takes 16 neighbouring codes of a key for the first product and 16
// neighbouring channels of four values for the second, and converts them in registers: nothing is transposed through shared memory.
// Bound by HBM as long as a chunk's 2 D B per position take longer than its products and conversions.
//
// kv8_combine_kernel: joins the slices' sums, one warp per row.
#include "kv8_attention.cuh"

namespace w4a8 {
namespace {

constexpr int AR_WARPS = 4, AR_CHUNK = 16;

template <int D, int RB>
struct ArCfg {
    static constexpr int ROWS = 16 * RB;
    static constexpr int K_BYTES = AR_CHUNK * D;                          // codes of a chunk's keys; as many of its values
    static constexpr int STAGE = 2 * K_BYTES;
    static constexpr int STAGES = 16384 / STAGE;                          // 16 KB in flight per warp
    static constexpr int RING = AR_WARPS * STAGES * STAGE;
    static constexpr int O_PITCH = D + 4;                                 // floats per row of the warps' sums at the end
    static constexpr int JOIN = AR_WARPS * ROWS * O_PITCH * 4;
    static constexpr int ML_OFF = RING > JOIN ? RING : JOIN;
    static constexpr int SMEM = ML_OFF + AR_WARPS * ROWS * 8;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Where 16-byte piece `p` of row `r` of a chunk lies: lines of 128 bytes (one row of 128 codes, or two of 64), the pieces of a line
// permuted so that the reads of eight lanes - two keys, four pieces; or four keys, two pieces - touch all banks once.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int r, int p) {
    const int line = D == 128 ? r : r >> 1, piece = D == 128 ? p : p + 4 * (r & 1);
    const int turn = D == 128 ? ((((line >> 1) & 3) << 1) ^ ((line & 1) << 2)) : ((line & 3) << 1);
    return (uint32_t)(line * 128 + ((piece ^ turn) << 4));
}

template <int D, int RB>
__global__ void __launch_bounds__(AR_WARPS * 32)
kv8_attend_rows_kernel(const __grid_constant__ AttendArgs a) {
    using C = ArCfg<D, RB>;
    constexpr int KS = D / 16;                               // k steps of the first product = words of codes per lane and key
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const uint32_t smem = ptx::smem_u32(smem_raw);
    ptx::pdl_launch_dependents();
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int tile = blockIdx.x / a.slices, slice = blockIdx.x - tile * a.slices, kv_head = blockIdx.z % a.kv_heads, seq = blockIdx.z / a.kv_heads;
    const int rows = a.T * a.rep, row0 = tile * C::ROWS;
    ptx::pdl_wait();

    // ---- this lane's rows: limits, q as fp16, and the factor that undoes its power of two
    int limit[RB][2];
    float factor[RB][2];
    uint32_t qf[RB][KS][4];
    int longest = 0, shortest = 0x7FFFFFFF;
    const int capacity = (int)min((long long)a.table_width << a.log2_block, 0x7FFFFFF0ll);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = row0 + rb * 16 + h * 8 + g;
            limit[rb][h] = 0;
            uint32_t w[KS * 2];
#pragma unroll
            for (int i = 0; i < KS * 2; ++i) w[i] = 0;
            if (r < rows) {
                const int token = r / a.rep, head = kv_head * a.rep + r - token * a.rep;
                const long long at = (long long)seq * a.T + token;
                limit[rb][h] = min(max(__ldcg(a.limits + at), 0), capacity);
                const uint16_t* src = a.q + at * a.q_stride + (long long)head * D + 16 * t;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    const uint4 x = __ldcg(reinterpret_cast<const uint4*>(src + 64 * i)), y = __ldcg(reinterpret_cast<const uint4*>(src + 64 * i + 8));
                    w[8 * i] = x.x, w[8 * i + 1] = x.y, w[8 * i + 2] = x.z, w[8 * i + 3] = x.w;
                    w[8 * i + 4] = y.x, w[8 * i + 5] = y.y, w[8 * i + 6] = y.z, w[8 * i + 7] = y.w;
                }
                shortest = min(shortest, limit[rb][h]);
            }
            longest = max(longest, limit[rb][h]);
            uint32_t run = 0;
#pragma unroll
            for (int i = 0; i < KS * 2; ++i) run = __vmaxu2(run, w[i] & 0x7FFF7FFFu);
            run = max(run & 0xFFFFu, run >> 16);
            run = max(run, __shfl_xor_sync(0xFFFFFFFFu, run, 1));
            run = max(run, __shfl_xor_sync(0xFFFFFFFFu, run, 2));
            const int e = kv8_row_exp(run);
            const float up = kv8_pow2(e);
            factor[rb][h] = a.scale_log2 * kv8_pow2(-e);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                qf[rb][i][h] = kv8_pack_half2(__uint_as_float(w[2 * i] << 16) * up, __uint_as_float(w[2 * i] & 0xFFFF0000u) * up);
                qf[rb][i][2 + h] = kv8_pack_half2(__uint_as_float(w[2 * i + 1] << 16) * up, __uint_as_float(w[2 * i + 1] & 0xFFFF0000u) * up);
            }
        }
    }
    longest = __reduce_max_sync(0xFFFFFFFFu, longest);
    shortest = __reduce_min_sync(0xFFFFFFFFu, shortest);

    // ---- this CTA's chunks of 16 positions, dealt to the warps in turn
    const int chunks = (int)(((long long)longest + AR_CHUNK - 1) / AR_CHUNK);
    const int c_lo = (int)((long long)slice * chunks / a.slices), c_hi = (int)((long long)(slice + 1) * chunks / a.slices);
    const int mine = (c_hi - c_lo - warp + AR_WARPS - 1) / AR_WARPS;
    const int chunk_shift = a.log2_block - 4;                // chunks per block, as a shift
    const int32_t* table = a.table + (size_t)seq * a.table_width;
    // lane j holds block number and scales of chunk 32 i + j of this warp, for the current 32 chunks and the next
    struct Meta { int number; uint32_t ks, vs; };
    auto meta_of = [&](int base) -> Meta {
        Meta m = {-1, 0u, 0u};
        const int i = base + lane;
        if (i < mine) {
            const int number = __ldcg(table + ((c_lo + warp + AR_WARPS * i) >> chunk_shift));
            if ((unsigned)number < (unsigned)a.num_blocks) {
                const size_t at = (size_t)number * a.kv_heads + kv_head;
                m.number = number;
                m.ks = __ldcg(a.k_scales + at);
                m.vs = __ldcg(a.v_scales + at);
            } else {
                *a.status = W4A8_ERR_INDEX;                  // positions of a block that does not exist count as not there
            }
        }
        return m;
    };
    Meta cur = meta_of(0), nxt = meta_of(32);
    int base = 0;
    const uint32_t ring = smem + warp * (C::STAGES * C::STAGE);
    auto issue = [&](int i) {
        if (i < mine) {
            const int number = __shfl_sync(0xFFFFFFFFu, i - base < 32 ? cur.number : nxt.number, i & 31);
            if (number >= 0) {
                const int c = c_lo + warp + AR_WARPS * i;
                const int slot = (c & ((1 << chunk_shift) - 1)) * AR_CHUNK;
                const size_t at = ((((size_t)number * a.kv_heads + kv_head) << a.log2_block) + slot) * D;
                const uint32_t dst = ring + (i % C::STAGES) * C::STAGE;
#pragma unroll
                for (int j = 0; j < C::K_BYTES / 512; ++j) {
                    const int idx = j * 32 + lane, r = idx / (D / 16), p = idx % (D / 16);
                    cp_async16(dst + chunk_at<D>(r, p), a.k_codes + at + idx * 16);
                    cp_async16(dst + C::K_BYTES + chunk_at<D>(r, p), a.v_codes + at + idx * 16);
                }
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) issue(i);

    float o[RB][D / 8][4];
    float ref[RB][2], sum[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) o[rb][j][0] = o[rb][j][1] = o[rb][j][2] = o[rb][j][3] = 0.0f;
        ref[rb][0] = ref[rb][1] = -INFINITY;
        sum[rb][0] = sum[rb][1] = 0.0f;
    }
    for (int i = 0; i < mine; ++i) {
        if (i == base + 32) {
            base += 32;
            cur = nxt;
            nxt = meta_of(base + 32);
        }
        cp_async_wait<C::STAGES - 2>();
        __syncwarp();
        issue(i + C::STAGES - 1);
        const int number = __shfl_sync(0xFFFFFFFFu, cur.number, i & 31);
        const uint32_t ks_bits = __shfl_sync(0xFFFFFFFFu, cur.ks, i & 31), vs_bits = __shfl_sync(0xFFFFFFFFu, cur.vs, i & 31);
        if (number < 0) continue;
        const int key0 = (c_lo + warp + AR_WARPS * i) * AR_CHUNK;
        const uint32_t kst = ring + (i % C::STAGES) * C::STAGE, vst = kst + C::K_BYTES;
        // ---- scores of 16 positions: columns 8 n + 2 t, + 1
        float s[RB][2][4];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int n = 0; n < 2; ++n) s[rb][n][0] = s[rb][n][1] = s[rb][n][2] = s[rb][n][3] = 0.0f;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int i4 = 0; i4 < D / 64; ++i4) {
                const uint4 x = ptx::lds128(kst + chunk_at<D>(8 * n + g, t + 4 * i4));
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t u = w[j] ^ 0x80808080u;
                    const uint32_t b0 = kv8_half2(u, 0x4140), b1 = kv8_half2(u, 0x4342);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) mma_f16(s[rb][n], qf[rb][4 * i4 + j], b0, b1);
                }
            }
        }
        float lg, inv;
        kv8_value_scale(vs_bits, lg, inv);
        const float ks = __half2float(__ushort_as_half((uint16_t)ks_bits));
        // ---- weights: x = score in base 2 + log2 of the value scale
        bool past = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float f = factor[rb][h] * ks, most = ref[rb][h] + KV8_SLACK;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float& x = s[rb][n][2 * h + j];
                        x = fmaf(x, f, lg);
                        if (key0 + AR_CHUNK > shortest && key0 + 8 * n + 2 * t + j >= limit[rb][h]) x = -INFINITY;
                        past |= x > most;
                    }
                }
            }
        }
        if (__any_sync(0xFFFFFFFFu, past)) {
            // some weight would pass the range that fp16 leaves for it: the references move to the rows' maxima
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = fmaxf(fmaxf(s[rb][0][2 * h], s[rb][0][2 * h + 1]), fmaxf(s[rb][1][2 * h], s[rb][1][2 * h + 1]));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                    top = fmaxf(top, ref[rb][h]);
                    const float f = ref[rb][h] == -INFINITY ? 0.0f : kv8_ex2(ref[rb][h] - top);
                    ref[rb][h] = top;
                    sum[rb][h] *= f;
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) {
                        o[rb][j][2 * h] *= f;
                        o[rb][j][2 * h + 1] *= f;
                    }
                }
            }
        }
        uint32_t wf[RB][4];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float off = ref[rb][h] == -INFINITY ? 0.0f : KV8_W_EXP - ref[rb][h];       // (no position seen yet: weights 0)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float w0 = kv8_ex2(s[rb][n][2 * h] + off), w1 = kv8_ex2(s[rb][n][2 * h + 1] + off);
                    sum[rb][h] = fmaf(w0 + w1, inv, sum[rb][h]);
                    wf[rb][2 * n + h] = kv8_pack_half2(w0, w1);
                }
            }
        }
        // ---- o += weights x values: this lane's positions 2 t, 2 t + 1, 2 t + 8, 2 t + 9, channels (D / 8) g + j
        uint32_t v[4][D / 32];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = 2 * t + (k & 1) + 8 * (k >> 1);
            if (D == 128) {
                const uint4 x = ptx::lds128(vst + chunk_at<D>(r, g));
                v[k][0] = x.x, v[k][1] = x.y, v[k][D / 32 - 2] = x.z, v[k][D / 32 - 1] = x.w;
            } else {
                const uint2 x = ptx::lds64(vst + chunk_at<D>(r, g >> 1) + 8 * (g & 1));
                v[k][0] = x.x, v[k][1] = x.y;
            }
        }
#pragma unroll
        for (int i4 = 0; i4 < D / 32; ++i4) {
            uint32_t p[2][2];                                // positions (0, 1) and (2, 3): channels 0 1 and 2 3 of this word, position by position
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t x = v[2 * k][i4] ^ 0x80808080u, y = v[2 * k + 1][i4] ^ 0x80808080u;
                p[k][0] = __byte_perm(x, y, 0x5140);
                p[k][1] = __byte_perm(x, y, 0x7362);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t sel = j & 1 ? 0x4342 : 0x4140;
                const uint32_t b0 = kv8_half2(p[0][j >> 1], sel), b1 = kv8_half2(p[1][j >> 1], sel);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) mma_f16(o[rb][4 * i4 + j], wf[rb], b0, b1);
            }
        }
    }
    cp_async_wait<0>();
    __syncthreads();                                         // the rings are free: they take the warps' sums

    // ---- the four warps' sums, joined
    float* join = reinterpret_cast<float*>(smem_raw);
    float2* ml = reinterpret_cast<float2*>(smem_raw + C::ML_OFF);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = rb * 16 + h * 8 + g;
            float l = sum[rb][h];
            l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
            l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
            if (t == 0) ml[warp * C::ROWS + r] = make_float2(ref[rb][h], l);
            // columns 2 t and 2 t + 1 of product j are channels (D / 8) (2 t) + j and (D / 8) (2 t + 1) + j
            float* dst = join + (warp * C::ROWS + r) * C::O_PITCH + (D / 8) * 2 * t;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int j = 0; j < D / 8; j += 4)
                    *reinterpret_cast<float4*>(dst + c * (D / 8) + j) = make_float4(o[rb][j][2 * h + c], o[rb][j + 1][2 * h + c], o[rb][j + 2][2 * h + c], o[rb][j + 3][2 * h + c]);
            }
        }
    }
    __syncthreads();
    const size_t unit = ((size_t)blockIdx.z * a.tiles + tile) * a.slices + slice;
    for (int idx = tid; idx < C::ROWS * (D / 4); idx += AR_WARPS * 32) {
        const int r = idx / (D / 4), d = (idx % (D / 4)) * 4, row = row0 + r;
        if (row >= rows) break;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < AR_WARPS; ++w) m = fmaxf(m, ml[w * C::ROWS + r].x);
        float l = 0.0f;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < AR_WARPS; ++w) {
            const float2 one = ml[w * C::ROWS + r];
            // (a row without a reference has no weights, or is not a number in all of them)
            const float f = one.x == -INFINITY ? 1.0f : kv8_ex2(one.x - m);
            const float4 y = *reinterpret_cast<const float4*>(join + (w * C::ROWS + r) * C::O_PITCH + d);
            l = fmaf(f, one.y, l);
            x.x = fmaf(f, y.x, x.x);
            x.y = fmaf(f, y.y, x.y);
            x.z = fmaf(f, y.z, x.z);
            x.w = fmaf(f, y.w, x.w);
        }
        if (a.slices > 1) {
            *reinterpret_cast<float4*>(a.part_o + (unit * C::ROWS + r) * D + d) = x;
            if (d == 0) a.part_ml[unit * C::ROWS + r] = make_float2(m, l);
        } else {
            const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
            const int token = row / a.rep, head = kv_head * a.rep + row - token * a.rep;
            uint2* dst = reinterpret_cast<uint2*>(a.out + (((long long)seq * a.T + token) * a.q_heads + head) * D + d);
            *dst = make_uint2(ptx::pack_bf16x2(x.x * inv, x.y * inv), ptx::pack_bf16x2(x.z * inv, x.w * inv));
        }
    }
}

// One warp per (token, head) row: the slices' sums, each weighted by how far its reference is below the largest.
template <int D>
__global__ void __launch_bounds__(128)
kv8_combine_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, uint16_t* __restrict__ out, long long total_rows,
                   int T, int q_heads, int kv_heads, int rep, int tiles, int slices, int tile_rows) {
    constexpr int V = D / 32;
    ptx::pdl_launch_dependents();
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    ptx::pdl_wait();
    if (row >= total_rows) return;
    const int head = (int)(row % q_heads);
    const long long at = row / q_heads;                      // seq T + token
    const int token = (int)(at % T), kv_head = head / rep;
    const long long r = (long long)token * rep + head - kv_head * rep;
    const size_t unit = (((size_t)(at / T) * kv_heads + kv_head) * tiles + (size_t)(r / tile_rows)) * slices;
    const size_t first = unit * tile_rows + (size_t)(r % tile_rows);
    float m = -INFINITY;
    for (int z = lane; z < slices; z += 32) m = fmaxf(m, __ldcg(&part_ml[first + (size_t)z * tile_rows]).x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float l = 0.0f, x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
#pragma unroll 4
    for (int z = 0; z < slices; ++z) {
        const size_t p = first + (size_t)z * tile_rows;
        const float2 one = __ldcg(&part_ml[p]);
        const float f = one.x == -INFINITY ? 1.0f : kv8_ex2(one.x - m);
        l = fmaf(f, one.y, l);
        const float* src = part_o + p * D + lane * V;
        if (V == 4) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(src));
            x[0] = fmaf(f, y.x, x[0]);
            x[1] = fmaf(f, y.y, x[1]);
            x[V - 2] = fmaf(f, y.z, x[V - 2]);
            x[V - 1] = fmaf(f, y.w, x[V - 1]);
        } else {
            const float2 y = __ldcg(reinterpret_cast<const float2*>(src));
            x[0] = fmaf(f, y.x, x[0]);
            x[1] = fmaf(f, y.y, x[1]);
        }
    }
    const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
    uint32_t* dst = reinterpret_cast<uint32_t*>(out + row * D) + lane * (V / 2);
    if (V == 4)
        *reinterpret_cast<uint2*>(dst) = make_uint2(ptx::pack_bf16x2(x[0] * inv, x[1] * inv), ptx::pack_bf16x2(x[V - 2] * inv, x[V - 1] * inv));
    else
        *dst = ptx::pack_bf16x2(x[0] * inv, x[1] * inv);
}

template <int D, int RB>
cudaError_t launch_rows(const AttendArgs& a, int B, cudaStream_t stream) {
    using C = ArCfg<D, RB>;
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(kv8_attend_rows_kernel<D, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.slices * (unsigned)a.tiles, 1, (unsigned)(B * a.kv_heads));
    cfg.blockDim = dim3(AR_WARPS * 32, 1, 1);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv8_attend_rows_kernel<D, RB>, a);
}

template <int D>
cudaError_t launch_combine(const AttendArgs& a, int B, int tile_rows, cudaStream_t stream) {
    const long long total = (long long)B * a.T * a.q_heads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((total + 3) / 4), 1, 1);
    cfg.blockDim = dim3(128, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv8_combine_kernel<D>, (const float*)a.part_o, (const float2*)a.part_ml, a.out, total, a.T, a.q_heads,
                              a.kv_heads, a.rep, a.tiles, a.slices, tile_rows);
}

}  // namespace

// Row tiles of 16 with three CTAs per SM, of 32 with two, of 256 with one: what is resident at once.
static int ctas_per_sm(int rows) { return rows == 16 ? 3 : (rows == 32 ? 2 : 1); }

Kv8Plan kv8_plan(int B, int T, int q_heads, int kv_heads, long long max_keys, int sms) {
    Kv8Plan p;
    const long long rows = (long long)T * (q_heads / kv_heads);
    p.rows = rows <= 16 ? 16 : (rows <= 32 ? 32 : 256);
    p.tiles = (int)((rows + p.rows - 1) / p.rows);
    const long long units = (long long)B * kv_heads * p.tiles;
    long long s = (long long)ctas_per_sm(p.rows) * sms / units;
    // two chunks for each of a CTA's warps, two steps of the tensor-memory kernel
    const long long most = p.rows == 256 ? (max_keys + 255) / 256 : (max_keys + 127) / 128;
    if (s > most) s = most;
    p.slices = (int)(s < 1 ? 1 : s);
    return p;
}

// Enough for any call: there are several slices only where all row tiles' slices together are resident at once.
size_t kv8_partial_bytes(int dim, int sms) { return (size_t)sms * 256 * (dim * 4 + 8); }

cudaError_t launch_kv8_attention(const w4a8_kv8_cache& c, const void* q, long long q_stride, int B, int T, int q_heads, const int32_t* table,
                                 int table_width, const int32_t* limits, float scale, void* out, void* workspace, cudaStream_t stream) {
    const Kv8Plan p = kv8_plan(B, T, q_heads, c.heads, (long long)table_width * c.block, device_sm_count());
    AttendArgs a;
    a.k_codes = c.k_codes;
    a.v_codes = c.v_codes;
    a.k_scales = c.k_scales;
    a.v_scales = c.v_scales;
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.table = table;
    a.limits = limits;
    a.out = static_cast<uint16_t*>(out);
    a.status = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + WS_STATUS_OFF);
    a.T = T;
    a.q_heads = q_heads;
    a.kv_heads = c.heads;
    a.rep = q_heads / c.heads;
    a.table_width = table_width;
    a.num_blocks = c.num_blocks;
    a.log2_block = kv8_log2(c.block);
    a.tiles = p.tiles;
    a.slices = p.slices;
    a.scale_log2 = scale * 1.44269504088896340736f;
    const size_t units = (size_t)B * c.heads * p.tiles * p.slices;
    a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + WS_SHARED_OFF);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + units * p.rows * c.dim);
    cudaError_t e;
    if (p.rows == 256)
        e = launch_kv8_tiles(a, B, c.dim, stream);
    else if (p.rows == 16)
        e = c.dim == 128 ? launch_rows<128, 1>(a, B, stream) : launch_rows<64, 1>(a, B, stream);
    else
        e = c.dim == 128 ? launch_rows<128, 2>(a, B, stream) : launch_rows<64, 2>(a, B, stream);
    if (e != cudaSuccess || p.slices == 1) return e;
    return c.dim == 128 ? launch_combine<128>(a, B, p.rows, stream) : launch_combine<64>(a, B, p.rows, stream);
}

}  // namespace w4a8
