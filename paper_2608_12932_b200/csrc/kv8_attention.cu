// Attention over the 8-bit key/value cache for few rows: single tokens and draft blocks (definition and number formats in
// kv8_attention.cuh).
//
// kv8_attend_rows_kernel: one CTA per (sequence, key head, slice of the keys) for the 16 or 32 (token, head) rows of the key
// head's group, so a group's heads share what is read of the cache.  Two pairs of warps walk chunks of 2 x 16 positions,
// each pair with its own running sums: a warp fetches 16 positions' codes (16-byte asynchronous copies into a ring of its own), forms their
// scores and weights, hands the weights to its partner through shared memory, and multiplies the values of all 32 positions for its half of the
// channels.  So a warp keeps half a tile's sums: a warp that keeps all of them needs 255 registers at 32 rows, and two warps
// per scheduler leave it idle most of the time (a draft block of 8 over 32749 positions: 39 us).  Bound by a chunk's chain of dependent steps and its
// 520 warp instructions per 16 positions, not by the cache's bytes: that block 27.4 us (2.4 TB/s, issue 0.48 a cycle and scheduler), one token over
// 65000 positions 31.5 us (4.2 TB/s, 0.59); a single short sequence by the chain of limits, table, codes, and by the second launch (4096 positions 8.4 us).
// mma.m16n8k16 with the rows on the 16-row side.  The order of the contraction index is free as long as both operands
// agree, and so is the order of the output channels, so a lane takes 16 neighbouring codes of a key for the first product and neighbouring
// channels of four values for the second, and converts them in registers: nothing is transposed through shared memory.  The
// weights come out of the first product as the second one's operand: a lane stores 16 bytes and its partner's lane loads them.
//
// kv8_combine_kernel: joins the slices' sums.
#include "kv8_attention.cuh"

namespace w4a8 {
namespace {

constexpr int AR_WARPS = 4, AR_CHUNK = 16;

template <int D, int RB>
struct ArCfg {
    static constexpr int ROWS = 16 * RB;
    static constexpr int CTAS = RB == 1 ? 4 : 3;                          // per SM
    static constexpr int K_BYTES = AR_CHUNK * D;                          // codes of a chunk's keys; as many of its values
    static constexpr int STAGE = 2 * K_BYTES;
    static constexpr int STAGES = 12288 / STAGE;                          // 12 KB per warp, one stage of it being worked on
    static constexpr int RING = AR_WARPS * STAGES * STAGE;
    static constexpr int O_PITCH = D + 4;                                 // floats per row of the pairs' sums at the end
    static constexpr int JOIN = 2 * ROWS * O_PITCH * 4;
    static constexpr int W_OFF = RING > JOIN ? RING : JOIN;               // weights on their way: [warp][turn & 1][RB][lane] 16 bytes
    static constexpr int W_BYTES = RB * 512;
    static constexpr int W_END = W_OFF + AR_WARPS * 2 * W_BYTES;
    static constexpr int Q_OFF = RB == 1 ? W_OFF : W_END;                 // q as operand: [D / 16][RB][lane] 16 bytes (16 rows: only passing through)
    static constexpr int FACTOR_OFF = RB == 1 ? W_END : Q_OFF + (D / 16) * RB * 512;        // rows' factors: [ROWS] float
    static constexpr int TOP_OFF = FACTOR_OFF + ROWS * 4;                 // rows' maxima where a reference moves: [warp][ROWS] float
    static constexpr int FLAG_OFF = TOP_OFF + AR_WARPS * ROWS * 4;        // whether one does: [warp][turn & 1]
    static constexpr int ML_OFF = FLAG_OFF + AR_WARPS * 8;                // at the end: references and sums of each warp's positions
    static constexpr int SMEM = ML_OFF + AR_WARPS * ROWS * 8;
    static_assert(CTAS * (SMEM + 1024) <= 228 * 1024, "shared memory");
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

// From a place to others, a chunk's first byte being a multiple of 128 (spelled out: eight rows on keep the turn, and so on, which the compiler does
// not see; with an evaluation of chunk_at for each access the loop had a fifth more instructions)
template <int D>
__device__ __forceinline__ constexpr uint32_t rows_on8() { return D == 128 ? 1024u : 512u; }
template <int D>
__device__ __forceinline__ uint32_t row_on1_from_even(uint32_t at) { return D == 128 ? (at + 128u) ^ 64u : at ^ 64u; }
__device__ __forceinline__ uint32_t pieces_on4(uint32_t at) { return at ^ 64u; }                   // D = 128
template <int D>
__device__ __forceinline__ uint32_t bytes_on512(uint32_t at, int j) { return D == 128 && (j & 1) ? (at ^ 64u) + 512u * j : at + 512u * j; }

template <int D, int RB>
__global__ void __launch_bounds__(AR_WARPS * 32, (ArCfg<D, RB>::CTAS))
kv8_attend_rows_kernel(const __grid_constant__ AttendArgs a) {
    using C = ArCfg<D, RB>;
    constexpr int KS = D / 16;                               // k steps of the first product = words of codes per lane and key
    constexpr int NB = D / 16;                               // 8-channel blocks of this warp's half of the second product
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const uint32_t smem = ptx::smem_u32(smem_raw);
    ptx::pdl_launch_dependents();
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int pair = warp >> 1, side = warp & 1;
    const int slice = blockIdx.x, kv_head = blockIdx.z % a.kv_heads, seq = blockIdx.z / a.kv_heads;
    const int rows = a.T * a.rep;
    ptx::pdl_wait();

    // ---- this lane's rows' limits (all loads ahead of the first use); and q: eight rows (half a block of 16) in each of the first 2 RB warps, in flight
    // while the first copies are issued, then as fp16 operand, with the factors that undo its powers of two, through shared memory
    int limit[RB][2];
    int longest = 0, shortest = 0x7FFFFFFF;
    const int capacity = (int)min((long long)a.table_width << a.log2_block, 0x7FFFFF00ll);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int h = 0; h < 2; ++h) limit[rb][h] = __ldcg(a.limits + (long long)seq * a.T + min(rb * 16 + h * 8 + g, rows - 1) / a.rep);
    }
    uint32_t w[KS * 2];
#pragma unroll
    for (int i = 0; i < KS * 2; ++i) w[i] = 0;
    if (warp < 2 * RB) {
        const int r = (warp >> 1) * 16 + (warp & 1) * 8 + g;
        if (r < rows) {
            const int token = r / a.rep, head = kv_head * a.rep + r - token * a.rep;
            const uint16_t* src = a.q + ((long long)seq * a.T + token) * a.q_stride + (long long)head * D + 16 * t;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const uint4 x = __ldcg(reinterpret_cast<const uint4*>(src + 64 * i)), y = __ldcg(reinterpret_cast<const uint4*>(src + 64 * i + 8));
                w[8 * i] = x.x, w[8 * i + 1] = x.y, w[8 * i + 2] = x.z, w[8 * i + 3] = x.w;
                w[8 * i + 4] = y.x, w[8 * i + 5] = y.y, w[8 * i + 6] = y.z, w[8 * i + 7] = y.w;
            }
        }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool real = rb * 16 + h * 8 + g < rows;
            limit[rb][h] = real ? min(max(limit[rb][h], 0), capacity) : 0;
            shortest = min(shortest, real ? limit[rb][h] : 0x7FFFFFFF);
            longest = max(longest, limit[rb][h]);
        }
    }
    longest = __reduce_max_sync(0xFFFFFFFFu, longest);
    shortest = __reduce_min_sync(0xFFFFFFFFu, shortest);
    if (lane < 2) asm volatile("st.shared.u32 [%0], %1;" ::"r"(smem + C::FLAG_OFF + warp * 8 + lane * 4), "r"(0u) : "memory");

    // ---- this CTA's chunks of 16 positions, dealt in twos to the pairs in turn, one of the two to each warp
    const int chunks = (int)(((long long)longest + AR_CHUNK - 1) / AR_CHUNK);
    const int c_lo = (int)((long long)slice * chunks / a.slices), c_hi = (int)((long long)(slice + 1) * chunks / a.slices);
    const int turns = (c_hi - c_lo - 2 * pair + 3) / 4;      // of the pair
    const int first = c_lo + warp;                           // this warp's chunk of turn i: first + 4 i (none where that is c_hi or more)
    const int chunk_shift = a.log2_block - 4;                // chunks per block, as a shift
    const int32_t* table = a.table + (size_t)seq * a.table_width;
    // lane j holds block number and scales of this warp's chunk of turn 32 i + j, for the current 32 turns and the next
    struct Meta { int number; uint32_t ks, vs; };
    auto meta_of = [&](int base) -> Meta {
        Meta m = {-1, 0u, 0u};
        const int c = first + 4 * (base + lane);
        if (base + lane < turns && c < c_hi) {
            const int number = __ldcg(table + (c >> chunk_shift));
            if ((unsigned)number < (unsigned)a.num_blocks) {
                const size_t at = (size_t)number * a.kv_heads + kv_head;
                m.number = number;
                m.ks = __ldcg(a.k_scales + at);
                m.vs = __ldcg(a.v_scales + at);
            } else {
                flag_index(a.status);                        // positions of a block that does not exist count as not there
            }
        }
        return m;
    };
    Meta cur = meta_of(0), nxt = {-1, 0u, 0u};
    if (turns > 32) nxt = meta_of(32);
    int base = 0;
    const uint32_t ring = smem + warp * (C::STAGES * C::STAGE), other_ring = smem + (warp ^ 1) * (C::STAGES * C::STAGE);
    int slot_in = 0;
    const uint32_t in_at = chunk_at<D>(lane / (D / 16), lane % (D / 16)), k_at = chunk_at<D>(g, t);
    const uint32_t v_at = C::K_BYTES + (D == 128 ? chunk_at<D>(2 * t, 4 * side + (g >> 1)) + 8 * (g & 1) : chunk_at<D>(2 * t, 2 * side + (g >> 2)) + 4 * (g & 3));
    auto issue = [&](int i) {
        if (i < turns) {
            const int number = __shfl_sync(0xFFFFFFFFu, i - base < 32 ? cur.number : nxt.number, i & 31);
            if (number >= 0) {
                const int inside = ((first + 4 * i) & ((1 << chunk_shift) - 1)) * AR_CHUNK;
                const size_t at = ((((size_t)number * a.kv_heads + kv_head) << a.log2_block) + inside) * D + lane * 16;
                const int8_t *k = a.k_codes + at, *v = a.v_codes + at;
                const uint32_t dst = ring + slot_in * C::STAGE + in_at;
#pragma unroll
                for (int j = 0; j < C::K_BYTES / 512; ++j) {
                    cp_async16(bytes_on512<D>(dst, j), k + j * 512);
                    cp_async16(bytes_on512<D>(dst, j) + C::K_BYTES, v + j * 512);
                }
            }
        }
        slot_in = slot_in + 1 == C::STAGES ? 0 : slot_in + 1;
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) issue(i);
    if (warp < 2 * RB) {                                     // (the first copies are on their way)
        const int rb = warp >> 1, h = warp & 1;
        uint32_t run = 0;
#pragma unroll
        for (int i = 0; i < KS * 2; ++i) run = __vmaxu2(run, w[i] & 0x7FFF7FFFu);
        run = max(run & 0xFFFFu, run >> 16);
        run = max(run, __shfl_xor_sync(0xFFFFFFFFu, run, 1));
        run = max(run, __shfl_xor_sync(0xFFFFFFFFu, run, 2));
        const int e = kv8_row_exp(run);
        const float up = kv8_pow2(e);
        const float factor = run >= 0x7F80u ? NAN : a.scale_log2 * kv8_pow2(-e);             // an infinity in the row: every score of it is not a number
        if (t == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + C::FACTOR_OFF + (rb * 16 + h * 8 + g) * 4), "f"(factor) : "memory");
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            // words h and 2 + h of the lane's four
            const uint32_t at = smem + C::Q_OFF + ((i * RB + rb) * 32 + lane) * 16 + 4 * h;
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(kv8_pack_half2(__uint_as_float(w[2 * i] << 16) * up, __uint_as_float(w[2 * i] & 0xFFFF0000u) * up)) : "memory");
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + 8), "r"(kv8_pack_half2(__uint_as_float(w[2 * i + 1] << 16) * up, __uint_as_float(w[2 * i + 1] & 0xFFFF0000u) * up)) : "memory");
        }
    }
    __syncthreads();                                         // q and flags are there
    float factor[RB][2];
    uint32_t qf[RB == 1 ? KS : 1][4];                        // 16 rows: q stays in registers
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int h = 0; h < 2; ++h) factor[rb][h] = __uint_as_float(ptx::lds32(smem + C::FACTOR_OFF + (rb * 16 + h * 8 + g) * 4));
    if (RB == 1) {
#pragma unroll
        for (int i = 0; i < (RB == 1 ? KS : 1); ++i) {
            const uint4 y = ptx::lds128(smem + C::Q_OFF + (i * 32 + lane) * 16);
            qf[i][0] = y.x, qf[i][1] = y.y, qf[i][2] = y.z, qf[i][3] = y.w;
        }
        __syncthreads();                                     // weights follow in its place
    }

    float o[RB][NB][4];
    float ref[RB][2], sum[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int j = 0; j < NB; ++j) o[rb][j][0] = o[rb][j][1] = o[rb][j][2] = o[rb][j][3] = 0.0f;
        ref[rb][0] = ref[rb][1] = -INFINITY;
        sum[rb][0] = sum[rb][1] = 0.0f;
    }
    const uint32_t w_out = smem + C::W_OFF + warp * (2 * C::W_BYTES) + lane * 16, w_in = smem + C::W_OFF + (warp ^ 1) * (2 * C::W_BYTES) + lane * 16;
    const uint32_t flag_out = smem + C::FLAG_OFF + warp * 8, flag_in = smem + C::FLAG_OFF + (warp ^ 1) * 8;
    int slot = 0;
    for (int i = 0; i < turns; ++i) {
        if (i == base + 32) {
            base += 32;
            cur = nxt;
            if (turns > base + 32) nxt = meta_of(base + 32);
        }
        cp_async_wait<C::STAGES - 2>();
        __syncwarp();
        const int number = __shfl_sync(0xFFFFFFFFu, cur.number, i & 31);
        const uint32_t scales = __shfl_sync(0xFFFFFFFFu, cur.ks | cur.vs << 16, i & 31);         // (put together here: copies do not wait for them)
        const int key0 = (first + 4 * i) * AR_CHUNK;
        const uint32_t kst = ring + slot * C::STAGE + k_at;
        // ---- scores of this warp's 16 positions: columns 8 n + 2 t, + 1
        float s[RB][2][4];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int n = 0; n < 2; ++n) s[rb][n][0] = s[rb][n][1] = s[rb][n][2] = s[rb][n][3] = 0.0f;
#pragma unroll
        for (int i4 = 0; i4 < D / 64; ++i4) {
            const uint32_t at = i4 ? pieces_on4(kst) : kst;
            const uint4 x0 = ptx::lds128(at), x1 = ptx::lds128(at + rows_on8<D>());
            const uint32_t w[2][4] = {{x0.x, x0.y, x0.z, x0.w}, {x1.x, x1.y, x1.z, x1.w}};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t q[RB][4];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    if (RB == 1) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) q[rb][k] = qf[(4 * i4 + j) % (RB == 1 ? KS : 1)][k];
                    } else {
                        const uint4 y = ptx::lds128(smem + C::Q_OFF + (((4 * i4 + j) * RB + rb) * 32 + lane) * 16);
                        q[rb][0] = y.x, q[rb][1] = y.y, q[rb][2] = y.z, q[rb][3] = y.w;
                    }
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint32_t u = w[n][j] ^ 0x80808080u;
                    const uint32_t b0 = kv8_half2(u, 0x4140), b1 = kv8_half2(u, 0x4342);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) mma_f16(s[rb][n], q[rb], b0, b1);
                }
            }
        }
        float lg, inv;
        kv8_value_scale(scales >> 16, lg, inv);
        const float ks = __half2float(__ushort_as_half((uint16_t)scales));
        // ---- weights at the references as they are: 2^x, x the score in base 2 + log2 of the value scale - reference + 7
        const bool none = number < 0, part = none || key0 + AR_CHUNK > shortest;
        bool past = false;
        uint32_t wf[RB][4];
        float more[RB][2];
        auto weigh = [&]() {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float all = 0.0f;
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const float w0 = kv8_ex2(s[rb][n][2 * h]), w1 = kv8_ex2(s[rb][n][2 * h + 1]);
                        all += w0 + w1;
                        wf[rb][2 * n + h] = kv8_pack_half2(w0, w1);
                    }
                    more[rb][h] = all;
                }
                ptx::sts128u(w_out + (i & 1) * C::W_BYTES + rb * 512, wf[rb][0], wf[rb][1], wf[rb][2], wf[rb][3]);
            }
        };
        float off[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                off[rb][h] = ref[rb][h] == -INFINITY ? 0.0f : KV8_W_EXP - ref[rb][h];
                const float f = factor[rb][h] * ks, add = lg + off[rb][h];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) s[rb][n][2 * h + j] = fmaf(s[rb][n][2 * h + j], f, add);
                }
            }
        }
        if (part) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (none || key0 + 8 * (e >> 2) + 2 * t + (e & 1) >= limit[rb][(e >> 1) & 1]) s[rb][e >> 2][e & 3] = -INFINITY;
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float top = fmaxf(fmaxf(s[rb][0][2 * h], s[rb][0][2 * h + 1]), fmaxf(s[rb][1][2 * h], s[rb][1][2 * h + 1]));
                past |= top > (ref[rb][h] == -INFINITY ? -INFINITY : KV8_W_EXP + KV8_SLACK);
            }
        }
        past = __any_sync(0xFFFFFFFFu, past);
        weigh();
        if (past) {
            // some weight is past the range that fp16 leaves for it: the rows' maxima, for both warps of the pair
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = fmaxf(fmaxf(s[rb][0][2 * h], s[rb][0][2 * h + 1]), fmaxf(s[rb][1][2 * h], s[rb][1][2 * h + 1]));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2)) - off[rb][h];
                    if (t == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + C::TOP_OFF + (warp * C::ROWS + rb * 16 + h * 8 + g) * 4), "f"(top) : "memory");
                }
            }
            if (lane == 0) asm volatile("st.shared.u32 [%0], 1;" ::"r"(flag_out + (i & 1) * 4) : "memory");
        }
        ptx::named_bar_sync(1 + pair, 64);                   // the pair's weights are there, and both warps' values; it is done with the turn before
        issue(i + C::STAGES - 1);
        const bool theirs = ptx::lds32(flag_in + (i & 1) * 4) != 0u;
        if (past || theirs) {
            // the references move to the larger of what they are and the maxima, and the weights of the turn are made anew
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = ref[rb][h];
                    const int r = rb * 16 + h * 8 + g;
                    if (past) top = fmaxf(top, __uint_as_float(ptx::lds32(smem + C::TOP_OFF + (warp * C::ROWS + r) * 4)));
                    if (theirs) top = fmaxf(top, __uint_as_float(ptx::lds32(smem + C::TOP_OFF + ((warp ^ 1) * C::ROWS + r) * 4)));
                    const float f = ref[rb][h] == -INFINITY ? 0.0f : kv8_ex2(ref[rb][h] - top);
                    ref[rb][h] = top;
                    sum[rb][h] = top == INFINITY ? NAN : sum[rb][h] * f;        // an infinite score: not a number from here on
                    const float shift = (top == -INFINITY ? 0.0f : KV8_W_EXP - top) - off[rb][h];
#pragma unroll
                    for (int n = 0; n < 2; ++n) s[rb][n][2 * h] += shift, s[rb][n][2 * h + 1] += shift;
#pragma unroll
                    for (int j = 0; j < NB; ++j) o[rb][j][2 * h] *= f, o[rb][j][2 * h + 1] *= f;
                }
            }
            weigh();
            ptx::named_bar_sync(1 + pair, 64);
            if (lane == 0) asm volatile("st.shared.u32 [%0], 0;" ::"r"(flag_out + (i & 1) * 4) : "memory");
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[rb][h] = fmaf(more[rb][h], inv, sum[rb][h]);
        // ---- o += weights x values, this warp's half of the channels: positions 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of either warp's 16, channels
        // NB g + j of the half
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {
            const uint32_t vst = (turn ? other_ring : ring) + slot * C::STAGE + v_at, vst1 = row_on1_from_even<D>(vst);
            if (turn) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const uint4 x = ptx::lds128(w_in + (i & 1) * C::W_BYTES + rb * 512);
                    wf[rb][0] = x.x, wf[rb][1] = x.y, wf[rb][2] = x.z, wf[rb][3] = x.w;
                }
            }
            uint32_t v[4][NB / 4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t at = (k & 1 ? vst1 : vst) + (k >> 1) * rows_on8<D>();
                if (D == 128) {
                    const uint2 x = ptx::lds64(at);
                    v[k][0] = x.x, v[k][NB / 4 - 1] = x.y;
                } else {
                    v[k][0] = ptx::lds32(at);
                }
            }
#pragma unroll
            for (int i4 = 0; i4 < NB / 4; ++i4) {
                uint32_t p[2][2];                            // positions (0, 1) and (2, 3): channels 0 1 and 2 3 of this word, position by position
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
        slot = slot + 1 == C::STAGES ? 0 : slot + 1;
    }
    cp_async_wait<0>();
    __syncthreads();                                         // the rings are free: they take the pairs' sums

    // ---- the two pairs' sums, joined
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
            // columns 2 t and 2 t + 1 of product j are channels NB 2 t + j and NB (2 t + 1) + j of the half
            float* dst = join + (pair * C::ROWS + r) * C::O_PITCH + side * (D / 2) + NB * 2 * t;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int j = 0; j < NB; j += 4)
                    *reinterpret_cast<float4*>(dst + c * NB + j) = make_float4(o[rb][j][2 * h + c], o[rb][j + 1][2 * h + c], o[rb][j + 2][2 * h + c], o[rb][j + 3][2 * h + c]);
            }
        }
    }
    __syncthreads();
    const size_t unit = (size_t)blockIdx.z * a.slices + slice;
    for (int idx = tid; idx < C::ROWS * (D / 4); idx += AR_WARPS * 32) {
        const int r = idx / (D / 4), d = (idx % (D / 4)) * 4;
        if (r >= rows) break;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < 2; ++w) m = fmaxf(m, ml[2 * w * C::ROWS + r].x);
        float l = 0.0f;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float2 one = ml[2 * w * C::ROWS + r], two = ml[(2 * w + 1) * C::ROWS + r];
            // (a row without a reference has no weights, or is not a number in all of them)
            const float f = one.x == -INFINITY ? 1.0f : kv8_ex2(one.x - m);
            const float4 y = *reinterpret_cast<const float4*>(join + (w * C::ROWS + r) * C::O_PITCH + d);
            l = fmaf(f, one.y + two.y, l);
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
            const int token = r / a.rep, head = kv_head * a.rep + r - token * a.rep;
            uint2* dst = reinterpret_cast<uint2*>(a.out + (((long long)seq * a.T + token) * a.q_heads + head) * D + d);
            *dst = make_uint2(ptx::pack_bf16x2(x.x * inv, x.y * inv), ptx::pack_bf16x2(x.z * inv, x.w * inv));
        }
    }
}

// W warps per (token, head) row, each with its share of the slices: sums weighted by how far their reference is below the largest.  With four
// warps per row one decode token's 32 slices take one round of loads (one warp per row took most of 6 us); up to eight slices, and so with many
// rows, one warp has them under way at once.  Attention altogether, one or four warps a row: 32 slices 10.6 and 8.4 us, 18 slices 34.3 and 27.4;
// 6 slices of 200 tokens x 28 heads 24.4 and 33.8.
template <int D, int W>
__global__ void __launch_bounds__(128)
kv8_combine_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, uint16_t* __restrict__ out, long long total_rows, int T,
                   int q_heads, int kv_heads, int rep, int tiles, int slices, int tile_rows) {
    constexpr int V = D / 32;
    __shared__ float sums[W == 1 ? 1 : W][W == 1 ? 1 : D];
    __shared__ float2 refs[W];
    ptx::pdl_launch_dependents();
    const int warp = W == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long row = W == 1 ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= total_rows) return;
    const int head = (int)(row % q_heads);
    const long long at = row / q_heads;                      // seq T + token
    const int token = (int)(at % T), kv_head = head / rep;
    const long long r = (long long)token * rep + head - kv_head * rep;
    const size_t unit = (((size_t)(at / T) * kv_heads + kv_head) * tiles + (size_t)(r / tile_rows)) * slices;
    const size_t first = unit * tile_rows + (size_t)(r % tile_rows);
    ptx::pdl_wait();
    float m = -INFINITY, l = 0.0f, x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
    // eight slices at a time, all loads ahead of the first use
    constexpr int U = 8;
    for (int z0 = warp; z0 < slices; z0 += W * U) {
        float2 one[U];
        float y[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int z = z0 + W * u;
            one[u] = make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) y[u][i] = 0.0f;
            if (z < slices) {
                const size_t p = first + (size_t)z * tile_rows;
                one[u] = __ldcg(&part_ml[p]);
                const float2* src = reinterpret_cast<const float2*>(part_o + p * D + lane * V);
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float2 v = __ldcg(src + i / 2);
                    y[u][i] = v.x;
                    y[u][i + 1] = v.y;
                }
            }
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, one[u].x);
        const float back = m == -INFINITY ? 1.0f : kv8_ex2(m - top);
        m = top;
        l *= back;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] *= back;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (a slice without a reference has no weights, or is not a number in all of them)
            const float f = one[u].x == -INFINITY ? 1.0f : kv8_ex2(one[u].x - m);
            l = fmaf(f, one[u].y, l);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = fmaf(f, y[u][i], x[i]);
        }
    }
    if constexpr (W == 1) {
        const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
        uint32_t* dst = reinterpret_cast<uint32_t*>(out + row * D) + lane * (V / 2);
#pragma unroll
        for (int i = 0; i < V; i += 2) dst[i / 2] = ptx::pack_bf16x2(x[i] * inv, x[i + 1] * inv);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) sums[warp][lane * V + i] = x[i];
        if (lane == 0) refs[warp] = make_float2(m, l);
        __syncthreads();
        if (threadIdx.x >= D / 2) return;
        m = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, refs[w].x);
        float2 total = make_float2(0.0f, 0.0f);
        l = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = refs[w].x == -INFINITY ? 1.0f : kv8_ex2(refs[w].x - m);
            l = fmaf(f, refs[w].y, l);
            total.x = fmaf(f, sums[w][2 * threadIdx.x], total.x);
            total.y = fmaf(f, sums[w][2 * threadIdx.x + 1], total.y);
        }
        const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
        reinterpret_cast<uint32_t*>(out + row * D)[threadIdx.x] = ptx::pack_bf16x2(total.x * inv, total.y * inv);
    }
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
    cfg.gridDim = dim3((unsigned)a.slices, 1, (unsigned)(B * a.kv_heads));
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
    const long long total = (long long)B * a.T * a.q_heads;              // few: there are slices only where tiles are
    const bool one = a.slices <= 8;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(one ? (total + 3) / 4 : total), 1, 1);
    cfg.blockDim = dim3(128, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, one ? kv8_combine_kernel<D, 1> : kv8_combine_kernel<D, 4>, (const float*)a.part_o, (const float2*)a.part_ml, a.out,
                              total, a.T, a.q_heads, a.kv_heads, a.rep, a.tiles, a.slices, tile_rows);
}

}  // namespace

// Row tiles of 16 with four CTAs per SM, of 32 with three, of 256 with one: what is resident at once.
// Measured (8 key heads of 128, 1000, 4096 and 32749 positions): 16 rows 6.3, 9.7, 25.2 us as tiles of 16; 7.6, 11.3, 26.6 as tiles of 32; 10.8, 13.5, 40.1
// as tiles of 256; all for one sequence.  32 rows 8.2, 12.1, 27.6 as tiles of 32; 10.9, 13.4, 40.3 as tiles of 256, which take no longer for 64 rows (10.7, 13.5, 40.5).
static int ctas_per_sm(int rows) { return rows == 16 ? ArCfg<128, 1>::CTAS : (rows == 32 ? ArCfg<128, 2>::CTAS : 1); }

// Slices are a whole number per row tile, so CTAs leave places empty just above a divisor of them and run a second wave just above all of them: 8 key heads,
// 2000 positions each, draft blocks of 8 for 27, 28, 55 and 56 sequences 40, 59, 61 and 84 us; single tokens for 37, 38, 74 and 75 33, 53, 55 and 71; 16 tokens for 18
// and 19 sequences 38 and 70.  The number goes by the table's width, not by the limits, which are on the device: one token over 4096 positions 8.5 us with
// a table as wide, 8.9 with one 16 times as wide.
Kv8Plan kv8_plan(int B, int T, int q_heads, int kv_heads, long long max_keys, int sms) {
    Kv8Plan p;
    const long long rows = (long long)T * (q_heads / kv_heads);
    p.rows = rows <= 16 ? 16 : (rows <= 32 ? 32 : 256);
    p.tiles = (int)((rows + p.rows - 1) / p.rows);
    const long long units = (long long)B * kv_heads * p.tiles;
    long long s = (long long)ctas_per_sm(p.rows) * sms / units;
    // at least two chunks for each of a CTA's warps (with one, or four: one token over 500 positions 5.0 and 6.7 instead of 5.5 us, over 4096 8.7 and 8.9
    // instead of 8.5; a draft block of 8 over 4096 13.4 and 13.8 instead of 12.2), two steps of the tensor-memory kernel (with four of those a chunk of 200 tokens over 2900
    // positions takes 35.6 instead of 30.8 us, and equally long with a bound of 512; 100 tokens over 1000 24.8 instead of 21.7)
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
    a.scale_log2 = scale * KV8_LOG2_E;
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
