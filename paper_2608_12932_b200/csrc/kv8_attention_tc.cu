// Attention over the 8-bit key/value cache for many rows: chunks of new tokens, prompts (definition and number formats in
// kv8_attention.cuh).  The 5th-generation tensor cores take fp16 operands, so the codes are made fp16 on their way into shared
// memory, once for the 256 rows of a CTA.
//
// One CTA per (sequence, key head, tile of 256 rows, slice of the keys), 128 positions a step, two halves of 128 rows in turn:
//   S_h = Q_h K^T         both operands in shared memory (K-major, 128-byte swizzle), sums in tensor memory
//   O_h += W_h V          W_h = the weights, fp16, in tensor memory over the scores they came from; V [position][channel] as it is in
//                         the cache (an MN-major operand: nothing is transposed)
// While one half's products run, the other half's weights are formed.  Warps: two groups of four form the weights, a thread per row (the
// lane of tensor memory that it may read is its row); four convert codes; one fetches them with bulk copies, 64 positions of K or V at a time,
// into a ring ahead of the conversion (loads through the converting threads' registers instead: a causal prompt of 4096 in 252 us);
// one issues the products.
// All waits are bounded: a role that gives up sets the CTA's abort flag, on which the others leave, too.
//
// A step's products cost 2 x 128 x 128 x D x 2 multiply-adds (2048 cycles of the tensor pipe at D = 128), its 32768 exponentials as much of the
// special-function units, its operands and the conversion as much of shared memory's bandwidth: none of the three bounds it alone, and it takes 3000.
// A CTA's first and last product are 5 us apart from its beginning and end.  Causal prompt of 4096, 32 heads of 128 over 8 key heads: 147 us, 935 TFLOP/s,
// in a graph of calls (156 us as a call by itself), at the 1.55 GHz that the power limit leaves; 200 tokens x 28 heads over 2900 positions 24.3 us; 4 views of 256 tokens over 4096 positions 70.5 us (as long as
// its longest tiles, on 128 of the SMs).
#include "kv8_attention.cuh"
#include "quant_common.cuh"

namespace w4a8 {
namespace {

constexpr int TC_THREADS = 512, TC_ROWS = 256, TC_KEYS = 128;
constexpr int TC_WARP_CVT0 = 8, TC_WARP_MMA = 12, TC_WARP_FETCH = 13;
constexpr int TC_META = 8;                                    // ring of the steps' block scales

template <int D>
struct TcCfg {
    static constexpr int PANEL = 128 * 128;                   // 128 rows of 64 halves
    static constexpr int PANELS = D / 64;
    static constexpr int TILE = PANEL * PANELS;
    static constexpr int Q_OFF = 0, K_OFF = 2 * TILE, V_OFF = 4 * TILE;
    static constexpr int RAW = 64 * D, SLOTS = D == 128 ? 4 : 8;  // codes of 64 positions; K, K, V, V of a step in turn
    static constexpr int RAW_OFF = 6 * TILE;
    static constexpr int BAR_OFF = RAW_OFF + SLOTS * RAW;
    // barriers: K and V stages full and empty, scores of a half and its weights in two parts, Q of a half, O of a half complete, scales, raw codes full and
    // empty, end
    static constexpr int KF = 0, KE = 2, VF = 4, VE = 6, SF = 8, PF = 10, QF = 14, OF = 16, MF = 18, RF = MF + TC_META, RE = RF + SLOTS, FINAL = RE + SLOTS, NUM_BARS = FINAL + 1;
    static constexpr int META_OFF = (BAR_OFF + NUM_BARS * 8 + 15) & ~15;        // [TC_META][8] float4: key scale, log2 of the value scale, its reciprocal
    static constexpr int MISC_OFF = META_OFF + TC_META * 8 * 16;                // tensor-memory base, abort flag, longest limit
    static constexpr int POISON_OFF = MISC_OFF + 16;                            // per warp of 32 rows, a bit for each that is not a number
    static constexpr int SMEM = POISON_OFF + 32 + 1024;
    static constexpr uint32_t S_COL = 0, O_COL = 256;                            // tensor memory: scores 2 x 128 columns, sums 2 x 128
};

template <int D>
__global__ void __launch_bounds__(TC_THREADS, 1)
kv8_attend_tiles_kernel(const __grid_constant__ AttendArgs a) {
    using C = TcCfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - ptx::smem_u32(smem_raw));
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    ptx::pdl_launch_dependents();
    auto bar = [&](int i) { return base + C::BAR_OFF + 8 * i; };
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(smem + C::MISC_OFF);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + C::MISC_OFF + 4);
    int* longest_at = reinterpret_cast<int*>(smem + C::MISC_OFF + 8);
    if (warp == TC_WARP_MMA) {
        if (lane == 0) {
            *abort_flag = 0;
            *longest_at = 0;
        }
        // by four warps: K and V stages full, weights in place, Q in place, raw codes converted; the others by one
        for (int i = lane; i < C::NUM_BARS; i += 32) {
            const bool four = (i >= C::KF && i < C::KE) || (i >= C::VF && i < C::VE) || (i >= C::PF && i < C::OF) || (i >= C::RE && i < C::FINAL);
            ptx::mbar_init(bar(i), four ? 4 : 1);
        }
        ptx::fence_mbar_init();
        __syncwarp();
        ptx::tmem_alloc(base + C::MISC_OFF, 512);
        ptx::tmem_relinquish();
    }
    // late tiles first: under a causal limit they are the longest
    const int units = gridDim.x / (a.tiles * a.slices);
    const int ts = blockIdx.x / units, unit = blockIdx.x - ts * units;
    const int tile = a.tiles - 1 - ts / a.slices, slice = ts % a.slices;
    const int seq = unit / a.kv_heads, kv_head = unit - seq * a.kv_heads;
    const int rows = a.T * a.rep, row0 = tile * TC_ROWS;
    const int halves = rows - row0 > 128 ? 2 : 1;
    const int capacity = (int)min((long long)a.table_width << a.log2_block, 0x7FFFFF00ll);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_holder;
    ptx::pdl_wait();

    int limit = 0;
    const int row = row0 + tid;                               // threads 0..255: this thread's row
    long long q_at = -1, out_at = -1;                         // where it begins in q and in out
    if (tid < TC_ROWS && row < rows) {
        const int token = row / a.rep, head = kv_head * a.rep + row - token * a.rep;
        q_at = ((long long)seq * a.T + token) * a.q_stride + (long long)head * D;
        out_at = (((long long)seq * a.T + token) * a.q_heads + head) * D;
        limit = min(max(__ldcg(a.limits + (long long)seq * a.T + token), 0), capacity);
    }
    if (tid < TC_ROWS) {
        const int top = __reduce_max_sync(0xFFFFFFFFu, limit);
        if (lane == 0 && top) atomicMax(longest_at, top);
    }
    __syncthreads();
    const int longest = *longest_at;
    const int tiles_n = (int)(((long long)longest + TC_KEYS - 1) / TC_KEYS);
    const int t_lo = (int)((long long)slice * tiles_n / a.slices), n = (int)((long long)(slice + 1) * tiles_n / a.slices) - t_lo;

    if (warp < TC_WARP_CVT0) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int h = warp >> 2;
        if (h < halves) {
            // ---- this warp's rows of q, scaled by powers of two and rounded to fp16, into the half's operand tile.  D / 8 lanes read a row: with a row per
            // lane the loads take a line each, 4096 of them in a CTA (and as many stores at its end): a prompt of 4096 in 169 instead of 156 us.
            constexpr int PIECES = D / 8, PER = 32 / PIECES;  // 16-byte pieces of a row; rows per load
            const int piece = lane % PIECES, r0 = (warp & 3) * 32;
            float factor = 0.0f;
            // A row with an infinity or not-a-number is walked as zeros and made not a number at the end, if it saw a key.  Shared memory keeps which rows
            // these are (a register kept for it beside the walk: the prompt takes 150 instead of 147.5 us).
            uint32_t* poisoned_at = reinterpret_cast<uint32_t*>(smem + C::POISON_OFF) + warp;
            {
                uint32_t mine = 0;                            // largest magnitude (bf16 bits) of this thread's row
                uint4 w[PIECES];
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    const long long from = __shfl_sync(0xFFFFFFFFu, q_at, PER * i + lane / PIECES);
                    w[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (from >= 0) w[i] = __ldcg(reinterpret_cast<const uint4*>(a.q + from) + piece);
                }
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    uint32_t run = absmax_bits_bf16x8(w[i], 0u);
                    run = max(run & 0xFFFFu, run >> 16);
#pragma unroll
                    for (int o = PIECES / 2; o; o >>= 1) run = max(run, __shfl_xor_sync(0xFFFFFFFFu, run, o));
                    const int e = kv8_row_exp(run);
                    const float up = kv8_pow2(e);
                    const uint32_t top = __shfl_sync(0xFFFFFFFFu, run, (lane % PER) * PIECES);
                    if (lane / PER == i) mine = top;
                    const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                    uint32_t y[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = kv8_pack_half2(__uint_as_float(x[k] << 16) * up, __uint_as_float(x[k] & 0xFFFF0000u) * up);
                    const int r = r0 + PER * i + lane / PIECES;
                    ptx::sts128u(base + C::Q_OFF + h * C::TILE + (piece >> 3) * C::PANEL + r * 128 + (((piece & 7) ^ (r & 7)) << 4), y[0], y[1], y[2], y[3]);
                }
                factor = a.scale_log2 * kv8_pow2(-kv8_row_exp(mine));
                const bool poisoned = mine >= 0x7F80u;
                const uint32_t which = __ballot_sync(0xFFFFFFFFu, poisoned);
                if (lane == 0) *poisoned_at = which;
                __syncwarp();
                if (poisoned) {
#pragma unroll 1
                    for (int i = 0; i < PIECES; ++i) ptx::sts128u(base + C::Q_OFF + h * C::TILE + (i >> 3) * C::PANEL + (r0 + lane) * 128 + ((i & 7) << 4), 0u, 0u, 0u, 0u);
                }
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar(C::QF + h));
            }
            const int shortest = __reduce_min_sync(0xFFFFFFFFu, row < rows ? limit : 0x7FFFFFFF);
            const uint32_t lanes = (uint32_t)(warp & 3) << 21;                  // tensor-memory lanes of this warp
            const uint32_t s_col = tmem + lanes + C::S_COL + h * 128, o_col = tmem + lanes + C::O_COL + h * 128;
            float ref = -INFINITY, sum = 0.0f;
            bool ok = true;
            for (int j = 0; j < n; ++j) {
                if (!(ok = ptx::warp_mbar_wait_suspend(bar(C::MF + j % TC_META), (j / TC_META) & 1, abort_flag))) break;
                if (!(ok = ptx::warp_mbar_wait_suspend(bar(C::SF + h), j & 1, abort_flag))) break;
                ptx::tc_fence_after_sync();
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32(s_col + 32 * c, s[c]);
                const uint32_t meta = base + C::META_OFF + (j % TC_META) * 128;
                const int key0 = (t_lo + j) * TC_KEYS;
                const float off = ref == -INFINITY ? 0.0f : KV8_W_EXP - ref;
                uint64_t f2[8], add2[8];
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                    const uint2 m = ptx::lds64(meta + 16 * b);
                    const uint32_t f = __float_as_uint(factor * __uint_as_float(m.x)), add = __float_as_uint(__uint_as_float(m.y) + off);
                    f2[b] = ptx::pack2(f, f);
                    add2[b] = ptx::pack2(add, add);
                }
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 128; i += 2) {
                    uint32_t &x = s[i >> 5][i & 31], &y = s[i >> 5][(i & 31) + 1];
                    const float2 z = ptx::unpack2(ptx::fma2(ptx::pack2(x, y), f2[i >> 4], add2[i >> 4]));
                    x = __float_as_uint(z.x);
                    y = __float_as_uint(z.y);
                }
                if (key0 + TC_KEYS > shortest) {
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (key0 + i >= limit) s[i >> 5][i & 31] = __float_as_uint(-INFINITY);
                }
                float tops[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    tops[c] = __uint_as_float(s[c][0]);
#pragma unroll
                    for (int i = 1; i < 31; i += 2) tops[c] = fmaxf(tops[c], fmaxf(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1])));
                    tops[c] = fmaxf(tops[c], __uint_as_float(s[c][31]));
                }
                const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                const bool past = top > (ref == -INFINITY ? -INFINITY : KV8_W_EXP + KV8_SLACK);
                if (__any_sync(0xFFFFFFFFu, past)) {
                    // (a step's scores are complete only when the products of the step before are: O is at rest)
                    float f = 1.0f, shift = 0.0f;
                    if (past) {
                        const float now = top - off;
                        f = ref == -INFINITY ? 0.0f : kv8_ex2(ref - now);
                        ref = now;
                        shift = KV8_W_EXP - ref - off;
                        sum = now == INFINITY ? NAN : sum * f;                  // an infinite score: not a number from here on
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i >> 5][i & 31] = __float_as_uint(__uint_as_float(s[i >> 5][i & 31]) + shift);
                    if (j > 0) {
#pragma unroll
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            ptx::tmem_ld_32x16(o_col + c, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            ptx::tmem_st_32x8(o_col + c, o[0], o[1], o[2], o[3], o[4], o[5], o[6], o[7]);
                            ptx::tmem_st_32x8(o_col + c + 8, o[8], o[9], o[10], o[11], o[12], o[13], o[14], o[15]);
                        }
                    }
                }
                // ---- the weights, handed over 64 positions at a time (a quarter of the exponentials by a polynomial on the FMA pipe: 147 -> 156 us for the
                // prompt; the special-function unit is not what the warps wait for)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t p[32];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        uint64_t g = 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int at = (4 * c + b) * 16 + 2 * i;
                            const float x = __uint_as_float(s[at >> 5][at & 31]), y = __uint_as_float(s[at >> 5][(at & 31) + 1]);
                            const float2 w = make_float2(kv8_ex2(x), kv8_ex2(y));
                            g = ptx::add2(g, ptx::pack2(__float_as_uint(w.x), __float_as_uint(w.y)));
                            p[b * 8 + i] = kv8_pack_half2(w.x, w.y);
                        }
                        const float2 g2 = ptx::unpack2(g);
                        sum = fmaf(g2.x + g2.y, __uint_as_float(ptx::lds32(meta + 16 * (4 * c + b) + 8)), sum);
                    }
                    ptx::tmem_st_32x32(s_col + 32 * c, p);
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(C::PF + 2 * h + c));
                }
            }
            // ---- the result: a row per thread out of tensor memory, through this warp's rows of the operand tile (no product reads it any more) to whole
            // lines in global memory
            if (ok && n > 0) ok = ptx::warp_mbar_wait_suspend(bar(C::OF + h), 0, abort_flag);
            if (ok) {
                ptx::tc_fence_after_sync();
                if ((*poisoned_at >> lane & 1u) && sum != 0.0f) sum = NAN;
                const float inv = sum == 0.0f ? 0.0f : __fdividef(1.0f, sum);
                const size_t part = (((size_t)unit * a.tiles + tile) * a.slices + slice) * TC_ROWS + (size_t)(row - row0);
                const uint32_t own = base + C::Q_OFF + h * C::TILE + r0 * 128;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    if (n > 0) {
                        ptx::tmem_ld_32x32(o_col + c, o);
                        ptx::tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0;
                    }
                    if (a.slices > 1) {
                        // 32 channels of 32 rows as they are: eight lanes write a row's 128 bytes
#pragma unroll
                        for (int i = 0; i < 8; ++i) ptx::sts128u(own + lane * 128 + ((i ^ (lane & 7)) << 4), o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int r = 4 * i + (lane >> 3);
                            const uint4 x = ptx::lds128(own + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                            if (row - lane + r < rows) *reinterpret_cast<uint4*>(a.part_o + (part - lane + r) * D + c + 4 * (lane & 7)) = x;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t y[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                y[k] = ptx::pack_bf16x2(__uint_as_float(o[8 * i + 2 * k]) * inv, __uint_as_float(o[8 * i + 2 * k + 1]) * inv);
                            const int p = c / 8 + i;
                            ptx::sts128u(own + (p >> 3) * C::PANEL + lane * 128 + (((p & 7) ^ (lane & 7)) << 4), y[0], y[1], y[2], y[3]);
                        }
                    }
                    __syncwarp();                            // ahead of the next load of tensor memory, and of the reads or writes of the operand tile
                }
                if (a.slices == 1) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        const int r = PER * i + lane / PIECES;
                        const long long to = __shfl_sync(0xFFFFFFFFu, out_at, r);
                        const uint4 x = ptx::lds128(own + (piece >> 3) * C::PANEL + r * 128 + (((piece & 7) ^ (r & 7)) << 4));
                        if (to >= 0) *(reinterpret_cast<uint4*>(a.out + to) + piece) = x;
                    }
                }
                if (a.slices > 1 && row < rows) a.part_ml[part] = make_float2(ref, sum);
            }
        }
    } else if (warp < TC_WARP_MMA) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // ---- codes -> fp16 operand tiles, 16 codes (a piece) of a key at a time.  Eight neighbouring lanes take eight different pieces
        // of 128 bytes, of two keys, so that neither the reads nor the stores (whose places are swizzled by the key) meet in a bank.
        constexpr int L = D / 32;                             // pieces per thread and 64 positions
        const int wv = warp - TC_WARP_CVT0;
        const int piece = D == 128 ? lane & 7 : lane & 3;
        const int key0 = wv * 16 + (D == 128 ? ((lane >> 4) & 1) * 2 + (((lane >> 2) ^ (lane >> 3)) & 1) : lane >> 2);
        constexpr int STEP = D == 128 ? 4 : 8;                // keys from one piece of a thread to its next
        const uint32_t from = key0 * D + piece * 16;
        const uint32_t to = (piece >> 2) * C::PANEL + key0 * 128 + (((2 * (piece & 3)) ^ (key0 & 7)) << 4);
        auto convert = [&](uint32_t src, uint32_t dst) {
            uint4 x[L];
#pragma unroll
            for (int i = 0; i < L; ++i) x[i] = ptx::lds128(src + from + i * STEP * D);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const uint32_t w[4] = {x[i].x ^ 0x80808080u, x[i].y ^ 0x80808080u, x[i].z ^ 0x80808080u, x[i].w ^ 0x80808080u};
                const uint32_t at = (dst + to + i * STEP * 128) ^ (D == 128 && (i & 1) ? 64u : 0u);      // (four keys on: bit 2 of the swizzle)
                ptx::sts128u(at, kv8_half2(w[0], 0x4140), kv8_half2(w[0], 0x4342), kv8_half2(w[1], 0x4140), kv8_half2(w[1], 0x4342));
                ptx::sts128u(at ^ 16u, kv8_half2(w[2], 0x4140), kv8_half2(w[2], 0x4342), kv8_half2(w[3], 0x4140), kv8_half2(w[3], 0x4342));
            }
        };
        bool ok = true;
        for (int j = 0; j < n && ok; ++j) {
            const int st = j & 1;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                if (!(ok = ptx::warp_mbar_wait_suspend(bar((kv ? C::VE : C::KE) + st), ((j >> 1) & 1) ^ 1, abort_flag))) break;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int at = 4 * j + 2 * kv + q, slot = at % C::SLOTS;
                    if (!(ok = ptx::warp_mbar_wait_suspend(bar(C::RF + slot), (at / C::SLOTS) & 1, abort_flag))) break;
                    convert(base + C::RAW_OFF + slot * C::RAW, base + (kv ? C::V_OFF : C::K_OFF) + st * C::TILE + q * 64 * 128);
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(C::RE + slot));
                }
                if (!ok) break;
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar((kv ? C::VF : C::KF) + st));
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == TC_WARP_MMA && n > 0) {
            // ---- products: the warp walks the loop, one elected lane issues
            const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
            constexpr uint32_t IDESC_S = ptx::idesc_f16(128, TC_KEYS, false), IDESC_O = ptx::idesc_f16(128, D, true);
            auto scores = [&](int h, int st) {
                const uint64_t q0 = ptx::smem_desc_k_sw128(base + C::Q_OFF + h * C::TILE), k0 = ptx::smem_desc_k_sw128(base + C::K_OFF + st * C::TILE);
                if (ptx::elect_one()) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint64_t at = (uint64_t)((i >> 2) * (C::PANEL / 16) + (i & 3) * 2);
                        ptx::mma_f16_ss(tm + C::S_COL + h * 128, q0 + at, k0 + at, IDESC_S, i > 0);
                    }
                    ptx::tc_commit(bar(C::SF + h));
                    if (h == halves - 1) ptx::tc_commit(bar(C::KE + st));
                }
                __syncwarp();
            };
            bool ok = true;
            for (int h = 0; h < halves && ok; ++h) {
                ok = ptx::mbar_wait_suspend(bar(C::QF + h), 0, abort_flag);
                if (ok && h == 0) ok = ptx::mbar_wait_suspend(bar(C::KF), 0, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (ok) {
                    ptx::tc_fence_after_sync();
                    scores(h, 0);
                }
            }
            for (int j = 0; j < n && ok; ++j) {
                const int st = j & 1;
                for (int h = 0; h < halves && ok; ++h) {
                    if (h == 0) ok = ptx::mbar_wait_suspend(bar(C::VF + st), (j >> 1) & 1, abort_flag);
                    const uint64_t v0 = ptx::smem_desc_mn_sw128(base + C::V_OFF + st * C::TILE, C::PANEL);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        ok = ok && ptx::mbar_wait_suspend(bar(C::PF + 2 * h + c), j & 1, abort_flag);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        ptx::tc_fence_after_sync();
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int i = 4 * c; i < 4 * c + 4; ++i)
                                ptx::mma_f16_ts(tm + C::O_COL + h * 128, tm + C::S_COL + h * 128 + 8 * i, v0 + (uint64_t)(i * 128), IDESC_O, j > 0 || i > 0);
                            if (c == 1 && h == halves - 1) ptx::tc_commit(bar(C::VE + st));
                            if (c == 1 && j == n - 1) ptx::tc_commit(bar(C::OF + h));
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (j + 1 < n) {
                        if (h == 0) ok = ptx::mbar_wait_suspend(bar(C::KF + (st ^ 1)), ((j + 1) >> 1) & 1, abort_flag);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        ptx::tc_fence_after_sync();
                        scores(h, st ^ 1);
                    }
                }
            }
            if (ptx::elect_one()) ptx::tc_commit(bar(C::FINAL));
            __syncwarp();
            ptx::mbar_wait(bar(C::FINAL), 0, abort_flag);    // nothing may still be executing when tensor memory is freed
        } else if (warp == TC_WARP_FETCH) {
            // ---- codes and scales.  Lane l holds block number and scales of positions 16 (l & 7) .. + 15 of step 4 i + (l >> 3), for these four
            // steps and the next four.
            struct Meta { int number; uint32_t ks, vs; };
            const int32_t* table = a.table + (size_t)seq * a.table_width;
            auto meta_of = [&](int j0) -> Meta {
                Meta m = {-1, 0u, 0u};
                const int j = j0 + (lane >> 3);
                const long long pos = (long long)(t_lo + j) * TC_KEYS + 16 * (lane & 7);
                if (j < n && pos < longest) {
                    const int number = __ldcg(table + (pos >> a.log2_block));
                    if ((unsigned)number < (unsigned)a.num_blocks) {
                        const size_t at = (size_t)number * a.kv_heads + kv_head;
                        m.number = number;
                        m.ks = __ldcg(a.k_scales + at);
                        m.vs = __ldcg(a.v_scales + at);
                    } else {
                        flag_index(a.status);                // positions of a block that does not exist count as not there
                    }
                }
                return m;
            };
            const int per = min(64, 1 << a.log2_block), copies = 64 / per;       // positions per copy, copies per 64 positions
            Meta cur = meta_of(0), nxt = meta_of(4);
            bool ok = true;
            for (int j = 0; j < n && ok; ++j) {
                if (j && (j & 3) == 0) {
                    cur = nxt;
                    nxt = meta_of(j + 4);
                }
                for (int q = 0; q < 4; ++q) {
                    const int at = 4 * j + q, slot = at % C::SLOTS, first = (j & 3) * 8 + (q & 1) * 4;
                    if (!(ok = ptx::warp_mbar_wait_suspend(bar(C::RE + slot), ((at / C::SLOTS) & 1) ^ 1, abort_flag))) break;
                    // lane i < copies: the i-th copy
                    const int number = __shfl_sync(0xFFFFFFFFu, cur.number, first + ((lane * per) >> 4 & 3));
                    const bool mine = lane < copies && number >= 0;
                    const uint32_t bytes = (uint32_t)(__popc(__ballot_sync(0xFFFFFFFFu, mine)) * per * D);
                    if (lane == 0) ptx::mbar_arrive_expect_tx(bar(C::RF + slot), bytes);
                    __syncwarp();
                    if (mine) {
                        const int inside = ((t_lo + j) * TC_KEYS + (q & 1) * 64 + lane * per) & ((1 << a.log2_block) - 1);
                        const int8_t* src = (q < 2 ? a.k_codes : a.v_codes) + ((((size_t)number * a.kv_heads + kv_head) << a.log2_block) + inside) * D;
                        ptx::bulk_g2s(base + C::RAW_OFF + slot * C::RAW + lane * per * D, src, per * D, bar(C::RF + slot));
                    }
                    __syncwarp();
                    if (q == 0) {
                        // After the copies, which need not wait for the scales.  The slot of the raw codes was free: the step that used it (one or two
                        // ago) is being converted, so the scores of the second before that are complete, which follow the weights of the third: scales
                        // of five steps ago are no longer read.
                        if ((lane >> 3) == (j & 3)) {
                            float lg, inv;
                            kv8_value_scale(cur.vs, lg, inv);
                            if (cur.number < 0) lg = -INFINITY, inv = 0.0f;
                            ptx::sts128(base + C::META_OFF + (j % TC_META) * 128 + (lane & 7) * 16,
                                        make_float4(__half2float(__ushort_as_half((uint16_t)cur.ks)), lg, inv, 0.0f));
                        }
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(bar(C::MF + j % TC_META));
                    }
                }
            }
            if (!ok) {   // let copies already in flight land before shared memory is released
                const uint64_t t0 = ptx::globaltimer_ns();
                while (ptx::globaltimer_ns() - t0 < 200000ull) {}
            }
        }
    }
    if (*abort_flag && lane == 0) atomicExch(a.status, (uint32_t)W4A8_ERR_TIMEOUT);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == TC_WARP_MMA) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

template <int D>
cudaError_t launch_tiles(const AttendArgs& a, int B, cudaStream_t stream) {
    using C = TcCfg<D>;
    static_assert(C::SMEM <= 227 * 1024, "shared memory");
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(kv8_attend_tiles_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.tiles * (unsigned)a.slices * (unsigned)(B * a.kv_heads), 1, 1);
    cfg.blockDim = dim3(TC_THREADS, 1, 1);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv8_attend_tiles_kernel<D>, a);
}

}  // namespace

cudaError_t launch_kv8_tiles(const AttendArgs& a, int B, int dim, cudaStream_t stream) {
    return dim == 128 ? launch_tiles<128>(a, B, stream) : launch_tiles<64>(a, B, stream);
}

}  // namespace w4a8
