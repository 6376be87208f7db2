"""numpy statement of what a decoder layer does between its quantised linears: residual addition with root-mean-square norm, the append
to a key/value cache held in 8 bits, and attention over it.  Test infrastructure only, like the rest of this package; loops over
sequences, heads and blocks, everything else in fp64."""
import numpy as np

from oracle.w4a8_oracle import FP16_MAX, bf16_bits_to_f64, f64_to_bf16_bits, f64_to_fp16_bits, fp16_bits_to_f64


def add_rmsnorm(x_bits, residual_bits, weight_bits, eps):
    """s = bf16(x + r) (x itself without a residual), h = bf16(s w / sqrt(mean s^2 + eps)): (s bits, h in fp64, h bits)."""
    s_bits = x_bits if residual_bits is None else f64_to_bf16_bits(bf16_bits_to_f64(x_bits) + bf16_bits_to_f64(residual_bits))
    s = bf16_bits_to_f64(s_bits)
    h = s * bf16_bits_to_f64(weight_bits)[None, :] / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    return s_bits, h, f64_to_bf16_bits(h)


def kv8_append(codes, scales, x_bits, table, start, count):
    """Appends x [B, T, heads, dim] (bf16 bits) to codes int8 [blocks, heads, block, dim], scales fp16 bits [blocks, heads], both in
    place: token i of sequence b goes to position start[b] + i for i < count[b].  Positions whose block is not there are left out."""
    B, T, heads, _ = x_bits.shape
    block, width = codes.shape[2], table.shape[1]
    for b in range(B):
        n = min(max(int(count[b]), 0), T)
        if int(start[b]) < 0:
            continue
        i = 0
        while i < n:
            pos = int(start[b]) + i
            slot, index = pos % block, pos // block
            take = min(block - slot, n - i)
            number = int(table[b, index]) if index < width else -1
            if 0 <= number < codes.shape[0]:
                for h in range(heads):
                    x = bf16_bits_to_f64(x_bits[b, i:i + take, h])
                    old = fp16_bits_to_f64(scales[number, h]) if slot else 0.0
                    new = max(float(old), float(fp16_bits_to_f64(f64_to_fp16_bits(np.minimum(np.abs(x).max() / 127.0, FP16_MAX)))))
                    if new != old:
                        codes[number, h, :slot] = np.clip(np.rint(codes[number, h, :slot].astype(np.float64) * old / new), -127, 127)
                    codes[number, h, slot:slot + take] = np.clip(np.rint(x / new), -127, 127) if new else 0
                    scales[number, h] = f64_to_fp16_bits(np.float64(new))
            i += take


def kv8_values(codes, scales, table_row, head, length):
    """Positions 0 .. length - 1 of one sequence and head, [length, dim] fp64; the second result says which of them are there."""
    block = codes.shape[2]
    out, there = np.zeros((length, codes.shape[3])), np.zeros(length, dtype=bool)
    for p0 in range(0, length, block):
        number, n = int(table_row[p0 // block]), min(block, length - p0)
        if 0 <= number < codes.shape[0]:
            out[p0:p0 + n] = codes[number, head, :n].astype(np.float64) * fp16_bits_to_f64(scales[number, head])
            there[p0:p0 + n] = True
    return out, there


def kv8_attention(q_bits, k_codes, k_scales, v_codes, v_scales, table, limits, scale):
    """out[b, t, h, :] in fp64 for q [B, T, q_heads, dim] (bf16 bits): softmax attention over the leading limits[b, t] positions, zero
    for a row that sees none.  Also, per output element, what an error bound is made of: `spread` = sum_j p_j |v_j| (p normalised),
    `tail` = max_j p_j |scale of v_j| 127 (what one weight can carry), and per row `size` = the largest sum_d |q_d k_jd| scale and the number of keys."""
    B, T, q_heads, dim = q_bits.shape
    heads = k_codes.shape[1]
    capacity = table.shape[1] * k_codes.shape[2]
    out = np.zeros((B, T, q_heads, dim))
    spread, tail, size = np.zeros_like(out), np.zeros((B, T, q_heads, 1)), np.zeros((B, T, q_heads, 1))
    q = bf16_bits_to_f64(q_bits)
    for b in range(B):
        limit = np.clip(np.asarray(limits[b], dtype=np.int64), 0, capacity)
        length = int(limit.max()) if T else 0
        if not length:
            continue
        for g in range(heads):
            k, there = kv8_values(k_codes, k_scales, table[b], g, length)
            v, _ = kv8_values(v_codes, v_scales, table[b], g, length)
            top_v = np.abs(v).max(axis=1)
            seen = (np.arange(length)[None, :] < limit[:, None]) & there[None, :]
            for h in range(g * (q_heads // heads), (g + 1) * (q_heads // heads)):
                x = np.where(seen, q[b, :, h] @ k.T * scale, -np.inf)
                m = x.max(axis=1, keepdims=True)
                p = np.exp(x - np.where(np.isinf(m), 0.0, m))
                total = p.sum(axis=1, keepdims=True)
                p = p / np.where(total > 0, total, 1.0)
                out[b, :, h], spread[b, :, h] = p @ v, p @ np.abs(v)
                tail[b, :, h, 0] = (p * top_v).max(axis=1)
                size[b, :, h, 0] = np.where(seen, np.abs(q[b, :, h]) @ np.abs(k).T, 0.0).max(axis=1) * abs(scale)
    return out, spread, tail, size


def kv8_attention_band(out, spread, tail, size, keys, dim):
    """How far a kernel may be from kv8_attention: half a bf16 step of the result (2^-8); a weight's rounding to fp16 (2^-11) and the
    error of its exponent, in nats, twice (numerator and denominator): a score is an fp32 sum of `dim` products, off by at most
    (dim + 8) 2^-23 of the sum of their sizes, 2^-23 a step to allow for truncating adders; its scaling, the shift by the reference
    and the fast exponential add 2^-20; and weights too small for fp16's full precision, 2^-32 of the largest (which is at least 2^-8 of
    one that the fp32 sums still hold) each, times the number of keys."""
    exponent = 2.0 * (size * (dim + 8) * 2.0 ** -23 + (1.0 + size) * 2.0 ** -20)
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + exponent) * 1.01 * spread + keys * 2.0 ** -24 * tail + 1e-30
