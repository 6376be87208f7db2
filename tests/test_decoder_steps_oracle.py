"""Pins for the oracle of the steps between the quantised linears (norm, 8-bit cache, attention): hand-worked values, reductions to
textbook forms, and the properties that the definitions must have."""
import numpy as np

from oracle import decoder_steps as ds
from oracle import streaming as so
from oracle import w4a8_oracle as onp
from paper_2608_12932_b200 import binding as B
from paper_2608_12932_b200 import workload as wl


def bf16(a):
    return wl.f32_to_bf16_bits(np.asarray(a, dtype=np.float32))


def test_norm_hand_worked_example():
    # s = (3, 4, 0, 0): mean square 25 / 4, root 2.5; h = s w / 2.5
    s, h, h_bits = ds.add_rmsnorm(bf16([[1.0, 1.0, -2.0, 0.5]]), bf16([[2.0, 3.0, 2.0, -0.5]]), bf16([1.0, 0.5, 7.0, 7.0]), 0.0)
    assert np.array_equal(s, bf16([[3.0, 4.0, 0.0, 0.0]]))
    assert np.allclose(h, [[1.2, 0.8, 0.0, 0.0]], rtol=1e-15) and np.array_equal(h_bits, bf16([[1.2, 0.8, 0.0, 0.0]]))
    # a power of two on the stream changes nothing without eps, and unit weights give rows of unit mean square
    rng = np.random.default_rng(3)
    x = bf16(rng.standard_normal((5, 256)))
    one = bf16(np.ones(256))
    a = ds.add_rmsnorm(x, None, one, 0.0)[1]
    assert np.allclose((a * a).mean(axis=1), 1.0, rtol=1e-13)
    assert np.array_equal(ds.add_rmsnorm(bf16(onp.bf16_bits_to_f64(x) * 8), None, one, 0.0)[1], a)


def test_append_hand_worked_example():
    codes, scales = np.full((2, 1, 16, 64), 99, dtype=np.int8), np.zeros((2, 1), dtype=np.uint16)
    x = np.zeros((1, 3, 1, 64))
    x[0, 0, 0, :3] = [127.0, -63.5, 0.5]           # scale 1: codes 127, -64 (tie to even), 0 (tie to even)
    x[0, 1, 0, :2] = [254.0, 1.0]                  # scale 2 from here on: 127, 0 (0.5, tie)
    x[0, 2, 0, 0] = 6.0                            # behind a block's border in the last part
    table = np.array([[1, 0]])
    ds.kv8_append(codes, scales, bf16(x[:, :1]), table, [14], [1])
    assert codes[1, 0, 14, :4].tolist() == [127, -64, 0, 0] and onp.fp16_bits_to_f64(scales[1, 0]) == 1.0
    assert (codes[1, 0, :14] == 0).all() and (codes[1, 0, 15] == 99).all()          # in front: a block of scale 0 holds zeros; behind: untouched
    ds.kv8_append(codes, scales, bf16(x[:, 1:]), table, [15], [2])
    # the block's scale doubles: 127 -> 63.5 -> 64 (tie to even), -64 -> -32; the next position opens block 0
    assert codes[1, 0, 14, :3].tolist() == [64, -32, 0] and codes[1, 0, 15, :2].tolist() == [127, 0]
    assert onp.fp16_bits_to_f64(scales[1, 0]) == 2.0
    assert codes[0, 0, 0, 0] == 127 and (codes[0, 0, 1] == 99).all()
    before = codes.copy(), scales.copy()
    ds.kv8_append(codes, scales, bf16(x[:, 1:]), table, [15], [2])                   # again: nothing changes
    assert np.array_equal(codes, before[0]) and np.array_equal(scales, before[1])


def test_append_error_is_half_a_step_per_rounding():
    rng = np.random.default_rng(5)
    codes, scales = np.zeros((6, 2, 16, 64), dtype=np.int8), np.zeros((6, 2), dtype=np.uint16)
    x = rng.standard_normal((1, 60, 2, 64)) * np.linspace(0.2, 3.0, 60)[None, :, None, None]
    table, done = np.array([[5, 0, 3, 1]]), 0
    steps = 0
    for n in (1, 7, 8, 1, 20, 23):
        ds.kv8_append(codes, scales, bf16(x[:, done:done + n]), table, [done], [n])
        done, steps = done + n, steps + 1
    got = np.stack([ds.kv8_values(codes, scales, table[0], h, 60)[0] for h in range(2)], axis=1)
    step = np.repeat(onp.fp16_bits_to_f64(scales[table[0]]), 16, axis=0)[:60, :, None]
    assert (np.abs(got - onp.bf16_bits_to_f64(bf16(x[0]))) <= 0.5 * step * steps * (1 + 2.0 ** -10)).all()


def _case(rng, B, T, heads, rep, dim, block, width):
    blocks = B * width
    codes = [rng.integers(-127, 128, size=(blocks, heads, block, dim)).astype(np.int8) for _ in range(2)]
    scales = [onp.f64_to_fp16_bits(rng.uniform(0.005, 0.02, size=(blocks, heads))) for _ in range(2)]
    table = rng.permutation(blocks).reshape(B, width)
    q = bf16(rng.standard_normal((B, T, heads * rep, dim)))
    return q, codes[0], scales[0], codes[1], scales[1], table


def test_attention_reduces_to_the_textbook_form():
    rng = np.random.default_rng(11)
    q, kc, ks, vc, vs, table = _case(rng, 2, 3, 2, 2, 64, 16, 3)
    limits = np.array([[40, 41, 42], [1, 0, 48]])
    out = ds.kv8_attention(q, kc, ks, vc, vs, table, limits, 0.125)[0]
    qf = onp.bf16_bits_to_f64(q)
    for b in range(2):
        for t in range(3):
            for h in range(4):
                num, den = np.zeros(64), 0.0
                for j in range(limits[b, t]):
                    n, s = table[b, j // 16], j % 16
                    k = kc[n, h // 2, s].astype(float) * onp.fp16_bits_to_f64(ks[n, h // 2])
                    p = np.exp(0.125 * qf[b, t, h] @ k)
                    num, den = num + p * vc[n, h // 2, s] * onp.fp16_bits_to_f64(vs[n, h // 2]), den + p
                assert np.allclose(out[b, t, h], num / den if den else 0.0, rtol=1e-12, atol=1e-14)
    # a scale of zero averages, and one position is returned as it is
    flat = ds.kv8_attention(q, kc, ks, vc, vs, table, limits, 0.0)[0]
    assert np.allclose(flat[0, 2, 0], ds.kv8_values(vc, vs, table[0], 0, 42)[0].mean(axis=0), rtol=1e-12, atol=1e-14)
    assert np.allclose(out[1, 0, 3], ds.kv8_values(vc, vs, table[1], 1, 1)[0][0], rtol=1e-14)


def test_streaming_limits_are_the_masks_row_sums():
    for V, F, n in ((1, 1, 6), (3, 4, 5), (4, 4, 18), (2, 7, 33)):
        mask = so.streaming_mask(V, F, n)
        limits = B.streaming_limits(V, F, n).numpy()
        assert np.array_equal(limits, mask.sum(axis=1))
        assert np.array_equal(mask, np.arange(mask.shape[1])[None, :] < limits[:, None])
