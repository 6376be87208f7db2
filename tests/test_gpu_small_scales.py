"""Codes, scales and group sums bit for bit where the fp16 scale is zero, subnormal or a small normal number: every bf16 magnitude from 2^-25 to
2^-7 as the largest of a row or block, either sign.  (A subnormal scale can be a third smaller than amax / 127, so quotients reach 190.)"""
import numpy as np
import pytest
import torch

from oracle import decoder_steps as ds
from oracle import w4a8_oracle as onp
from paper_2608_12932_b200 import binding as B
from paper_2608_12932_b200 import workload as wl
from tests.gpu_util import bits, t_u16

pytestmark = pytest.mark.gpu

TOPS = np.arange((127 - 25) << 7, (127 - 7) << 7, dtype=np.uint16)         # 2304 magnitudes


def rows_below(rng, tops, K):
    """One row per largest magnitude: that value with either sign, the largest values below it, others spread over it."""
    x = onp.bf16_bits_to_f64(tops)[:, None] * rng.uniform(-1.0, 1.0, size=(len(tops), K))
    x = (wl.f32_to_bf16_bits(x.astype(np.float32)) & 0x8000) | np.minimum(wl.f32_to_bf16_bits(x.astype(np.float32)) & 0x7FFF, tops[:, None])
    sign = (rng.integers(0, 2, size=(len(tops), 2)) << 15).astype(np.uint16)
    x[:, 3], x[:, K - 2] = tops | sign[:, 0], tops | (sign[:, 0] ^ 0x8000)
    x[:, 17], x[:, 40] = (tops - 1) | sign[:, 1], (tops - 2) | sign[:, 1]
    return x.astype(np.uint16)


def same(got, x_bits):
    for g, want in zip((got[0].cpu().numpy(), bits(got[1]), got[2].cpu().numpy()), onp.quantize_act(x_bits, 128)):
        assert np.array_equal(g, want)


def test_the_rows_reach_what_they_should():
    s = onp.quantize_act(rows_below(np.random.default_rng(0), TOPS, 128), 128)[1]
    assert s[0] == 0 and s[-1] > 0x0400 and len(set(s[s < 0x80])) == 0x80


@pytest.mark.parametrize("M,K", [(2304, 4096), (2304, 4224), (600, 128), (100, 4096), (40, 640), (1, 256)])
def test_quantize(M, K):
    """More than 512 rows: the reciprocal form; fewer: the division."""
    x = rows_below(np.random.default_rng(M + K), TOPS if M > 1 else TOPS[::37], K)
    for i in range(0, len(x), M):
        part = x[i:i + M]
        same(B.w4a8_quantize_act(t_u16(part, torch.bfloat16)), part)


@pytest.mark.parametrize("M,I", [(2304, 640), (2304, 4352), (576, 256), (128, 1152), (32, 640), (16, 128),
                                 (576, 10240), (256, 8192), (128, 12288), (16, 5120)])
def test_silu_mul_quantize(M, I):
    """On the kernel's own h: gate near one and up small, many rows, one CTA each, a row shared by a cluster of eight, four or two."""
    rng = np.random.default_rng(M + I)
    up = rows_below(rng, TOPS if I < 5000 else TOPS[::4], I)
    gate = wl.f32_to_bf16_bits(rng.uniform(1.0, 2.0, size=up.shape).astype(np.float32))
    y = np.stack([gate.reshape(-1, I // 8, 8), up.reshape(-1, I // 8, 8)], axis=2).reshape(-1, 2 * I)
    for i in range(0, len(up), M):
        h, *q = B.w4a8_silu_mul_quantize(t_u16(y[i:i + M], torch.bfloat16))
        same(q, bits(h))


@pytest.mark.parametrize("M,K", [(2304, 640), (2304, 4096), (1152, 5120), (576, 6272), (128, 4096), (128, 6272), (16, 256), (1, 128)])
def test_norm(M, K):
    """Every launch shape.  With eps = 1 and weights of one h is s again: the root is off from one by 2^-15 at most, a bf16 value keeps to itself within 2^-9."""
    x = rows_below(np.random.default_rng(M + K), TOPS if M > 1 else TOPS[::37], K)
    one = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    for i in range(0, len(x), M):
        part = x[i:i + M]
        xt, h = t_u16(part, torch.bfloat16), torch.empty((len(part), K), dtype=torch.bfloat16, device="cuda")
        s, *q = B.w4a8_add_rmsnorm_quantize(xt, one, 1.0, h_out=h)
        assert np.array_equal(bits(h), part)
        same(q, part)
        # half of the row from the residual
        s, *q = B.w4a8_add_rmsnorm_quantize(torch.zeros_like(xt), one, 1.0, residual=xt)
        same(q, part)


@pytest.mark.parametrize("dim,block", [(64, 16), (128, 16), (64, 128), (128, 64)])
def test_append(dim, block):
    """Fresh blocks, then new maxima behind the first tokens of each: some scales rise from one subnormal number to another."""
    rng = np.random.default_rng(dim + block)
    heads, seqs = 8, len(TOPS) // 8
    dev = B.KV8Cache.empty(seqs, heads, dim, block)
    for t in (dev.k_codes, dev.v_codes, dev.k_scales, dev.v_scales):
        t.zero_()
    ws = B.new_kv8_workspace(dev)
    codes, scales = ([np.zeros((seqs, heads, block, dim), dtype=np.int8) for _ in range(2)], [np.zeros((seqs, heads), dtype=np.uint16) for _ in range(2)])
    table = rng.permutation(seqs).reshape(seqs, 1).astype(np.int32)
    done = 0
    for T in (5, block - 5):
        kv = []
        for _ in range(2):
            x = rows_below(rng, rng.permutation(TOPS), T * dim).reshape(seqs, heads, T, dim).transpose(0, 2, 1, 3)
            kv.append(np.ascontiguousarray(x))
        for i in range(2):
            ds.kv8_append(codes[i], scales[i], kv[i], table, [done] * seqs, [T] * seqs)
        B.w4a8_kv8_append(dev, *(t_u16(x.reshape(seqs * T, heads, dim), torch.bfloat16) for x in kv), torch.from_numpy(table).cuda(),
                          torch.full((seqs,), done, dtype=torch.int32, device="cuda"), ws)
        torch.cuda.synchronize()
        done += T
        for got, want in ((dev.k_scales, scales[0]), (dev.v_scales, scales[1])):
            assert np.array_equal(bits(got), want)
        for got, want in ((dev.k_codes, codes[0]), (dev.v_codes, codes[1])):
            assert np.array_equal(got.cpu().numpy(), want)
    B.w4a8_check_status(ws)
