"""The steps of a decoder layer in a row, as they are used: norm, QKV projection, rotary embedding, append, attention, O projection with the
residual, norm, gate+up with SiLU, down with the residual; eagerly, and captured once and replayed while the sequence grows."""
import numpy as np
import pytest
import torch

from oracle import decoder_steps as ds
from oracle import w4a8_oracle as onp
from paper_2608_12932_b200 import binding as B
from paper_2608_12932_b200 import workload as wl
from tests.gpu_util import bits, t_u16

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV, DIM, INTER, BLOCK = 512, 8, 2, 64, 640, 16
QKV = (HEADS + 2 * KV) * DIM


def packed(rng, n, k):
    w = (rng.standard_normal((n, k // 128, 128)) * 0.04).astype(np.float32)
    lo, hi = np.minimum(w.min(2), 0), np.maximum(w.max(2), 0)
    s = ((hi - lo) / 15).astype(np.float16)
    z = np.clip(np.rint(-lo / s.astype(np.float32)), 0, 15)
    q = np.clip(np.rint(w / s.astype(np.float32)[:, :, None]) + z[:, :, None], 0, 15).astype(np.uint8).reshape(n, k)
    return B.w4a8_pack_weights(torch.from_numpy(q).cuda(), torch.from_numpy(np.ascontiguousarray(s.T)).cuda(),
                               torch.from_numpy(np.ascontiguousarray(z.T.astype(np.uint8))).cuda())


class Layer:
    """One layer's weights, cache and buffers for `seqs` sequences of T new tokens a step; everything is allocated here, as a captured step needs."""

    def __init__(self, seqs, T, width, seed):
        rng = np.random.default_rng(seed)
        M = seqs * T
        self.seqs, self.T, self.M = seqs, T, M
        self.w_qkv, self.w_o = packed(rng, QKV, HIDDEN), packed(rng, HIDDEN, HIDDEN)
        self.w_gu, self.w_down = packed(rng, 2 * INTER, HIDDEN), packed(rng, HIDDEN, INTER)
        self.n1, self.n2 = (t_u16(wl.f32_to_bf16_bits(rng.uniform(0.5, 1.5, HIDDEN).astype(np.float32)), torch.bfloat16) for _ in range(2))
        blocks = seqs * width
        self.cache = B.KV8Cache.empty(blocks, KV, DIM, BLOCK)
        self.table = torch.from_numpy(rng.permutation(blocks).reshape(seqs, width).astype(np.int32)).cuda()
        # one workspace for the linears, the append and the attention
        need = max([B.w4a8_kv8_workspace_bytes(DIM)] + [B.w4a8_workspace_bytes(M, n, k) for n, k in ((QKV, HIDDEN), (HIDDEN, HIDDEN), (2 * INTER, HIDDEN), (HIDDEN, INTER))])
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        assert B.lib().w4a8_workspace_init(self.ws.data_ptr(), need, None) == B.OK
        bf, i32 = dict(dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.int32, device="cuda")
        self.x, self.stream, self.out = torch.empty((M, HIDDEN), **bf), torch.empty((M, HIDDEN), **bf), torch.empty((M, HIDDEN), **bf)
        self.qkv, self.attn, self.mid = torch.empty((M, QKV), **bf), torch.empty((M, HEADS * DIM), **bf), torch.empty((M, HIDDEN), **bf)
        self.q_rot, self.k_rot = torch.empty((M, HEADS, DIM), **bf), torch.empty((M, KV, DIM), **bf)
        self.y_gu = torch.empty((M, 2 * INTER), **bf)
        self.start, self.limits, self.pos = torch.empty(seqs, **i32), torch.empty((seqs, T), **i32), torch.empty(M, **i32)
        quant = lambda k: (torch.empty((M, k), dtype=torch.int8, device="cuda"), torch.empty(M, dtype=torch.float16, device="cuda"), torch.empty((M, k // 128), **i32))
        self.q1, self.q2, self.q3 = quant(HIDDEN), quant(HIDDEN), quant(HIDDEN)
        self.h = (torch.empty((M, INTER), **bf), *quant(INTER))

    def at(self, starts):
        i = torch.arange(self.T, dtype=torch.int32)
        s = torch.tensor(starts, dtype=torch.int32)
        self.start.copy_(s)
        self.pos.copy_((s[:, None] + i).reshape(-1))
        self.limits.copy_(s[:, None] + i + 1)

    def step(self):
        B.w4a8_add_rmsnorm_quantize(self.x, self.n1, 1e-6, residual=self.stream, sum_out=self.stream, out=self.q1)
        B.w4a8_gemm(*self.q1, self.w_qkv, QKV, self.ws, out=self.qkv)
        q, k, v = self.qkv[:, :HEADS * DIM], self.qkv[:, HEADS * DIM:(HEADS + KV) * DIM], self.qkv[:, (HEADS + KV) * DIM:]
        B.w4a8_rope_shifted_keys(q.contiguous().view(self.M, HEADS, DIM), self.pos, 0, 1e4, out=self.q_rot)
        B.w4a8_rope_shifted_keys(k.contiguous().view(self.M, KV, DIM), self.pos, 0, 1e4, out=self.k_rot)
        B.w4a8_kv8_append(self.cache, self.k_rot, v.unflatten(1, (KV, DIM)), self.table, self.start, self.ws)
        B.w4a8_kv8_attention(self.q_rot, self.cache, self.table, self.limits, DIM ** -0.5, self.ws, out=self.attn)
        B.w4a8_quantize_act(self.attn, out=self.q2)
        B.w4a8_gemm_residual(*self.q2, self.w_o, self.stream, HIDDEN, self.ws, out=self.mid)
        B.w4a8_add_rmsnorm_quantize(self.mid, self.n2, 1e-6, out=self.q3)
        B.w4a8_gate_up_silu_quantize(*self.q3, self.w_gu, 2 * INTER, self.ws, y_scratch=self.y_gu, out=self.h)
        B.w4a8_gemm_residual(*self.h[1:], self.w_down, self.mid, HIDDEN, self.ws, out=self.out)


def host_cache(layer):
    return (layer.cache.k_codes.cpu().numpy().copy(), bits(layer.cache.k_scales).copy(), layer.cache.v_codes.cpu().numpy().copy(), bits(layer.cache.v_scales).copy())


@pytest.mark.parametrize("seqs,T", [(1, 1), (3, 1), (2, 8), (1, 70)])
def test_decoder_layer_step_by_step(seqs, T):
    steps, width = 4, (4 * T + 20 + BLOCK - 1) // BLOCK
    layer = Layer(seqs, T, width, seqs * 100 + T)
    rng = np.random.default_rng(T)
    kc, ks, vc, vs = host_cache(layer)
    table = layer.table.cpu().numpy()
    # a prefix of a few tokens, different for each sequence
    starts = [3 + 5 * b for b in range(seqs)]
    pre = [wl.f32_to_bf16_bits(rng.standard_normal((seqs, 20, KV, DIM)).astype(np.float32)) for _ in range(2)]
    B.w4a8_kv8_append(layer.cache, *(t_u16(p.reshape(-1, KV, DIM), torch.bfloat16) for p in pre), layer.table, torch.zeros(seqs, dtype=torch.int32, device="cuda"),
                      layer.ws, count=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    for codes, scales, p in ((kc, ks, pre[0]), (vc, vs, pre[1])):
        ds.kv8_append(codes, scales, p, table, [0] * seqs, starts)
    inputs = [wl.f32_to_bf16_bits(rng.standard_normal((layer.M, HIDDEN)).astype(np.float32)) for _ in range(steps)]
    stream0 = wl.f32_to_bf16_bits(rng.standard_normal((layer.M, HIDDEN)).astype(np.float32))
    layer.stream.copy_(t_u16(stream0, torch.bfloat16))
    kept, seen = [], []
    for i, x in enumerate(inputs):
        layer.x.copy_(t_u16(x, torch.bfloat16))
        layer.at([s + i * T for s in starts])
        before = bits(layer.stream).copy()
        layer.step()
        B.w4a8_check_status(layer.ws)
        # the stream and the operands of the QKV projection
        s_bits, _, h_bits = ds.add_rmsnorm(x, before, bits(layer.n1), 1e-6)
        assert np.array_equal(bits(layer.stream), s_bits)
        off = layer.q1[0].float() * layer.q1[1].float()[:, None] - t_u16(h_bits, torch.bfloat16).float()
        assert (off.abs() <= 0.51 * layer.q1[1].float()[:, None] + 2.0 ** -7 * t_u16(h_bits, torch.bfloat16).float().abs()).all()
        # the cache: bit for bit what the oracle makes of the same keys and values
        v = bits(layer.qkv[:, (HEADS + KV) * DIM:].contiguous()).reshape(seqs, T, KV, DIM)
        for codes, scales, p in ((kc, ks, bits(layer.k_rot).reshape(seqs, T, KV, DIM)), (vc, vs, v)):
            ds.kv8_append(codes, scales, p, table, [s + i * T for s in starts], [T] * seqs)
        used = sorted({int(n) for b in range(seqs) for n in table[b, :-(-(starts[b] + (i + 1) * T) // BLOCK)]})
        got = host_cache(layer)
        for mine, theirs in zip((ks, vs), (got[1], got[3])):
            assert np.array_equal(mine[used], theirs[used])
        last = {int(table[b, (starts[b] + (i + 1) * T - 1) // BLOCK]): (starts[b] + (i + 1) * T - 1) % BLOCK + 1 for b in range(seqs)}
        for mine, theirs in zip((kc, vc), (got[0], got[2])):
            for n in used:
                m = last.get(n, BLOCK)
                assert np.array_equal(mine[n, :, :m], theirs[n, :, :m])
        # attention over it
        limits = np.array([[s + i * T + t + 1 for t in range(T)] for s in starts])
        ref, spread, tail, size = ds.kv8_attention(bits(layer.q_rot).reshape(seqs, T, HEADS, DIM), got[0], got[1], got[2], got[3], table, limits, DIM ** -0.5)
        band = ds.kv8_attention_band(ref, spread, tail, size, width * BLOCK, DIM)
        out = onp.bf16_bits_to_f64(bits(layer.attn)).reshape(ref.shape)
        assert (np.abs(out - ref) <= band).all()
        kept.append((layer.attn.clone(), layer.out.clone(), layer.stream.clone()))
        assert torch.isfinite(layer.out.float()).all()
        seen.append(i)
    # the same from an empty cache, captured once and replayed: positions, limits and inputs are data
    again = Layer(seqs, T, width, seqs * 100 + T)
    B.w4a8_kv8_append(again.cache, *(t_u16(p.reshape(-1, KV, DIM), torch.bfloat16) for p in pre), again.table, torch.zeros(seqs, dtype=torch.int32, device="cuda"),
                      again.ws, count=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    again.stream.copy_(t_u16(stream0, torch.bfloat16))
    again.at(starts)
    again.x.copy_(t_u16(inputs[0], torch.bfloat16))
    codes = host_cache(again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again.step()                                          # warm-up: it appends and moves the stream, so both are put back
    torch.cuda.current_stream().wait_stream(side)
    again.stream.copy_(t_u16(stream0, torch.bfloat16))
    for t, c in zip((again.cache.k_codes, again.cache.v_codes), (codes[0], codes[2])):
        t.copy_(torch.from_numpy(c))
    for t, c in zip((again.cache.k_scales, again.cache.v_scales), (codes[1], codes[3])):
        t.copy_(t_u16(c, torch.float16))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again.step()
    for i in seen:
        again.x.copy_(t_u16(inputs[i], torch.bfloat16))
        again.at([s + i * T for s in starts])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((again.attn, again.out, again.stream), kept[i]):
            assert torch.equal(a, b), i
    B.w4a8_check_status(again.ws)


def test_scores_scaled_by_zero_and_by_a_negative_number():
    from tests.test_gpu_decoder_steps import attend_case, causal
    for T in (1, 8, 150):
        _, c, table, q = attend_case(T + 21, 1, T, 2, 4, 64, 16, 300)
        for scale in (0.0, -0.07):
            c.check_attend(q, table, causal([300], T), scale=scale)


def test_two_streams_with_a_workspace_each():
    """Calls that overlap on the GPU have workspaces of their own and do not disturb each other."""
    from tests.test_gpu_decoder_steps import attend_case, causal, i32
    _, c, table, q = attend_case(31, 1, 8, 4, 4, 128, 64, 9000)
    qt, tt, lt = t_u16(q[0], torch.bfloat16), i32(table), i32(causal([9000], 8))
    want = B.w4a8_kv8_attention(qt, c.dev, tt, lt, 0.1, c.ws)
    streams, spaces = [torch.cuda.Stream() for _ in range(3)], [B.new_kv8_workspace(c.dev) for _ in range(3)]
    outs = [[torch.zeros_like(want) for _ in range(6)] for _ in range(3)]
    torch.cuda.synchronize()
    for i in range(6):
        for s, w, o in zip(streams, spaces, outs):
            B.w4a8_kv8_attention(qt, c.dev, tt, lt, 0.1, w, out=o[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for o in outs for x in o)
