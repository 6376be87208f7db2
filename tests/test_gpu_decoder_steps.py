"""GPU parity of the steps between the quantised linears: residual + RMS norm + quantisation, the append to the 8-bit cache (codes and
scales bit for bit), attention over it (fp64 definition, with a band per element that counts the kernel's roundings)."""
import numpy as np
import pytest
import torch

from oracle import decoder_steps as ds
from oracle import w4a8_oracle as onp
from paper_2608_12932_b200 import binding as B
from paper_2608_12932_b200 import workload as wl
from tests.gpu_util import bits, t_u16

pytestmark = pytest.mark.gpu


def ordered(b):
    b = b.astype(np.int32)
    return np.where(b & 0x8000, -(b & 0x7FFF), b & 0x7FFF)


def bf16(a):
    return wl.f32_to_bf16_bits(np.asarray(a, dtype=np.float32))


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ---- norm ---------------------------------------------------------------------------------------------------------------

def norm_case(M, K, seed, size=1.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((M, K)) * size
    x[:, rng.integers(0, K, size=max(1, K // 100))] *= 20
    return bf16(x), bf16(rng.standard_normal((M, K)) * 4 * size), bf16(rng.uniform(-1.5, 1.5, size=K))


def check_norm(x, r, w, eps, got_sum, got_h, qa, sa, asum):
    s_bits, h, h_bits = ds.add_rmsnorm(x, r, w, eps)
    if r is not None:
        assert np.array_equal(bits(got_sum), s_bits)
    got = bits(got_h)
    # fp32 arithmetic on the way (2^-20 at most over a long row): the bf16 of the definition or its neighbour
    assert np.abs(ordered(got) - ordered(h_bits)).max() <= 1
    q_ref, s_ref, a_ref = onp.quantize_act(got, 128)
    assert np.array_equal(bits(sa), s_ref) and np.array_equal(qa.cpu().numpy(), q_ref) and np.array_equal(asum.cpu().numpy(), a_ref)


@pytest.mark.parametrize("M,K", [(1, 128), (1, 4096), (3, 256), (8, 4096), (17, 12288), (200, 2048), (513, 640), (600, 5120), (515, 12416),
                                 (2, 33024), (700, 128), (1025, 1152)])
@pytest.mark.parametrize("add", [True, False])
def test_norm(M, K, add):
    x, r, w = norm_case(M, K, M + K)
    r = r if add else None
    xt, rt, wt = t_u16(x, torch.bfloat16), t_u16(r, torch.bfloat16) if add else None, t_u16(w, torch.bfloat16)
    h = torch.empty_like(xt)
    total, qa, sa, asum = B.w4a8_add_rmsnorm_quantize(xt, wt, 1e-6, residual=rt, h_out=h)
    torch.cuda.synchronize()
    assert add or total is xt
    check_norm(x, r, w, 1e-6, total, h, qa, sa, asum)
    # without h, and in place on the stream: the same
    for out in ((xt, rt) if add else ()):
        again = B.w4a8_add_rmsnorm_quantize(xt, wt, 1e-6, residual=rt, sum_out=out)
        torch.cuda.synchronize()
        assert again[0] is out and torch.equal(out, total)
        assert torch.equal(again[1], qa) and torch.equal(again[2], sa) and torch.equal(again[3], asum)
        xt, rt = t_u16(x, torch.bfloat16), t_u16(r, torch.bfloat16)


@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e4, 1e15])
def test_norm_of_small_and_large_rows(size):
    x, r, w = norm_case(5, 512, 7, size)
    x[2], r[2] = 0, 0                                          # a row of zeros: scale 0, codes 0
    h = torch.empty((5, 512), dtype=torch.bfloat16, device="cuda")
    total, qa, sa, asum = B.w4a8_add_rmsnorm_quantize(t_u16(x, torch.bfloat16), t_u16(w, torch.bfloat16), 1e-6, residual=t_u16(r, torch.bfloat16), h_out=h)
    torch.cuda.synchronize()
    assert (qa[2] == 0).all() and sa[2] == 0
    check_norm(x, r, w, 1e-6, total, h, qa, sa, asum)


def test_norm_refusals():
    x = torch.zeros((2, 256), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(256, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(weight=w[:128]), dict(residual=x[:1]), dict(sum_out=x[:1], residual=x), dict(h_out=x[:1])):
        with pytest.raises(B.W4A8Error) as e:
            B.w4a8_add_rmsnorm_quantize(**{**dict(x=x, weight=w, eps=1e-6), **bad})
        assert e.value.code == B.ERR_SHAPE
    with pytest.raises(TypeError):
        B.w4a8_add_rmsnorm_quantize(x.t(), w, 1e-6)
    with pytest.raises(B.W4A8Error):
        B.w4a8_add_rmsnorm_quantize(x, w, -1.0)
    empty = B.w4a8_add_rmsnorm_quantize(x[:0], w, 1e-6)
    assert empty[1].shape == (0, 256)


# ---- the cache ----------------------------------------------------------------------------------------------------------

class Cache:
    """Random codes and scales, on the host and on the device."""

    def __init__(self, rng, blocks, heads, block, dim, k_scale=(0.005, 0.02), v_scale=(0.005, 0.02)):
        self.k, self.v = (rng.integers(-127, 128, size=(blocks, heads, block, dim)).astype(np.int8) for _ in range(2))
        self.ks, self.vs = (onp.f64_to_fp16_bits(np.exp(rng.uniform(np.log(lo), np.log(hi), size=(blocks, heads)))) for lo, hi in (k_scale, v_scale))
        self.upload()

    def upload(self):
        self.dev = B.KV8Cache(torch.from_numpy(self.k).cuda(), torch.from_numpy(self.v).cuda(), t_u16(self.ks, torch.float16), t_u16(self.vs, torch.float16))
        self.ws = B.new_kv8_workspace(self.dev)

    def append(self, k, v, table, start, count=None, wide=0):
        """The oracle on the host arrays and the library on the device's; k, v bf16 bits [B, T, heads, dim]."""
        Bn, T, heads, dim = k.shape
        ds.kv8_append(self.k, self.ks, k, table, start, [T] * Bn if count is None else count)
        ds.kv8_append(self.v, self.vs, v, table, start, [T] * Bn if count is None else count)
        both = torch.zeros((Bn * T, wide + 2 * heads * dim), dtype=torch.bfloat16, device="cuda")
        for i, x in enumerate((k, v)):
            both[:, wide + i * heads * dim: wide + (i + 1) * heads * dim] = t_u16(x.reshape(Bn * T, -1), torch.bfloat16)
        kt, vt = (both[:, wide + i * heads * dim: wide + (i + 1) * heads * dim].unflatten(1, (heads, dim)) for i in range(2))
        B.w4a8_kv8_append(self.dev, kt, vt, i32(table), i32(start), self.ws, count=None if count is None else i32(count))
        torch.cuda.synchronize()

    def check(self):
        assert np.array_equal(bits(self.dev.k_scales), self.ks) and np.array_equal(bits(self.dev.v_scales), self.vs)
        assert np.array_equal(self.dev.k_codes.cpu().numpy(), self.k) and np.array_equal(self.dev.v_codes.cpu().numpy(), self.v)

    def attend(self, q, table, limits, scale, out=None, stream=None):
        Bn, T, qh, dim = q.shape
        got = B.w4a8_kv8_attention(t_u16(q.reshape(Bn * T, qh, dim), torch.bfloat16), self.dev, i32(table), i32(limits), scale, self.ws, out=out)
        torch.cuda.synchronize()
        return got

    def check_attend(self, q, table, limits, scale=None):
        Bn, T, qh, dim = q.shape
        scale = dim ** -0.5 if scale is None else scale
        got = onp.bf16_bits_to_f64(bits(self.attend(q, table, limits, scale))).reshape(Bn, T, qh, dim)
        ref, spread, tail, size = ds.kv8_attention(q, self.k, self.ks, self.v, self.vs, table, limits, scale)
        band = ds.kv8_attention_band(ref, spread, tail, size, table.shape[1] * self.k.shape[2], dim)
        worst = (np.abs(got - ref) / band).max()
        assert worst <= 1.0, f"worst |err| / band = {worst}"
        return got


def new_values(rng, B_, T, heads, dim, size=1.0):
    return (bf16(rng.standard_normal((B_, T, heads, dim)) * size * np.exp(rng.uniform(-1, 1, size=(B_, T, 1, 1)))) for _ in range(2))


@pytest.mark.parametrize("B_,T,heads,dim,block,start", [(1, 1, 8, 128, 64, 37), (1, 1, 1, 64, 16, 0), (5, 8, 4, 64, 16, 21), (2, 33, 2, 128, 32, 15),
                                                       (1, 300, 3, 64, 128, 127), (3, 129, 2, 128, 128, 1), (2, 64, 2, 64, 64, 64), (1, 17, 5, 128, 16, 31)])
def test_append(B_, T, heads, dim, block, start):
    rng = np.random.default_rng(B_ * 100 + T)
    width = (start + 3 * B_ + T + block - 1) // block
    c = Cache(rng, B_ * width + 2, heads, block, dim)
    table = rng.permutation(B_ * width + 2)[: B_ * width].reshape(B_, width)
    starts = [start + 3 * b for b in range(B_)]
    for size in (1.0, 4.0, 0.01):                            # scales stay, rise (old codes are rounded anew), stay
        c.append(*new_values(rng, B_, T, heads, dim, size), table, starts, wide=64)
        c.check()
    c.append(*new_values(rng, B_, T, heads, dim, 8.0), table, starts, count=[(b * 7 + T - 1) % (T + 1) for b in range(B_)])
    c.check()
    B.w4a8_check_status(c.ws)


def test_append_token_by_token_and_back():
    """Draft tokens that were not accepted are written over; zeros, ties and tiny values among the tokens."""
    rng = np.random.default_rng(77)
    c = Cache(rng, 9, 2, 16, 64)
    table = rng.permutation(9)[:8].reshape(2, 4)
    at = [0, 3]
    for step in range(30):
        T = int(rng.integers(1, 6))
        k, v = new_values(rng, 2, T, 2, 64, 10.0 ** rng.uniform(-3, 2))
        if step % 5 == 0:
            k[:] = 0
        if step % 7 == 3:
            v[0] = bf16(np.full(v[0].shape, 2.0 ** -130))      # below every fp16 scale
        c.append(k, v, table, at)
        c.check()
        at = [(a + int(rng.integers(1, T + 1))) % 50 for a in at]
    B.w4a8_check_status(c.ws)


def test_append_leaves_out_what_has_no_place():
    rng = np.random.default_rng(78)
    c = Cache(rng, 4, 2, 16, 128)
    for table, start, count in ((np.array([[2, 4]]), 10, [12]), (np.array([[-1, 1]]), 3, [12]), (np.array([[0, 3]]), 25, [12]),
                                (np.array([[0, 3]]), -1, [12]), (np.array([[0, 3]]), 2 ** 31 - 2, [12])):
        c.append(*new_values(rng, 1, 12, 2, 128), table, [start], count)
        c.check()
        with pytest.raises(B.W4A8Error) as e:
            B.w4a8_check_status(c.ws)
        assert e.value.code == B.ERR_INDEX
        B.w4a8_check_status(c.ws)                             # cleared
    c.append(*new_values(rng, 1, 12, 2, 128), np.array([[0, 9]]), [0], [-5])
    c.append(*new_values(rng, 1, 12, 2, 128), np.array([[0, 3]]), [3], [99])          # counts as 12
    c.check()
    B.w4a8_check_status(c.ws)


# ---- attention ----------------------------------------------------------------------------------------------------------

def attend_case(seed, B_, T, heads, rep, dim, block, keys, spare=1, **scales):
    rng = np.random.default_rng(seed)
    width = max(1, -(-keys // block))
    blocks = B_ * width + spare
    c = Cache(rng, blocks, heads, block, dim, **scales)
    table = rng.permutation(blocks)[: B_ * width].reshape(B_, width)
    q = bf16(rng.standard_normal((B_, T, heads * rep, dim)) * 1.5)
    return rng, c, table, q


def causal(keys, T):
    return np.maximum(np.asarray(keys)[:, None] - T + 1 + np.arange(T)[None, :], 0)


@pytest.mark.parametrize("keys", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000, 2049])
@pytest.mark.parametrize("dim,block,heads,rep", [(128, 64, 8, 4), (64, 16, 2, 8), (128, 128, 1, 1), (64, 32, 3, 5)])
def test_attention_of_one_token(keys, dim, block, heads, rep):
    _, c, table, q = attend_case(keys + dim, 1, 1, heads, rep, dim, block, keys)
    c.check_attend(q, table, [[keys]])


@pytest.mark.parametrize("T,rep,heads", [(1, 16, 1), (1, 17, 2), (8, 4, 2), (5, 3, 2), (16, 2, 1), (11, 3, 1), (33, 1, 2), (3, 40, 1), (64, 4, 1),
                                        (65, 4, 1), (128, 1, 1), (129, 1, 2), (200, 7, 1), (300, 4, 2), (513, 1, 1)])
@pytest.mark.parametrize("dim,block", [(128, 64), (64, 128), (128, 16)])
def test_attention_rows(T, rep, heads, dim, block):
    """Causal rows over a prefix: every way the rows can fill a tile."""
    keys = T + 77
    _, c, table, q = attend_case(T * rep + dim + block, 1, T, heads, rep, dim, block, keys)
    c.check_attend(q, table, causal([keys], T))


@pytest.mark.parametrize("B_,T,heads,rep,dim,block,keys", [(1, 1210, 8, 4, 128, 64, 1300), (3, 500, 8, 5, 64, 32, 640), (40, 40, 5, 7, 128, 128, 90)])
def test_attention_of_more_tiles_than_are_resident(B_, T, heads, rep, dim, block, keys):
    """Every kernel's later rounds: a CTA that walks several row tiles of different lengths, one of them without any key."""
    _, c, table, q = attend_case(T + rep, B_, T, heads, rep, dim, block, keys)
    limits = causal([keys - 13 * (b % 5) for b in range(B_)], T)
    limits[B_ // 2, T // 2:T // 2 + 300] = 0
    c.check_attend(q, table, limits)


@pytest.mark.parametrize("T", [1, 8, 70])
def test_attention_of_a_padded_batch(T):
    """Ragged sequences, some rows and one whole sequence that see nothing: those give zeros."""
    rng, c, table, q = attend_case(T, 7, T, 2, 4, 128, 32, 700)
    limits = causal([700, 1, 33, T, 699, 256, 31], T)
    limits[2, T // 2:] = 0
    limits[5] = 0
    got = c.check_attend(q, table, limits)
    assert (got[limits == 0] == 0).all()
    # limits outside 0 .. capacity count as the nearest
    wild = limits.copy()
    wild[limits == 0] = -2 ** 31
    wild[0] = 2 ** 31 - 1
    limits[0] = table.shape[1] * 32
    assert torch.equal(c.attend(q, table, wild, 0.1), c.attend(q, table, limits, 0.1))


def test_streaming_prefill_rows():
    V, F, n = 3, 3, 37
    _, c, table, q = attend_case(5, 1, V * n, 2, 4, 64, 64, V * F * n)
    c.check_attend(q, table, B.streaming_limits(V, F, n).numpy()[None])


@pytest.mark.parametrize("T,keys", [(1, 700), (8, 700), (150, 700)])
@pytest.mark.parametrize("v_scale", [(2.0 ** -20, 2.0 ** 10), (100.0, 400.0)])
def test_attention_with_scales_far_apart(T, keys, v_scale):
    """Value scales that differ by nine decades from block to block, and large ones."""
    _, c, table, q = attend_case(T + 3, 1, T, 2, 2, 128, 16, keys, v_scale=v_scale)
    c.check_attend(q, table, causal([keys], T))


@pytest.mark.parametrize("T", [1, 8, 150])
@pytest.mark.parametrize("size", [2.0 ** -60, 1e-3, 40.0, 2.0 ** 40])
def test_attention_with_small_and_large_queries(T, size):
    """Flat weights, weights on a single key, and a factor that leaves the range of fp16 either way; the score scale undoes it."""
    rng, c, table, q = attend_case(T + 4, 1, T, 2, 4, 64, 16, 500)
    big = bf16(onp.bf16_bits_to_f64(q) * size)
    c.check_attend(big, table, causal([500], T), scale=0.125 * (1.0 if size in (1e-3, 40.0) else 1.0 / size))


@pytest.mark.parametrize("T", [1, 8, 150])
def test_rising_scores(T):
    """Keys aligned with the query, later ones more so: the running reference moves again and again."""
    rng, c, table, q = attend_case(T + 5, 1, T, 1, 2, 128, 16, 400)
    c.k[:] = np.sign(onp.bf16_bits_to_f64(q)[0, 0, 0]).astype(np.int8)[None, None, None, :] * 127
    order = np.argsort(table[0])
    level = np.empty(c.ks.shape[0])
    level[table[0]] = np.linspace(0.0005, 0.02, table.shape[1])
    level[[i for i in range(len(level)) if i not in set(table[0])]] = 0.001
    c.ks = onp.f64_to_fp16_bits(level)[:, None].copy()
    assert len(order)
    c.upload()
    c.check_attend(q, table, causal([400], T))


@pytest.mark.parametrize("T", [1, 8, 150])
def test_what_lies_behind_the_limits_does_not_matter(T):
    """Not-a-number scales and any codes in blocks that are not visible, block numbers that are never needed, codes behind the last token."""
    rng, c, table, q = attend_case(T + 6, 2, T, 2, 4, 128, 16, 400, spare=3)
    limits = causal([333, 150], T)
    want = c.attend(q, table, limits, 0.1)
    t2 = table.copy()
    unused = [n for n in range(c.k.shape[0]) if n not in set(table.ravel())]
    for b, longest in ((0, 333), (1, 150)):
        first = -(-longest // 16)
        t2[b, first:] = rng.choice([-7, 2 ** 30, unused[0]], size=table.shape[1] - first)
        c.k[table[b, first - 1], :, longest % 16 or 16:] = 127
        c.v[table[b, first - 1], :, longest % 16 or 16:] = -127
        gone = table[b, first:]
        c.k[gone], c.v[gone] = 127, 127
        c.ks[gone] = c.vs[gone] = 0x7E00                      # not a number
    c.ks[unused] = c.vs[unused] = 0x7C00                      # infinity
    c.upload()
    assert torch.equal(c.attend(q, t2, limits, 0.1), want)
    B.w4a8_check_status(c.ws)


@pytest.mark.parametrize("T", [1, 8, 150])
def test_blocks_that_do_not_exist_are_left_out(T):
    rng, c, table, q = attend_case(T + 7, 1, T, 2, 4, 64, 32, 400, spare=0)
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        t2 = table.copy()
        t2[0, 3] = bad
        c.check_attend(q, t2, causal([400], T))
        with pytest.raises(B.W4A8Error) as e:
            B.w4a8_check_status(c.ws)
        assert e.value.code == B.ERR_INDEX
    t2[:] = -1                                                # nothing is there at all
    assert (c.attend(q, t2, causal([400], T), 0.1) == 0).all()


@pytest.mark.parametrize("T", [1, 8, 150])
def test_scales_of_zero(T):
    rng, c, table, q = attend_case(T + 8, 1, T, 1, 4, 128, 16, 200)
    c.ks[table[0, 3]], c.vs[table[0, 5]], c.ks[table[0, 7]], c.vs[table[0, 7]] = 0, 0, 0, 0
    c.v[table[0, [5, 7]]] = 0                                 # what an append leaves where all values are zero
    c.upload()
    c.check_attend(q, table, causal([200], T))
    c.vs[:], c.v[:] = 0, 0
    c.upload()
    assert (c.attend(q, table, causal([200], T), 0.1) == 0).all()


@pytest.mark.parametrize("T", [1, 8, 150])
def test_a_row_that_is_not_a_number_stays_alone(T):
    rng, c, table, q = attend_case(T + 9, 1, T, 2, 4, 128, 64, 300)
    limits = causal([300], T)
    clean = c.attend(q, table, limits, 0.1).view(T, 8, 128)
    for poison in (0x7F80, 0x7FC0):                           # infinity, not a number
        bad = q.copy()
        bad[0, T // 2, 5, 17] = poison
        got = c.attend(bad, table, limits, 0.1).view(T, 8, 128)
        assert torch.isnan(got[T // 2, 5]).all()
        got[T // 2, 5] = clean[T // 2, 5]
        assert torch.equal(got, clean)


@pytest.mark.parametrize("T,keys", [(1, 5000), (8, 5000), (200, 1500)])
def test_attention_strides_streams_and_graphs(T, keys):
    """Rows of q as columns of a wider matrix; another stream; a captured call replayed on new inputs; the same bits every time."""
    rng, c, table, q = attend_case(T + 10, 1, T, 2, 4, 128, 64, keys)
    limits = causal([keys], T)
    want = c.check_attend(q, table, limits)
    wide = torch.full((T, 8 * 128 + 64 + 256), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 64:64 + 1024] = t_u16(q.reshape(T, -1), torch.bfloat16)
    view = wide[:, 64:64 + 1024].unflatten(1, (8, 128))
    out = torch.empty((T, 1024), dtype=torch.bfloat16, device="cuda")
    tt, lt = i32(table), i32(limits)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    B.w4a8_kv8_attention(view, c.dev, tt, lt, 128 ** -0.5, c.ws, out=out, stream=side)
    side.synchronize()
    first = out.clone()
    assert np.array_equal(onp.bf16_bits_to_f64(bits(first)).reshape(want.shape), want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.w4a8_kv8_attention(view, c.dev, tt, lt, 128 ** -0.5, c.ws, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    lt.fill_(keys // 2)                                       # the sequence as it was earlier, without a new capture
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, c.attend(q, table, np.full((1, T), keys // 2), 128 ** -0.5))


def test_a_cache_beyond_32_bit_offsets():
    """Block numbers whose codes lie past 4 GB."""
    rng = np.random.default_rng(12)
    blocks, heads, block, dim = 36000, 8, 128, 128
    small = Cache(rng, 8, heads, block, dim)
    dev = B.KV8Cache.empty(blocks, heads, dim, block)
    numbers = np.array([35999, 1, 34000, 17000, 35998, 20000, 33333, 30001])
    n = torch.from_numpy(numbers).cuda()
    for big, little in ((dev.k_codes, small.dev.k_codes), (dev.v_codes, small.dev.v_codes), (dev.k_scales, small.dev.k_scales), (dev.v_scales, small.dev.v_scales)):
        big[n] = little
    table = rng.permutation(8).reshape(1, 8)
    for T in (1, 8, 100):
        q = bf16(rng.standard_normal((1, T, 32, dim)))
        limits = causal([1000], T)
        want = small.attend(q, table, limits, 0.1)
        got = B.w4a8_kv8_attention(t_u16(q[0], torch.bfloat16), dev, i32(numbers[table]), i32(limits), 0.1, small.ws)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    k, v = new_values(rng, 1, 200, heads, dim)
    small.append(k, v, table, [130])
    B.w4a8_kv8_append(dev, t_u16(k[0], torch.bfloat16), t_u16(v[0], torch.bfloat16), i32(numbers[table]), i32([130]), small.ws)
    torch.cuda.synchronize()
    for big, little in ((dev.k_codes, small.dev.k_codes), (dev.v_codes, small.dev.v_codes), (dev.k_scales, small.dev.k_scales), (dev.v_scales, small.dev.v_scales)):
        assert torch.equal(big[n], little)


def test_cache_refusals():
    _, c, table, q = attend_case(1, 2, 3, 2, 4, 64, 16, 64)
    qt, tt, lt = t_u16(q.reshape(6, 8, 64), torch.bfloat16), i32(table), i32(causal([64, 64], 3))
    k = torch.zeros((6, 2, 64), dtype=torch.bfloat16, device="cuda")
    start = i32([0, 0])
    good = dict(q=qt, cache=c.dev, table=tt, limits=lt, scale=0.1, workspace=c.ws)
    for bad, code in ((dict(q=qt[:5], limits=lt), B.ERR_SHAPE), (dict(limits=lt[:1]), B.ERR_SHAPE), (dict(q=qt[:, :7].contiguous()), B.ERR_SHAPE),
                      (dict(workspace=c.ws[:4096]), B.ERR_WORKSPACE), (dict(q=qt[:, :, :32].contiguous()), B.ERR_SHAPE),
                      (dict(out=torch.empty(5, dtype=torch.bfloat16, device="cuda")), B.ERR_SHAPE)):
        with pytest.raises(B.W4A8Error) as e:
            B.w4a8_kv8_attention(**{**good, **bad})
        assert e.value.code == code
    for bad in (dict(q=qt.float()), dict(table=tt.long()), dict(limits=lt.cpu()), dict(q=qt.transpose(0, 1))):
        with pytest.raises(TypeError):
            B.w4a8_kv8_attention(**{**good, **bad})
    good = dict(cache=c.dev, k=k, v=k.clone(), table=tt, start=start, workspace=c.ws)
    for bad, code in ((dict(start=start[:1]), B.ERR_SHAPE), (dict(k=k[:5], v=k[:5]), B.ERR_SHAPE), (dict(v=k[:3]), B.ERR_SHAPE),
                      (dict(count=i32([1])), B.ERR_SHAPE), (dict(workspace=c.ws[:2048]), B.ERR_WORKSPACE), (dict(k=k[:, :1], v=k[:, :1]), B.ERR_SHAPE)):
        with pytest.raises(B.W4A8Error) as e:
            B.w4a8_kv8_append(**{**good, **bad})
        assert e.value.code == code
    assert B.w4a8_kv8_attention(qt[:0], c.dev, tt[:0], lt[:0], 0.1, c.ws).shape == (0, 512)
    B.w4a8_kv8_append(c.dev, k[:0], k[:0], tt, start, c.ws)
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("T", [1, 8, 150])
@pytest.mark.parametrize("dim,keys", [(64, 90), (128, 900)])
def test_rows_without_a_key_beside_large_value_scales(T, dim, keys):
    """Their sums hold nothing, also where the reciprocals of the scales are small; the other rows' do not gain from what is masked."""
    _, c, table, q = attend_case(T + dim, 2, T, 1, 4, dim, 16, keys, v_scale=(20000.0, 60000.0))
    limits = causal([keys, keys - 50], T)
    limits[:, ::3] = 0
    got = c.check_attend(q, table, limits)
    assert (got[limits == 0] == 0).all()


@pytest.mark.parametrize("T", [8, 150])
def test_many_blocks_of_scale_zero_with_next_to_no_weight(T):
    """Values of zero whose keys score far below the others: they change neither sum nor result, however many there are."""
    _, c, table, q = attend_case(T, 1, T, 1, 4, 64, 16, 120000)
    q[:] = bf16(np.ones(q.shape))
    c.k[:] = -127                                             # scores of -50.8, the first block's 0.4
    c.ks[:] = onp.f64_to_fp16_bits(np.float64(0.05))
    c.vs[:], c.v[:] = 0, 0
    first = table[0, 0]
    c.k[first], c.v[first], c.vs[first] = 1, 100, onp.f64_to_fp16_bits(np.float64(60000.0))
    c.upload()
    got = c.check_attend(q, table, np.full((1, T), 120000))
    assert np.abs(got / 6e6 - 1).max() <= 2.0 ** -7


@pytest.mark.parametrize("B_,T,heads,rep,dim,block,keys", [(1, 1024, 8, 4, 128, 64, 1400), (2, 400, 10, 4, 64, 16, 1500), (90, 33, 1, 1, 64, 32, 1300)])
@pytest.mark.parametrize("shape", ["even", "rising", "one long", "none"])
def test_attention_where_some_tiles_are_long(B_, T, heads, rep, dim, block, keys, shape):
    """Nearly as many row tiles as SMs, of equal and of very different lengths, rows without a key among them."""
    _, c, table, q = attend_case(B_ + T, B_, T, heads, rep, dim, block, keys)
    limits = np.full((B_, T), keys)
    if shape == "rising":
        limits = (keys * (np.arange(B_ * T) + 1) // (B_ * T)).reshape(B_, T)
        limits[0, :5] = 0
    elif shape != "even":
        limits[:] = 0 if shape == "none" else 100
        limits[B_ // 2, T // 2] = 0 if shape == "none" else keys
        limits[B_ - 1, 3] = 0
    got = c.check_attend(q, table, limits)
    assert (got[limits == 0] == 0).all()
    again = c.attend(q, table, limits, dim ** -0.5)
    assert torch.equal(again, c.attend(q, table, limits, dim ** -0.5))


@pytest.mark.parametrize("T", [1, 8, 150])
def test_blocks_that_are_shared(T):
    """Sequences with a common prefix, and one that names a block twice."""
    _, c, table, q = attend_case(T + 40, 3, T, 2, 4, 64, 16, 400)
    table[1, :7] = table[0, :7]
    table[2, 9] = table[2, 3]
    c.check_attend(q, table, causal([400, 333, 390], T))


def test_two_graphs_on_one_workspace():
    """Captured calls of different kernels that share a workspace, replayed in turn."""
    cases = []
    for T, keys in ((1, 3000), (150, 900)):
        _, c, table, q = attend_case(T + 41, 1, T, 2, 4, 128, 64, keys)
        cases.append((c, i32(table), t_u16(q[0], torch.bfloat16), i32(causal([keys], T)), torch.empty((T, 1024), dtype=torch.bfloat16, device="cuda")))
    ws = cases[0][0].ws
    want = [B.w4a8_kv8_attention(q, c.dev, t, l, 0.1, ws) for c, t, q, l, _ in cases]
    torch.cuda.synchronize()
    graphs = []
    for c, t, q, l, out in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.w4a8_kv8_attention(q, c.dev, t, l, 0.1, ws, out=out)
        graphs.append(g)
    for i in (0, 1, 0, 0, 1, 1, 0):
        cases[i][-1].zero_()
        graphs[i].replay()
        graphs[1 - i].replay()
        torch.cuda.synchronize()
        for (*_, out), w in zip(cases, want):
            assert torch.equal(out, w)


@pytest.mark.parametrize("T,B_", [(1, 1), (3, 5), (8, 2), (37, 3), (150, 1), (300, 2)])
def test_rows_behind_the_last_are_left_as_they_are(T, B_):
    """Outputs in the middle of larger buffers, not-a-number in front of and behind q's rows."""
    _, c, table, q = attend_case(T + 60, B_, T, 2, 3, 64, 16, 310)
    limits = causal([310 - 7 * b for b in range(B_)], T)
    M = B_ * T
    big = torch.full((M + 40, 6 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    qb = torch.full((M + 40, 6, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    qb[20:20 + M] = t_u16(q.reshape(M, 6, 64), torch.bfloat16)
    B.w4a8_kv8_attention(qb[20:20 + M], c.dev, i32(table), i32(limits), 0.1, c.ws, out=big[20:20 + M])
    torch.cuda.synchronize()
    assert torch.equal(big[20:20 + M], c.attend(q, table, limits, 0.1))
    assert (big[:20] == 7).all() and (big[20 + M:] == 7).all()
    x, r, w = norm_case(M, 640, T)
    outs = [torch.full((M + 2, n), 5, dtype=t, device="cuda") for n, t in ((640, torch.bfloat16), (640, torch.int8), (1, torch.float16), (5, torch.int32))]
    s, qa, sa, asum = (o[1:1 + M] for o in outs)
    B.w4a8_add_rmsnorm_quantize(t_u16(x, torch.bfloat16), t_u16(w, torch.bfloat16), 1e-6, residual=t_u16(r, torch.bfloat16), sum_out=s, out=(qa, sa.view(-1), asum))
    torch.cuda.synchronize()
    assert all((o[0] == 5).all() and (o[-1] == 5).all() for o in outs)


def test_many_sequences():
    """The largest grids: 65528 (sequence, head) pairs that all read the same blocks, for single tokens, draft blocks and more rows; as many appends."""
    n, heads = 8191, 8
    _, c, table, q = attend_case(70, 1, 40, heads, 1, 64, 16, 50)
    wide = torch.from_numpy(np.repeat(table, n, axis=0).astype(np.int32)).cuda()
    for T in (1, 20, 40):
        limits = causal([50], T)
        want = c.attend(q[:, :T], table, limits, 0.1)
        got = B.w4a8_kv8_attention(t_u16(q[0, :T], torch.bfloat16).repeat(n, 1, 1), c.dev, wide, i32(np.repeat(limits, n, axis=0)), 0.1, c.ws)
        torch.cuda.synchronize()
        assert (got.view(n, T, -1) == want).all()
    rng = np.random.default_rng(71)
    k, v = new_values(rng, 1, 3, heads, 64)
    one, many = Cache(rng, 1, heads, 16, 64), B.KV8Cache.empty(n, heads, 64, 16)
    one.append(k, v, np.array([[0]]), [0])
    B.w4a8_kv8_append(many, t_u16(k[0], torch.bfloat16).repeat(n, 1, 1), t_u16(v[0], torch.bfloat16).repeat(n, 1, 1),
                      torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.zeros(n, dtype=torch.int32, device="cuda"), one.ws)
    torch.cuda.synchronize()
    assert (many.k_codes[:, :, :3] == one.dev.k_codes[:, :, :3]).all() and (many.v_codes[:, :, :3] == one.dev.v_codes[:, :, :3]).all()
    assert (many.k_scales == one.dev.k_scales).all() and (many.v_scales == one.dev.v_scales).all()
