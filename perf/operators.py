"""What a decoder layer does between its quantised linears, as cases that can be timed and compared.

Three operators, used together: the norm in front of the QKV and the gate+up projection (residual stream added, result
quantised for the linear behind it), the append of new keys and values to a cache held in 8 bits with one scale per block of
tokens and head, and the attention that reads that cache.  Token counts are those of streaming inference: one decode token,
a draft block of 8 tokens, a few requests together, a ragged chunk, a window of new-frame tokens, a whole prompt.

What is held in 8 bits is returned as the values it stands for (code x scale, fp16).
"""
import math
import random

import torch

own = False

GROUP = 128
EPS = 1e-6
# query heads over key/value heads: the 8B-class layer's, then ratios from 1 to 8, odd ones among them
HEADS = ((32, 8), (16, 2), (8, 8), (40, 8), (12, 4), (28, 4))


def _norm(name, tokens, k, add):
    return dict(name=name, kind="norm", tokens=tokens, k=k, add=add)


def _append(name, seqs, tokens, heads, dim, block, start):
    return dict(name=name, kind="append", seqs=seqs, tokens=tokens, heads=heads, dim=dim, block=block, start=start)


def _attend(name, seqs, tokens, keys, heads=HEADS[0], dim=128, block=64, views=0):
    """views = 0: causal, the rows are the last `tokens` of a sequence's keys; else `views` camera views of keys / tokens frames each."""
    return dict(name=name, kind="attend", seqs=seqs, tokens=tokens, keys=keys, q_heads=heads[0], kv_heads=heads[1], dim=dim, block=block,
                views=views)


def listed():
    return [
        # one decode token: the residual stream, its norm, the operands of the next projection
        _norm("norm_decode_1", 1, 4096, True),
        # a ragged chunk whose residual was added in the projection before
        _norm("norm_chunk_200", 200, 2048, False),
        # the whole window as one prompt, a layer a size up
        _norm("norm_prompt_4096", 4096, 5120, True),
        # one decode token into a block that is partly full
        _append("append_decode_1", 1, 1, 8, 128, 64, 37),
        # five requests with a draft block each, some shorter (padded), small blocks
        _append("append_batch_5x8", 5, 8, 4, 64, 16, 21),
        # a ragged chunk of new tokens behind a partly full block
        _append("append_chunk_1391", 1, 1391, 8, 128, 128, 77),
        # one decode token over a window
        _attend("attend_decode_1", 1, 1, 4096),
        # verification of a draft block over a long cache, odd length
        _attend("attend_verify_8_long", 1, 8, 32749),
        # many requests with one token each, ragged lengths, an empty place among them
        _attend("attend_batch_33", 33, 1, 4001, (16, 2), 64, 16),
        # a ragged chunk behind a cached prefix
        _attend("attend_chunk_200", 1, 200, 2900, (28, 4), 128, 32),
        # streaming prefill: the newest frame's tokens of four views in a window of four frames
        _attend("attend_stream_1024", 1, 1024, 4096, views=4),
        # the whole window as one prompt, causal
        _attend("attend_prompt_4096", 1, 4096, 4096, block=128),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "append", "attend", "attend", "attend"))
    block, dim = rng.choice((16, 32, 64, 128)), rng.choice((64, 128))
    if kind == "norm":
        return dict(kind=kind, tokens=_log_int(rng, 1, 4096), k=GROUP * _log_int(rng, 1, 40), add=rng.random() < 0.6)
    heads = rng.choice(HEADS)
    if kind == "append":
        seqs = _log_int(rng, 1, 64)
        tokens = _log_int(rng, 1, min(2048, 4096 // seqs))
        return dict(kind=kind, seqs=seqs, tokens=tokens, heads=heads[1], dim=dim, block=block, start=rng.randint(0, 2 * block))
    if rng.random() < 0.2:                                    # streaming: views x frames x tokens of a frame
        views, frames, n = rng.randint(1, 4), rng.randint(1, 6), _log_int(rng, 8, 170)
        return dict(kind=kind, seqs=1, tokens=views * n, keys=views * frames * n, q_heads=heads[0], kv_heads=heads[1], dim=dim, block=block, views=views)
    seqs = _log_int(rng, 1, 64)
    tokens = rng.randint(1, 16) if rng.random() < 0.6 else _log_int(rng, 17, max(17, 3200 // seqs))
    most = min(65536, 26 * 10 ** 7 // (seqs * tokens * heads[0]), 10 ** 8 // (seqs * heads[1] * dim))
    keys = max(tokens, _log_int(rng, 1, max(2, most)))
    return dict(kind=kind, seqs=seqs, tokens=tokens, keys=keys, q_heads=heads[0], kv_heads=heads[1], dim=dim, block=block, views=0)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _counts(c):
    """New tokens of each sequence: all of them, but every third sequence stops short (a padded batch)."""
    return [c["tokens"] - (c["tokens"] // 3 if b % 3 == 1 else 0) for b in range(c["seqs"])]


def _starts(c):
    return [c["start"] + (b * 5) % (c["block"] + 3) for b in range(c["seqs"])]


def _limits(c):
    """How many leading positions each row sees, [seqs][tokens]."""
    t = c["tokens"]
    if c["views"]:                                            # view-major order, the newest frame's tokens of each view are the rows
        n, frames = t // c["views"], c["keys"] // t
        return [[(v * frames + frames - 1) * n + i + 1 for v in range(c["views"]) for i in range(n)]]
    rng = random.Random(c["seqs"] * 7919 + c["keys"])
    rows = []
    for b in range(c["seqs"]):
        keys = c["keys"] if b == 0 else max(t, int(c["keys"] * rng.uniform(0.2, 1.0)))
        full = [keys - t + 1 + i for i in range(t)]
        if b % 8 == 2:                                        # a place of the batch that is not in use, or half of one
            full[(0 if t == 1 else t // 2):] = [0] * len(full[(0 if t == 1 else t // 2):])
        rows.append(full)
    return rows


def _ceil(a, b):
    return -(-a // b)


def _cache(gen, blocks, heads, block, dim, outliers):
    """Codes and scales of N(0, 1) values, as an append into fresh blocks leaves them; `outliers`: a few channels four times as large."""
    x = torch.randn((blocks, heads, block, dim), generator=gen, device="cuda")
    if outliers:
        x[..., torch.randperm(dim, generator=gen, device="cuda")[:2]] *= 4
    scale = (x.abs().amax((2, 3)) / 127).half()
    codes = (x / scale.float()[:, :, None, None]).round_().clamp_(-127, 127).to(torch.int8)
    return codes, scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, s = case, dict(case)
    if c["kind"] == "norm":
        m, k = c["tokens"], c["k"]
        x = torch.randn((m, k), generator=gen, device="cuda")
        x[:, torch.randperm(k, generator=gen, device="cuda")[: max(1, k // 100)]] *= 20
        s["x"] = x.to(torch.bfloat16)
        s["residual"] = torch.randn((m, k), generator=gen, device="cuda").mul_(4).to(torch.bfloat16) if c["add"] else None
        s["weight"] = torch.rand((k,), generator=gen, device="cuda").add_(0.5).to(torch.bfloat16)
        s["sum"] = torch.empty((m, k), dtype=torch.bfloat16, device="cuda") if c["add"] else None
        s["q"] = (torch.empty((m, k), dtype=torch.int8, device="cuda"), torch.empty((m,), dtype=torch.float16, device="cuda"),
                  torch.empty((m, k // GROUP), dtype=torch.int32, device="cuda"))
        return s
    n, t, d, block = c["seqs"], c["tokens"], c["dim"], c["block"]
    i32 = dict(dtype=torch.int32, device="cuda")
    if c["kind"] == "append":
        heads = c["heads"]
        starts = _starts(c)
        width = _ceil(max(starts) + t, block)
        # keys and values as they lie in the QKV projection's rows, behind four times as many query channels
        s["qkv"] = torch.randn((n * t, 6 * heads * d), generator=gen, device="cuda").mul_(1.5).to(torch.bfloat16)
        s["k"], s["v"] = (s["qkv"][:, i * heads * d:(i + 1) * heads * d].view(n * t, heads, d) for i in (4, 5))
        s["start"], s["count"] = torch.tensor(starts, **i32), torch.tensor(_counts(c), **i32)
    else:
        heads = c["kv_heads"]
        limits = _limits(c)
        width = _ceil(max(max(r) for r in limits), block)
        s["q"] = torch.randn((n * t, c["q_heads"], d), generator=gen, device="cuda").mul_(1.5).to(torch.bfloat16)
        s["limits"] = torch.tensor(limits, **i32)
        s["out"] = torch.empty((n * t, c["q_heads"] * d), dtype=torch.bfloat16, device="cuda")
        s["scale"] = d ** -0.5
    blocks = n * width + 1
    s["table"] = torch.randperm(blocks, generator=gen, device="cuda")[: n * width].view(n, width).to(torch.int32)
    s["k_codes"], s["k_scales"] = _cache(gen, blocks, heads, block, d, True)
    s["v_codes"], s["v_scales"] = _cache(gen, blocks, heads, block, d, False)
    if own:                                                   # the handle and the workspace that a program makes once and keeps
        from paper_2608_12932_b200 import binding as w4a8
        s["cache"] = w4a8.KV8Cache(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"])
        s["workspace"] = w4a8.new_kv8_workspace(s["cache"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2608_12932_b200 import binding as w4a8
    if s["kind"] == "norm":
        total, qa, sa, asum = w4a8.w4a8_add_rmsnorm_quantize(s["x"], s["weight"], EPS, residual=s["residual"], sum_out=s["sum"], out=s["q"])
        scale = sa[:, None]
        r = {"codes": qa * scale, "sums": asum * scale, "scale": sa}
        return dict(r, sum=total) if s["add"] else r
    if s["kind"] == "append":
        w4a8.w4a8_kv8_append(s["cache"], s["k"], s["v"], s["table"], s["start"], s["workspace"], count=s["count"])
        return {"k": s["k_codes"] * s["k_scales"][:, :, None, None], "v": s["v_codes"] * s["v_scales"][:, :, None, None]}
    return w4a8.w4a8_kv8_attention(s["q"], s["cache"], s["table"], s["limits"], s["scale"], s["workspace"], out=s["out"])


def _plain_norm(s):
    x = s["x"].float()
    total = (x + s["residual"].float()).to(torch.bfloat16) if s["add"] else s["x"]
    f = total.float()
    h = (f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * s["weight"].float()).to(torch.bfloat16).float()
    sa = (h.abs().amax(1) / torch.full((), 127.0, device=h.device)).clamp_max(65504.0).half()
    scale = sa.float()[:, None]
    codes = torch.where(scale > 0, (h / scale).round().clamp(-127, 127), torch.zeros((), device=h.device))
    sums = codes.view(h.shape[0], -1, GROUP).sum(2)
    r = {"codes": (codes * scale).half(), "sums": (sums * scale).half(), "scale": sa}
    return dict(r, sum=total) if s["add"] else r


def _plain_append(s, x, codes, scales):
    """Token i of sequence b to position start[b] + i: every block that a sequence can touch is taken out, rewritten and put back."""
    n, t, heads, d, block = s["seqs"], s["tokens"], s["heads"], s["dim"], s["block"]
    width, touched = s["table"].shape[1], (t + block - 2) // block + 1
    start, count = s["start"].long()[:, None], s["count"].long()[:, None]
    index = start // block + torch.arange(touched, device="cuda")                        # [n, touched]: the block's place in the table
    number = s["table"].long().gather(1, index.clamp_max(width - 1))
    pos = index[:, :, None] * block + torch.arange(block, device="cuda")                 # [n, touched, block]
    new = (pos >= start[:, :, None]) & (pos < (start + count)[:, :, None])
    live = new.any(2) & (index < width)
    at = (pos - start[:, :, None]).clamp(0, t - 1) + torch.arange(n, device="cuda")[:, None, None] * t
    value = x.float()[at].permute(0, 1, 3, 2, 4)                                         # [n, touched, heads, block, d]
    new = new[:, :, None, :, None]
    amax = torch.where(new, value.abs(), torch.zeros((), device="cuda")).amax((3, 4))
    held = (index * block < start)[:, :, None]
    before = torch.where(held, scales[number], torch.zeros((), dtype=torch.float16, device="cuda"))
    scale = torch.maximum(before, (amax / torch.full((), 127.0, device="cuda")).clamp_max(65504.0).half())
    div = scale.float()[..., None, None]
    old = codes[number].float()
    kept = torch.where((pos < start[:, :, None])[:, :, None, :, None], (old * before.float()[..., None, None] / div).round(), old)
    got = torch.where(new, (value / div).round(), kept)
    got = torch.where((div > 0) | (pos >= (start + count)[:, :, None])[:, :, None, :, None], got, torch.zeros((), device="cuda"))
    codes[number[live]] = got.clamp(-128, 127)[live].to(torch.int8)
    scales[number[live]] = scale[live]
    return (codes.float() * scales.float()[:, :, None, None]).half()


def _plain_attend(s):
    n, t, d, block = s["seqs"], s["tokens"], s["dim"], s["block"]
    kv, rep = s["kv_heads"], s["q_heads"] // s["kv_heads"]
    width = s["table"].shape[1]
    number = s["table"].long()

    def values(codes, scales):                                # [n, kv, width * block, d]
        v = codes[number].float() * scales[number].float()[..., None, None]
        return v.permute(0, 2, 1, 3, 4).reshape(n, kv, width * block, d)

    q = s["q"].float().view(n, t, kv, rep, d).permute(0, 2, 1, 3, 4).reshape(n, kv, t * rep, d) * s["scale"]
    score = torch.matmul(q, values(s["k_codes"], s["k_scales"]).transpose(2, 3)).view(n, kv, t, rep, width * block)
    seen = (torch.arange(width * block, device="cuda") < s["limits"][:, :, None])[:, None, :, None, :]
    score = score.masked_fill_(~seen, -math.inf)
    top = score.amax(4, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(4, keepdim=True)
    o = torch.matmul(p.view(n, kv, t * rep, width * block), values(s["v_codes"], s["v_scales"])).view(n, kv, t, rep, d)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 2, 1, 3, 4).reshape(n * t, s["q_heads"] * d).to(torch.bfloat16)


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "norm":
        return _plain_norm(s)
    if s["kind"] == "append":
        return {"k": _plain_append(s, s["k"], s["k_codes"], s["k_scales"]), "v": _plain_append(s, s["v"], s["v_codes"], s["v_scales"])}
    return _plain_attend(s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "norm":
        e = c["tokens"] * c["k"]
        return {"bytes": e * (7 if c["add"] else 3) + 2 * c["k"] + 2 * c["tokens"] + 4 * e // GROUP, "flops": 6 * e}
    if c["kind"] == "append":
        row = c["heads"] * c["dim"]
        touched = sum(_ceil(a + m, c["block"]) - a // c["block"] for a, m in zip(_starts(c), _counts(c)))
        return {"bytes": 2 * 3 * row * sum(_counts(c)) + 4 * c["heads"] * touched + 4 * touched + 8 * c["seqs"], "flops": 6 * row * sum(_counts(c))}
    limits = _limits(c)
    keys = sum(max(r) for r in limits)
    blocks = sum(_ceil(max(r), c["block"]) for r in limits)
    rows = c["seqs"] * c["tokens"] * c["q_heads"] * c["dim"]
    return {"bytes": 2 * keys * c["kv_heads"] * c["dim"] + 4 * blocks * c["kv_heads"] + 4 * blocks + 4 * rows + 4 * c["seqs"] * c["tokens"],
            "flops": 4 * c["q_heads"] * c["dim"] * sum(map(sum, limits))}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def _exact_scale(amax):
    """fp16(amax / 127), as the codes' scale is defined."""
    return (amax / 127.0).clamp(max=65504.0).to(torch.float16).double()


def _exact_norm(s):
    total = s["x"].double()
    if s["add"]:
        total = (total + s["residual"].double()).to(torch.bfloat16).double()             # the stream is held in bf16
    size = total.pow(2).sum(1).div(s["k"]).add(EPS).sqrt()
    h = (total / size[:, None] * s["weight"].double()).to(torch.bfloat16).double()       # the quantiser takes bf16
    scale = _exact_scale(h.abs().max(1).values)[:, None]
    codes = torch.nan_to_num(h / scale, nan=0.0).round().clamp(-127.0, 127.0)
    r = {"codes": codes * scale, "sums": codes.reshape(codes.shape[0], -1, GROUP).sum(-1) * scale, "scale": scale[:, 0]}
    return dict(r, sum=total) if s["add"] else r


def _exact_append(s, x, codes, scales):
    q, f = codes.double(), scales.double()
    x = x.double()
    for b, (start, count) in enumerate(zip(s["start"].tolist(), s["count"].tolist())):
        table, done = s["table"][b].tolist(), 0
        while done < count:
            pos = start + done
            number, slot = table[pos // s["block"]], pos % s["block"]
            take = min(s["block"] - slot, count - done)
            rows = x[b * s["tokens"] + done: b * s["tokens"] + done + take].transpose(0, 1)          # [heads, take, dim]
            scale = _exact_scale(rows.abs().amax((1, 2)))
            if slot:
                scale = torch.maximum(scale, f[number])
                q[number, :, :slot] = (q[number, :, :slot] * f[number][:, None, None] / scale[:, None, None]).round().clamp(-127, 127)
            q[number, :, slot:slot + take] = (rows / scale[:, None, None]).round().clamp(-127, 127)
            f[number] = scale
            done += take
    return q * f[:, :, None, None]


def _exact_attend(s):
    d, rep = s["dim"], s["q_heads"] // s["kv_heads"]
    out = torch.zeros((s["seqs"], s["tokens"], s["q_heads"], d), dtype=torch.float64, device="cuda")
    q = s["q"].double().view(s["seqs"], s["tokens"], s["q_heads"], d)
    for b in range(s["seqs"]):
        limit = s["limits"][b].long()
        length = int(limit.max())
        if not length:
            continue
        table = s["table"][b, : _ceil(length, s["block"])].long()
        hidden = torch.arange(length, device="cuda")[None, :] >= limit[:, None]
        for g in range(s["kv_heads"]):
            k, v = ((c[table, g].double() * f[table, g].double()[:, None, None]).reshape(-1, d)[:length]
                    for c, f in ((s["k_codes"], s["k_scales"]), (s["v_codes"], s["v_scales"])))
            for h in range(g * rep, (g + 1) * rep):
                w = torch.softmax((q[b, :, h] @ k.T * s["scale"]).masked_fill(hidden, -1e300), 1).masked_fill(hidden, 0.0)
                out[b, :, h] = w @ v
    return out.reshape(s["seqs"] * s["tokens"], s["q_heads"] * d)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    if case["kind"] == "append":
        return {"k": _exact_append(s, s["k"], s["k_codes"], s["k_scales"]), "v": _exact_append(s, s["v"], s["v_codes"], s["v_scales"])}
    return _exact_attend(s)
