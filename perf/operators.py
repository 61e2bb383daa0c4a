"""Operator cases of the paged KV pool: appending a step's keys and values (with the position rotation applied on the
way) and attending over the pool, each on a 16-bit pool and on an 8-bit (e4m3) pool with one scale for every block of
tokens and KV head.

`run` computes a case in elementary torch operations (`own` false) or through the library's calls (`own` true); `exact`
states the same operators in 64 bits, one sequence and head at a time."""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
SCALE_FLOOR = 2.0 ** -100


def case_(name, op, cache, dtype, heads, kv_heads, dim, block, seqs, prefix, new, *, hnd=False, style="half", rot=None, mix=1):
    """prefix and new: (lowest, highest) tokens of a sequence that are in the pool already and that the step brings."""
    c = {"op": op, "cache": cache, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block, "seqs": seqs,
         "prefix_lo": prefix[0], "prefix_hi": prefix[1], "new_lo": new[0], "new_hi": new[1], "hnd": hnd, "mix": mix}
    if op == "append":
        c |= {"style": style, "rot": rot or dim}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one decode step of a 64-request batch (the batch size of the 1-token-page workload): latency
        case_("append decode", "append", "16", "bf16", 32, 8, 128, 16, 64, (511, 4095), (1, 1)),
        # the prompts of four requests behind restored prefixes
        case_("append prefill", "append", "16", "bf16", 32, 8, 128, 16, 4, (0, 4096), (4096, 4096)),
        # the same two steps into an 8-bit pool; the second with ragged chunks and head-major blocks
        case_("append decode 8-bit", "append", "8", "bf16", 32, 8, 128, 16, 64, (511, 4095), (1, 1)),
        case_("append chunk 8-bit", "append", "8", "fp16", 64, 8, 128, 16, 8, (100, 4000), (1000, 2047), hnd=True, style="pairs"),
        # a few short chats: latency
        case_("decode short", "attend", "16", "fp16", 32, 8, 128, 16, 4, (99, 999), (1, 1)),
        # one request with a 131072-token prefix, 64 query heads (the 80-layer geometry)
        case_("decode 128K", "attend", "16", "bf16", 64, 8, 128, 16, 1, (131071, 131071), (1, 1)),
        # 64 ragged requests on 1-token pages
        case_("decode pages", "attend", "16", "bf16", 32, 8, 128, 1, 64, (511, 16383), (1, 1)),
        # 8 requests of 32768 tokens over an 8-bit pool
        case_("decode 8-bit", "attend", "8", "bf16", 32, 8, 128, 16, 8, (32767, 32767), (1, 1)),
        # ragged 8-bit decode, 64-wide heads, head-major blocks
        case_("decode 8-bit ragged", "attend", "8", "fp16", 32, 8, 64, 32, 48, (99, 8191), (1, 1), hnd=True),
        # new prompt chunks over restored prefixes
        case_("chunk", "attend", "16", "bf16", 32, 8, 128, 16, 2, (8192, 8192), (777, 1024)),
        case_("chunk 8-bit", "attend", "8", "fp16", 32, 8, 128, 16, 4, (2000, 9000), (300, 700), hnd=True),
        # a long prompt over a 32768-token prefix: the largest
        case_("chunk long", "attend", "16", "bf16", 32, 8, 128, 16, 1, (32768, 32768), (2048, 2048)),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend"])
    cache, dtype = rng.choice(["16", "8"]), rng.choice(["bf16", "fp16"])
    heads, kv_heads = rng.choice([(32, 8), (64, 8), (28, 4), (8, 8), (40, 8), (8, 1), (16, 16), (6, 2)])
    dim, block, hnd = rng.choice([64, 128, 128]), rng.choice([1, 8, 16, 16, 32, 64]), rng.random() < 0.3
    if cache == "8" and block == 1:
        block = 16
    mix = rng.randrange(1 << 20)
    if op == "append":
        new = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
        seqs = _log(rng, 1, max(1, min(64, 16384 // new)))
        prefix = _log(rng, 1, 4096)
        return case_("", op, cache, dtype, heads, kv_heads, dim, block, seqs, (prefix // 2, prefix), (max(1, new // 2), new), hnd=hnd,
                     style=rng.choice(["half", "pairs"]), rot=rng.choice([dim, dim // 2]), mix=mix)
    if rng.random() < 0.5:
        seqs = _log(rng, 1, 64)
        prefix = _log(rng, 1, min(131071, 393216 // seqs))
        return case_("", op, cache, dtype, heads, kv_heads, dim, block, seqs, (prefix // 4, prefix), (1, 1), hnd=hnd, mix=mix)
    new, seqs = _log(rng, 2, 2048), _log(rng, 1, 8)
    most = 32 * 2048 * 34816 // (heads * new * seqs) - new
    prefix = _log(rng, 1, max(1, min(32768, most)))
    while seqs > 1 and heads * seqs * new * (prefix + new) > 32 * 2048 * 34816:
        seqs //= 2
    return case_("", op, cache, dtype, heads, kv_heads, dim, block, seqs, (prefix // 2, prefix), (max(1, new // 2), new), hnd=hnd, mix=mix)


def lengths(c):
    """Tokens in the pool before the step and new ones, by sequence: part of the case, not of the seed."""
    rng = random.Random(c["mix"])
    return [(rng.randint(c["prefix_lo"], c["prefix_hi"]), rng.randint(c["new_lo"], c["new_hi"])) for _ in range(c["seqs"])]


def _csr(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV).manual_seed(seed)
    lens = lengths(c)
    dt, hq, hk, d, bs = TYPES[c["dtype"]], c["heads"], c["kv_heads"], c["dim"], c["block"]
    blocks = [-(-(p + n) // bs) for p, n in lens]
    need = sum(blocks)
    n_blocks = need + need // 4 + 1
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    n_tok = sum(n for _, n in lens)
    s = {"case": c, "q_start": ints(_csr([n for _, n in lens])), "ctx_len": ints([p + n for p, n in lens]),
         "blk_start": ints(_csr(blocks)), "block_ids": torch.randperm(n_blocks, generator=g, device=DEV)[:need].to(torch.int32),
         "n_tok": n_tok, "max_q": max(n for _, n in lens), "max_ctx": max(p + n for p, n in lens), "n_blocks": n_blocks}
    # a projection's output: queries, keys and values of a token side by side, a few features with larger values
    spread = torch.exp(torch.randn((hq + 2 * hk) * d, generator=g, device=DEV) * 0.4)
    packed = (torch.randn(n_tok, (hq + 2 * hk) * d, generator=g, device=DEV) * spread).to(dt)
    s["q"], s["k"], s["v"] = (packed[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    shape = (n_blocks, hk, bs, d) if c["hnd"] else (n_blocks, bs, hk, d)
    if c["cache"] == "16":
        s["pools"] = [torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g) for _ in range(2)]
    else:
        s["pools"] = [_codes(shape, g) for _ in range(2)]
        s["scales"] = [torch.exp2(torch.randint(-9, -5, (n_blocks, hk), generator=g, device=DEV).float()) for _ in range(2)]
    if c["op"] == "append":
        at = torch.arange(s["max_ctx"], dtype=torch.float64, device=DEV)[:, None]
        angle = at * 500000.0 ** (-torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV) * 2 / c["rot"])
        s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    return s


def _codes(shape, g):
    n, out = math.prod(shape), torch.empty(shape, dtype=E4M3, device=DEV)
    step = 1 << 26
    for a in range(0, n, step):
        parts = (torch.randn(min(step, n - a), generator=g, device=DEV) * 64).clamp_(-448, 448)
        out.view(-1)[a:a + step] = parts.to(E4M3)
    return out


# ---------------------------------------------------------------------------- the library's calls

_contexts = {}
LAYERS = 64


def _context(c):
    """The library context of a geometry (one for the program's life), its attention handle and how often a layer of it has
    been registered: the layers are taken in turn."""
    from paper_2605_03375_b200 import tutti as T
    size = 1 if c["cache"] == "8" else 2
    key = (c["kv_heads"], c["dim"], size, c["block"], c["hnd"])
    if key not in _contexts:
        ctx = T.Context(T.Geom(LAYERS, c["kv_heads"], c["dim"], size, c["block"], c["block"], 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
        ctx.tutti_set_option(T.OPT_POOL_LAYOUT, T.POOL_HND if c["hnd"] else T.POOL_NHD)
        _contexts[key] = [T, ctx, T.Attn(ctx), 0]
    return _contexts[key]


def _bind(s):
    """What a program sets up once for its pool and once for a step (all its layers share it): the registration and the step."""
    c = s["case"]
    entry = _context(c)
    T, ctx, attn, turn = entry
    entry[3] += 1
    layer = turn % LAYERS
    k, v = s["pools"]
    ctx.tutti_pool_register(layer, k.data_ptr(), v.data_ptr(), c["block"] * c["kv_heads"] * c["dim"] * k.element_size(), s["n_blocks"])
    if c["cache"] == "8":
        ctx.tutti_scales_register(layer, s["scales"][0].data_ptr(), s["scales"][1].data_ptr(), s["n_blocks"])
    step = T.make_step(s["q_start"], s["ctx_len"], s["blk_start"], s["block_ids"], s["n_tok"], s["max_q"])
    s["bound"], s["turn"] = (T, ctx, attn, layer, step), (entry, turn)
    return s["bound"]


def _bound(s):
    """The state's binding, made anew once its layer has been registered for another state."""
    if "bound" in s:
        entry, turn = s["turn"]
        if entry[3] - turn <= LAYERS:
            return s["bound"]
    return _bind(s)


def _own(s):
    c = s["case"]
    T, ctx, attn, layer, step = _bound(s)
    stream = torch._C._cuda_getCurrentRawStream(0)          # torch.cuda.current_stream().cuda_stream takes 4 us more
    if c["op"] == "append":
        out = torch.empty((s["n_tok"], c["heads"], c["dim"]), dtype=s["q"].dtype, device=DEV)
        rope = T.make_rope(s["table"], T.ROPE_HALF if c["style"] == "half" else T.ROPE_PAIRS)
        ctx.tutti_kv_append_layer(layer, step, T.make_tokens(s["k"], s["v"], s["q"], out), rope, stream)
        return {"q": out, "pools": s["pools"], "scales": s.get("scales")}
    out = torch.empty((s["n_tok"], c["heads"], c["dim"]), dtype=s["q"].dtype, device=DEV)
    lse = torch.empty((s["n_tok"], c["heads"]), dtype=torch.float32, device=DEV)
    attn.tutti_kv_attend_layer(layer, step, T.make_attend(s["q"], out, lse), c["dim"] ** -0.5, stream)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------- plain forms

def _rotate(x, table, c):
    """x [token, head, dim] in 32 bits, table [token, cos | sin]."""
    r = c["rot"]
    cos, sin = table[:, None, :r // 2], table[:, None, r // 2:]
    if c["style"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., r:]], -1)


def _places(s):
    """Sequence and position of every token of the step."""
    t = torch.arange(s["n_tok"], device=DEV)
    q_start = s["q_start"].long()
    seq = torch.bucketize(t, q_start[1:], right=True)
    return seq, s["ctx_len"].long()[seq] - q_start[seq + 1] + t


def _token_major(pool, c):
    return pool.transpose(1, 2) if c["hnd"] else pool


def _pow2_scale(amax):
    """The smallest power of two s with amax / s <= 448, at least the floor: 448 = 0.875 * 2^9."""
    m, e = torch.frexp(amax)
    s = torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875).to(e.dtype))
    return torch.where(amax > 0, s, 0.0).clamp_min(SCALE_FLOOR)


def _append_plain(s):
    c = s["case"]
    seq, pos = _places(s)
    table = s["table"][pos]
    q = _rotate(s["q"].float(), table, c).to(s["q"].dtype)
    rows = [_rotate(s["k"].float(), table, c), s["v"].float()]
    bs = c["block"]
    ids, starts = s["block_ids"].long(), s["blk_start"].long()
    blk = ids[starts[seq] + pos // bs]
    if c["cache"] == "16":
        _token_major(s["pools"][0], c)[blk, pos % bs] = rows[0].to(s["k"].dtype)
        _token_major(s["pools"][1], c)[blk, pos % bs] = rows[1].to(s["k"].dtype)
        return {"q": q, "pools": s["pools"], "scales": None}
    first = s["ctx_len"].long() - (s["q_start"][1:] - s["q_start"][:-1]).long()   # first new position of each sequence
    held = first % bs                                                         # earlier tokens of the block it falls in
    edge = ids[starts[:-1] + first // bs]
    kept = torch.arange(bs, device=DEV)[None, :] < held[:, None]              # [seq, row of the block]
    _quantise(rows[0], s["pools"][0], s["scales"][0], c, blk, pos % bs, edge, kept)
    _quantise(rows[1], s["pools"][1], s["scales"][1], c, blk, pos % bs, edge, kept)
    return {"q": q, "pools": s["pools"], "scales": s["scales"]}


def _quantise(x, pool, scales, c, blk, row, edge, kept):
    n_blocks, hk = scales.shape
    peak = torch.zeros(n_blocks, hk, device=DEV).scatter_reduce_(0, blk[:, None].expand(-1, hk), x.abs().amax(-1), "amax")
    old = scales[edge]                                                        # [seq, head]
    fresh = _pow2_scale(peak)
    new = torch.where(kept.any(1)[:, None], torch.maximum(fresh[edge], old), fresh[edge])
    fresh[edge] = new
    tokens = _token_major(pool, c)
    was = tokens[edge].float()                                                # [seq, row, head, dim]
    tokens[edge] = torch.where(kept[:, :, None, None], was * (old / new)[:, None, :, None], was).to(E4M3)
    tokens[blk, row] = (x / fresh[blk][:, :, None]).to(E4M3)
    scales[blk] = fresh[blk]


def _attend_plain(s):
    c = s["case"]
    bs, hk, d, g = c["block"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    q_start, ctx, starts = s["q_start"].long(), s["ctx_len"].long(), s["blk_start"].long()
    j = torch.arange(s["max_ctx"], device=DEV)
    there = j[None, :] < ctx[:, None]                                         # [seq, key]
    blk = s["block_ids"].long()[torch.where(there, starts[:-1, None] + j // bs, 0)]
    keys, values = (_token_major(p, c)[blk, j % bs].float() for p in s["pools"])   # [seq, key, kv head, dim]
    if c["cache"] == "8":
        keys *= s["scales"][0][blk][..., None]
        values *= s["scales"][1][blk][..., None]
    i = torch.arange(s["max_q"], device=DEV)
    n_new = q_start[1:] - q_start[:-1]
    q = s["q"][torch.where(i[None, :] < n_new[:, None], q_start[:-1, None] + i, 0)].float()
    q = q.unflatten(2, (hk, g)).permute(0, 2, 3, 1, 4).flatten(2, 3)          # [seq, kv head, (query head, new token), dim]
    scores = (q * d ** -0.5) @ keys.permute(0, 2, 3, 1)
    seen = j[None, None, :] <= (ctx - n_new)[:, None, None] + i[None, :, None]     # [seq, new token, key]
    scores = scores.unflatten(2, (g, -1)).masked_fill_(~(seen & there[:, None])[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = (scores - top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ values.transpose(1, 2)).unflatten(2, (g, -1)) / total
    lse = (top + total.log()).squeeze(-1)
    seq, pos = _places(s)
    at = pos - (ctx - n_new)[seq]
    return {"out": out[seq, :, :, at].flatten(1, 2).to(s["q"].dtype), "lse": lse[seq, :, :, at].flatten(1, 2)}


def run(state):
    if own:
        return _own(state)
    return _append_plain(state) if state["case"]["op"] == "append" else _attend_plain(state)


# ---------------------------------------------------------------------------- cost and the statement in 64 bits

def work(case):
    c, lens = case, lengths(case)
    size = 1 if c["cache"] == "8" else 2
    tokens, row = sum(n for _, n in lens), c["dim"] * c["kv_heads"]
    if c["op"] == "append":
        table = sum(n for _, n in lens) * c["rot"] * 4
        touched = sum(-(-(p + n) // c["block"]) - p // c["block"] for p, n in lens)
        scales = touched * c["kv_heads"] * 2 * 4 if size == 1 else 0
        return {"bytes": tokens * (2 * c["heads"] * c["dim"] * 2 + 2 * row * (2 + size)) + table + scales,
                "flops": 3 * tokens * c["rot"] * (c["heads"] + c["kv_heads"])}
    held = sum(p + n for p, n in lens)
    blocks = sum(-(-(p + n) // c["block"]) for p, n in lens)
    pairs = sum(n * p + n * (n + 1) // 2 for p, n in lens)
    return {"bytes": held * 2 * row * size + blocks * (4 + (c["kv_heads"] * 8 if size == 1 else 0)) + tokens * c["heads"] * (c["dim"] * 4 + 4),
            "flops": 4 * c["heads"] * c["dim"] * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    return _append_exact(case, s) if case["op"] == "append" else _attend_exact(case, s)


def _block(pool, c, b):
    """Block b as [row, head, dim]: a view."""
    return pool[b].transpose(0, 1) if c["hnd"] else pool[b]


def _append_exact(c, s):
    """Codes of an 8-bit pool are given before their rounding, in units of the block's scale."""
    r, bs, d = c["rot"], c["block"], c["dim"]
    one, two = (list(range(r // 2)), list(range(r // 2, r))) if c["style"] == "half" else (list(range(0, r, 2)), list(range(1, r, 2)))

    def turned(x, at):
        y = x.double().clone()
        cos, sin = s["table"][at:at + len(x), :r // 2].double()[:, None], s["table"][at:at + len(x), r // 2:].double()[:, None]
        y[..., one] = x[..., one].double() * cos - x[..., two].double() * sin
        y[..., two] = x[..., two].double() * cos + x[..., one].double() * sin
        return y

    q = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    pools, ids = [p.double() for p in s["pools"]], s["block_ids"].tolist()
    scales = [x.clone() for x in s["scales"]] if c["cache"] == "8" else None
    row = blk = 0
    for p, n in lengths(c):
        q[row:row + n] = turned(s["q"][row:row + n], p)
        new = [turned(s["k"][row:row + n], p), s["v"][row:row + n].double()]
        if c["cache"] == "16":
            pos = torch.arange(p, p + n, device=DEV)
            at = s["block_ids"].long()[blk + pos // bs]
            for pool, x in zip(pools, new):
                if c["hnd"]:
                    pool[at, :, pos % bs] = x
                else:
                    pool[at, pos % bs] = x
        else:
            for b in range(p // bs, (p + n - 1) // bs + 1):
                lo, hi = max(p, b * bs), min(p + n, (b + 1) * bs)
                for pool, scale, x in zip(pools, scales, new):
                    part, rows = x[lo - p:hi - p], _block(pool, c, ids[blk + b])
                    peak = part.abs().amax((0, 2)).clamp_min(SCALE_FLOOR)
                    need = torch.exp2(torch.round(torch.log2(peak / 448)))    # near it: then the smallest that holds the peak
                    need = torch.where(need * 448 < peak, need * 2, need)
                    need = torch.where(need * 224 >= peak, need / 2, need).clamp_min(SCALE_FLOOR)
                    if lo > b * bs:
                        before = scale[ids[blk + b]].double()
                        need = torch.maximum(need, before)
                        rows[:lo - b * bs] *= (before / need)[:, None]
                    rows[lo - b * bs:hi - b * bs] = part / need[:, None]
                    scale[ids[blk + b]] = need.float()
        row, blk = row + n, blk + -(-(p + n) // bs)
    return {"q": q, "pools": pools, "scales": [x.double() for x in scales] if scales else None}


def _attend_exact(c, s):
    hk, g, bs, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["block"], c["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    row = blk = 0
    for p, n in lengths(c):
        nb = -(-(p + n) // bs)
        ids = s["block_ids"][blk:blk + nb].long()
        for h in range(hk):
            kv = []
            for a in range(2):
                x = (s["pools"][a][ids, h] if c["hnd"] else s["pools"][a][ids, :, h]).double()
                if c["cache"] == "8":
                    x = x * s["scales"][a][ids, h].double()[:, None, None]
                kv.append(x.reshape(-1, d)[:p + n])
            step = max(1, (1 << 27) // (p + n))
            for a in range(0, n, step):
                b = min(n, a + step)
                hidden = torch.arange(p + n, device=DEV)[None, :] > torch.arange(p + a, p + b, device=DEV)[:, None]
                for x in range(h * g, (h + 1) * g):
                    w = s["q"][row + a:row + b, x].double() @ kv[0].T / math.sqrt(d)
                    w.masked_fill_(hidden, -math.inf)
                    lse[row + a:row + b, x] = torch.logsumexp(w, -1)
                    out[row + a:row + b, x] = torch.softmax(w, -1) @ kv[1]
        row, blk = row + n, blk + nb
    return {"out": out, "lse": lse}
