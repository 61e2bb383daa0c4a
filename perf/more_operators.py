"""More operator cases of the paged KV pool: attention with a sliding window and a few first tokens that stay visible, and
the pages of the pool themselves: copied in all layers, handed from beam to beam, freed behind a window, taken for new
tokens, freed and moved together.

`run` computes a case in elementary torch operations (`own` false) or through the library's calls (`own` true); `exact`
states the attention in 64 bits, one sequence and head at a time.  What the pages' operators give is whole numbers and
copies of bytes."""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn


def attend_(name, cache, dtype, heads, kv_heads, dim, block, seqs, prefix, new, window, sinks, *, hnd=False, mix=1):
    """prefix and new: (lowest, highest) tokens of a sequence that are in the pool already and that the step brings."""
    c = {"op": "attend", "cache": cache, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block, "hnd": hnd,
         "seqs": seqs, "prefix_lo": prefix[0], "prefix_hi": prefix[1], "new_lo": new[0], "new_hi": new[1], "window": window, "sinks": sinks, "mix": mix}
    return {"name": name, **c} if name else c


def pages_(name, op, cache, kv_heads, dim, block, layers, mix=1, **more):
    """more: by operator, see listed()."""
    c = {"op": op, "cache": cache, "kv_heads": kv_heads, "dim": dim, "block": block, "hnd": False, "layers": layers, "mix": mix, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a few short chats of a model with a window: latency
        attend_("window decode short", "16", "fp16", 32, 8, 128, 16, 4, (99, 999), (1, 1), 256, 4),
        # one decode step of a 64-request batch, whose pages behind the window are gone
        attend_("window decode", "16", "bf16", 32, 8, 128, 16, 64, (511, 32767), (1, 1), 4096, 4),
        # ragged chunks over restored prefixes of an 8-bit pool with head-major blocks
        attend_("window chunk 8-bit", "8", "fp16", 32, 8, 128, 16, 4, (2000, 9000), (300, 700), 1024, 4, hnd=True),
        # a long prompt, of which every row sees 4096 keys: the largest
        attend_("window chunk long", "16", "bf16", 32, 8, 128, 16, 1, (24576, 24576), (8192, 8192), 4096, 16),
        # blocks that a few requests write to while others share them, with their scales: latency
        pages_("copy few", "copy", "8", 8, 128, 16, 32, blocks=256, pairs=6),
        # 32768 tokens of a request duplicated in 8 layers
        pages_("copy many", "copy", "16", 8, 128, 16, 8, blocks=5120, pairs=2048),
        # 16 requests of 4 beams go on from the beams that a step chose, by a token
        pages_("beams", "beams", "16", 8, 128, 16, 8, requests=16, beams=4, prompt_lo=511, prompt_hi=4095, apart=37),
        # the same on 1-token pages, where the tables are long and no page is ever shared by writers
        pages_("beams pages", "beams", "16", 8, 128, 1, 1, requests=16, beams=8, prompt_lo=511, prompt_hi=16383, apart=100),
        # a decode step's pages in a 64-request batch: the ones behind the window are freed, new ones taken
        pages_("slide", "slide", "16", 8, 128, 16, 0, seqs=64, len_lo=511, len_hi=32767, window=4096, sinks=4, new=1, blocks=40960),
        # the same for the largest batch, whose restored prefixes are all still there, with 4 tokens a step
        pages_("slide restored", "slide", "16", 8, 128, 16, 0, seqs=1024, len_lo=99, len_hi=16383, window=1024, sinks=4, new=4, blocks=1048576),
        # a small 8-bit pool after some requests have ended
        pages_("compact small", "compact", "8", 8, 128, 16, 4, seqs=16, len_lo=99, len_hi=999, share=64, gone=0.4),
        # 64 requests, a third of which have ended, in 4 layers
        pages_("compact", "compact", "16", 8, 128, 16, 4, seqs=64, len_lo=255, len_hi=2047, share=128, gone=0.33),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "copy", "beams", "slide", "compact"])
    cache, mix = rng.choice(["16", "8"]), rng.randrange(1 << 20)
    kv_heads, dim, block = rng.choice([8, 8, 4, 2, 1]), rng.choice([64, 128, 128]), rng.choice([1, 8, 16, 16, 32, 64])
    if op == "attend":
        dtype, hnd = rng.choice(["bf16", "fp16"]), rng.random() < 0.3
        heads, kv_heads = rng.choice([(32, 8), (64, 8), (28, 4), (8, 8), (40, 8), (8, 1), (16, 16), (6, 2)])
        if cache == "8" and block == 1:
            block = 16
        window, sinks = _log(rng, 1, 8192), rng.choice([0, 1, 4, 4, 16, 100])
        if rng.random() < 0.5:
            seqs = _log(rng, 1, 64)
            prefix = _log(rng, 1, 65535)
            return attend_("", cache, dtype, heads, kv_heads, dim, block, seqs, (prefix // 4, prefix), (1, 1), min(window, 262144 // seqs), sinks, hnd=hnd, mix=mix)
        new, seqs = _log(rng, 2, 8192), _log(rng, 1, 8)
        window = min(window, 4096)
        while seqs > 1 and heads * seqs * new * (new + window) > 32 * 8192 * 12288:
            seqs //= 2
        while heads * seqs * new * (new + window) > 32 * 8192 * 12288:
            new //= 2
        prefix = _log(rng, 1, 32768)
        return attend_("", cache, dtype, heads, kv_heads, dim, block, seqs, (prefix // 2, prefix), (max(1, new // 2), new), window, sinks, hnd=hnd, mix=mix)
    size = 1 if cache == "8" else 2
    if op == "copy":
        layers, pairs = _log(rng, 1, 32), _log(rng, 1, 2048)
        most = 2 * 2048 * 8 * 16 * 8 * 128                      # bytes of the largest listed one, a plane
        pairs = max(1, min(pairs, most // (layers * block * kv_heads * dim * size)))
        return pages_("", op, cache, kv_heads, dim, block, layers, mix, blocks=2 * pairs + rng.randrange(1, 2 + pairs), pairs=pairs)
    if op == "beams":
        requests, beams = _log(rng, 1, 32), rng.choice([1, 2, 3, 4, 5, 8, 16])
        prompt = _log(rng, 1, 16383 if block < 16 else 4095)
        layers = max(1, min(rng.choice([1, 2, 4, 8]), (1 << 31) // (2 * requests * (prompt + 200 * beams) * kv_heads * dim * size)))
        return pages_("", op, cache, kv_heads, dim, block, layers, mix, requests=requests, beams=beams, prompt_lo=prompt // 2, prompt_hi=prompt, apart=_log(rng, 1, 200))
    if op == "slide":
        seqs, length = _log(rng, 1, 1024), _log(rng, 1, 16383)
        spare = rng.choice([2, 3, 8])
        most = seqs * (-(-(length + 8) // block) + 1)
        if most > 800000:
            seqs = max(1, 800000 * seqs // most)
            most = seqs * (-(-(length + 8) // block) + 1)
        return pages_("", op, "16", kv_heads, dim, block, 0, mix, seqs=seqs, len_lo=length // 4, len_hi=length, window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 16, 100]),
                      new=rng.choice([1, 1, 1, 2, 5, 8]), blocks=most + seqs * spare)
    seqs, length = _log(rng, 1, 64), _log(rng, 1, 2047)
    layers = rng.choice([1, 2, 4])
    return pages_("", op, cache, kv_heads, dim, block, layers, mix, seqs=seqs, len_lo=length // 2, len_hi=length, share=_log(rng, 1, 256), gone=rng.choice([0.0, 0.2, 0.5, 0.8]))


# ---------------------------------------------------------------------------- inputs

def lengths(c):
    """Tokens in the pool before the step and new ones, by sequence: part of the case, not of the seed."""
    rng = random.Random(c["mix"])
    if c["op"] == "attend":
        return [(rng.randint(c["prefix_lo"], c["prefix_hi"]), rng.randint(c["new_lo"], c["new_hi"])) for _ in range(c["seqs"])]
    if c["op"] == "beams":
        return [(rng.randint(c["prompt_lo"], c["prompt_hi"]), rng.randint(1, c["apart"])) for _ in range(c["requests"])]
    return [(rng.randint(c["len_lo"], c["len_hi"]), c.get("new", 0)) for _ in range(c["seqs"])]


def _csr(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _ints(v):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v), dtype=np.int32)).to(DEV)


def prepare(case, seed):
    return {"attend": _prepare_attend, "copy": _prepare_copy, "beams": _prepare_beams, "slide": _prepare_slide,
            "compact": _prepare_compact}[case["op"]](case, np.random.default_rng(seed), torch.Generator(device=DEV).manual_seed(seed))


def _pools(s, c, n_blocks, planes, g, dtype=None):
    """`planes` key and value planes of n_blocks blocks, a tensor [plane, block, ...], and the scales of an 8-bit pool."""
    inner = (c["kv_heads"], c["block"], c["dim"]) if c["hnd"] else (c["block"], c["kv_heads"], c["dim"])
    shape = (planes, n_blocks, *inner)
    s["n_blocks"] = n_blocks
    if c["cache"] == "16":
        s["pool"] = torch.empty(shape, dtype=dtype or torch.bfloat16, device=DEV).normal_(generator=g)
        return
    s["pool"] = torch.empty(shape, dtype=E4M3, device=DEV)
    flat, step = s["pool"].view(-1), 1 << 26
    for a in range(0, flat.numel(), step):
        flat[a:a + step] = (torch.randn(min(step, flat.numel() - a), generator=g, device=DEV) * 64).clamp_(-448, 448).to(E4M3)
    s["scales"] = torch.exp2(torch.randint(-9, -5, (planes, n_blocks, c["kv_heads"]), generator=g, device=DEV).float())


def _prepare_attend(c, rng, g):
    lens, bs = lengths(c), c["block"]
    dt, hq, d = TYPES[c["dtype"]], c["heads"], c["dim"]
    rows = []                                                   # by sequence, which of its blocks any row of the step sees
    for p, n in lens:
        first = np.arange(-(-(p + n) // bs)) * bs               # key of a block
        rows.append((first < c["sinks"]) | (first + bs > p - c["window"] + 1))
    need = int(sum(r.sum() for r in rows))
    n_blocks = need + need // 4 + 1
    ids = np.full(sum(len(r) for r in rows), -1, dtype=np.int32)
    ids[np.concatenate(rows)] = rng.permutation(n_blocks)[:need]
    n_tok = sum(n for _, n in lens)
    s = {"case": c, "q_start": _ints(_csr([n for _, n in lens])), "ctx_len": _ints([p + n for p, n in lens]), "blk_start": _ints(_csr([len(r) for r in rows])),
         "block_ids": _ints(ids), "n_tok": n_tok, "max_q": max(n for _, n in lens),
         "max_seen": max(p + n - max(0, p - c["window"] + 1) for p, n in lens) + c["sinks"]}
    spread = torch.exp(torch.randn(hq * d, generator=g, device=DEV) * 0.4)
    s["q"] = (torch.randn(n_tok, hq * d, generator=g, device=DEV) * spread).to(dt).unflatten(1, (hq, d))
    _pools(s, c, n_blocks, 2, g, dt)
    return s


def _prepare_copy(c, rng, g):
    s = {"case": c}
    _pools(s, c, c["blocks"], 2 * c["layers"], g)
    s["pairs"] = _ints(rng.permutation(c["blocks"])[:2 * c["pairs"]].reshape(2, -1).T)     # [pair, (from, to)]
    return s


def _tables(c, rows, cap, lens, n_blocks):
    """A state with rows of ids (numpy) as a table of `cap` entries a row, the rows' lengths and the blocks' counts: in one
    buffer, and in another that each pass begins from."""
    ids = np.full((len(rows), cap), -1, dtype=np.int32)
    for r, row in zip(ids, rows):
        r[:len(row)] = row
    n, m = n_blocks, ids.size
    at = [-(-n // 4) * 4, -(-n // 4) * 4 + -(-m // 4) * 4]      # 16-byte aligned
    flat = np.zeros(at[1] + len(lens), dtype=np.int32)
    flat[:n], flat[at[0]:at[0] + m], flat[at[1]:] = np.bincount(ids[ids >= 0], minlength=n), ids.reshape(-1), lens
    s = {"case": c, "n_blocks": n, "blk_start": _ints(np.arange(len(rows) + 1) * cap), "start": torch.from_numpy(flat).to(DEV)}
    s["now"] = s["start"].clone()
    for x, name in (("start", "0"), ("now", "")):
        s["refs" + name], s["ids" + name], s["len" + name] = s[x][:n], s[x][at[0]:at[0] + m], s[x][at[1]:]
    return s


def _prepare_beams(c, rng, g):
    bs, b, lens = c["block"], c["beams"], lengths(c)
    shared = [p // bs for p, _ in lens]                         # full blocks of the prompt
    held = [-(-(p + a) // bs) for p, a in lens]
    need = sum(f + (h - f) * b for f, h in zip(shared, held))
    n_blocks = need + need // 4 + 2 * b * len(lens) + 1         # room for every beam's next block
    free, rows = rng.permutation(n_blocks).astype(np.int32), []
    for f, h in zip(shared, held):
        prompt, free = free[:f], free[f:]
        for _ in range(b):
            rows.append(np.concatenate([prompt, free[:h - f]]))
            free = free[h - f:]
    s = _tables(c, rows, max(held) + 1, np.repeat([p + a for p, a in lens], b), n_blocks)
    parent = rng.integers(0, b, (len(lens), b))                 # of a request's beams
    s["parent"] = _ints((parent + np.arange(len(lens))[:, None] * b).reshape(-1))
    n_seq = len(lens) * b
    s["to_ids"], s["to_len"] = torch.full((s["ids"].numel(),), -1, dtype=torch.int32, device=DEV), torch.zeros(n_seq, dtype=torch.int32, device=DEV)
    s["n_new"], s["pairs"] = torch.ones(n_seq, dtype=torch.int32, device=DEV), torch.zeros(n_seq, 2, dtype=torch.int32, device=DEV)
    _pools(s, c, n_blocks, 2 * c["layers"], g)
    return s


def _prepare_slide(c, rng, g):
    bs, lens, n_blocks = c["block"], [p for p, _ in lengths(c)], c["blocks"]
    held = [-(-n // bs) for n in lens]
    free, rows = rng.permutation(n_blocks).astype(np.int32), []
    for i, (n, h) in enumerate(zip(lens, held)):
        row, free = free[:h].copy(), free[h:]
        if i and i % 4 == 0:                                    # a prompt that another request has, too
            k = min(held[i - 1], h) // 2
            row[:k] = rows[-1][:k]
        rows.append(row)
    if c["new"] == 1:                                           # earlier steps have freed all but the last few
        for row, n in zip(rows, lens):
            first = np.arange(len(row)) * bs
            row[(first >= c["sinks"]) & (first + bs <= n - c["window"] + 1 - rng.integers(0, 3 * bs))] = -1
    s = _tables(c, rows, max(held) + c["new"] + 1, lens, n_blocks)
    s["n_new"], s["pairs"] = torch.full((len(lens),), c["new"], dtype=torch.int32, device=DEV), torch.zeros(len(lens), 2, dtype=torch.int32, device=DEV)
    return s


def _prepare_compact(c, rng, g):
    bs, lens = c["block"], [p for p, _ in lengths(c)]
    held = [-(-n // bs) for n in lens]
    n_blocks = int(sum(held) / 0.8) + 8
    free, rows = rng.permutation(n_blocks).astype(np.int32), []
    for i, h in enumerate(held):
        row, free = free[:h].copy(), free[h:]
        if i % 3 == 2:                                          # a prompt that another request has, too
            k = min(c["share"] // bs, held[i - 1], h)
            row[:k] = rows[-1][:k]
        rows.append(row)
    s = _tables(c, rows, max(held) + 1, lens, n_blocks)
    s["which"] = torch.from_numpy(rng.random(len(lens)) < c["gone"]).to(DEV)
    s["pairs"], s["n_pairs"] = torch.zeros(n_blocks // 2, 2, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    _pools(s, c, n_blocks, 2 * c["layers"], g)
    return s


# ---------------------------------------------------------------------------- the library's calls

_contexts = {}
LAYERS = 128


def _bind(s):
    """What a program sets up once for its pool and its tables: the registration of the layers (those of a geometry's one
    context are taken in turn), the step, the counts."""
    from paper_2605_03375_b200 import tutti as T
    c = s["case"]
    size = 1 if c["cache"] == "8" else 2
    key = (c["kv_heads"], c["dim"], size, c["block"], c["hnd"])
    if key not in _contexts:
        ctx = T.Context(T.Geom(LAYERS, c["kv_heads"], c["dim"], size, c["block"], c["block"], 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
        ctx.tutti_set_option(T.OPT_POOL_LAYOUT, T.POOL_HND if c["hnd"] else T.POOL_NHD)
        _contexts[key] = [ctx, None, 0, 0]                      # its attention handle, the next layer, how often the layers have begun anew
    entry = _contexts[key]
    ctx, n = entry[0], c.get("layers", 1)
    if entry[2] + n > LAYERS:
        entry[2:] = 0, entry[3] + 1
    first, entry[2] = entry[2], entry[2] + n
    block_bytes = c["block"] * c["kv_heads"] * c["dim"] * size
    for l in range(n):
        k, v = s["pool"][2 * l], s["pool"][2 * l + 1]
        ctx.tutti_pool_register(first + l, k.data_ptr(), v.data_ptr(), block_bytes, s["n_blocks"])
        if c["cache"] == "8":
            ctx.tutti_scales_register(first + l, s["scales"][2 * l].data_ptr(), s["scales"][2 * l + 1].data_ptr(), s["n_blocks"])
    b = {"T": T, "ctx": ctx, "first": first, "turn": (entry, entry[3])}
    if c["op"] == "attend":
        entry[1] = entry[1] or T.Attn(ctx)
        b["attn"] = entry[1]
        b["step"] = T.make_step(s["q_start"], s["ctx_len"], s["blk_start"], s["block_ids"], s["n_tok"], s["max_q"])
    elif c["op"] != "copy":
        b["pages"] = T.Pages(ctx, s["refs"])
        b["tables"] = T.make_tables(s["blk_start"], s["ids"], s["len"])
        if c["op"] == "beams":
            b["to"] = T.make_tables(s["blk_start"], s["to_ids"], s["to_len"])
    if c["op"] in ("attend", "slide"):
        b["window"] = T.make_window(c["window"], c["sinks"])
    s["bound"] = b
    return b


def _own(s):
    c = s["case"]
    b = s.get("bound")
    if b is None or (c.get("layers", 1) and b["turn"][0][3] != b["turn"][1]):       # its layers may be another state's by now
        b = _bind(s)
    T, ctx, first = b["T"], b["ctx"], b["first"]
    stream = torch._C._cuda_getCurrentRawStream(0)
    if c["op"] == "attend":
        out = torch.empty((s["n_tok"], c["heads"], c["dim"]), dtype=s["q"].dtype, device=DEV)
        lse = torch.empty((s["n_tok"], c["heads"]), dtype=torch.float32, device=DEV)
        b["attn"].tutti_kv_attend_window_layer(first, b["step"], T.make_attend(s["q"], out, lse), c["dim"] ** -0.5, b["window"], stream)
        return {"out": out, "lse": lse}
    if c["op"] == "copy":
        ctx.tutti_kv_copy_blocks(first, c["layers"], s["pairs"], stream=stream)
        return _moved(s)
    pages = b["pages"]
    if c["op"] == "beams":
        s["refs"].copy_(s["refs0"])                             # the rows are left as they are, the counts change
        pages.tutti_pages_fork(b["tables"], s["parent"], b["to"], T.FORK_MOVE, stream)
        pages.tutti_pages_extend(b["to"], s["n_new"], s["pairs"], stream)
        ctx.tutti_kv_copy_blocks(first, c["layers"], s["pairs"], stream=stream)
        return {"ids": s["to_ids"], "len": s["to_len"], "refs": s["refs"], "pairs": s["pairs"], **_moved(s)}
    s["now"].copy_(s["start"])                                  # a pass begins with the same tables
    if c["op"] == "slide":
        pages.tutti_pages_trim(b["tables"], b["window"], stream)
        pages.tutti_pages_extend(b["tables"], s["n_new"], s["pairs"], stream)
        return {"ids": s["ids"], "len": s["len"], "refs": s["refs"], "pairs": s["pairs"]}
    pages.tutti_pages_release(b["tables"], s["which"], stream)
    pages.tutti_pages_compact(b["tables"], s["pairs"], s["n_pairs"], stream)
    ctx.tutti_kv_copy_blocks(first, c["layers"], s["pairs"], s["n_pairs"], stream=stream)
    return {"ids": s["ids"], "len": s["len"], "refs": s["refs"], "pairs": s["pairs"], "n_pairs": s["n_pairs"], **_moved(s)}


def _moved(s):
    """The pool and its scales as the whole numbers that their bytes are."""
    pool = s["pool"].view(torch.uint8 if s["case"]["cache"] == "8" else torch.int16)
    return {"pool": pool, "scales": s["scales"].view(torch.int32) if "scales" in s else None}


# ---------------------------------------------------------------------------- plain forms

def _token_major(pool, c):
    return pool.transpose(1, 2) if c["hnd"] else pool


def _attend_plain(s):
    c = s["case"]
    bs, hk, g, window, sinks = c["block"], c["kv_heads"], c["heads"] // c["kv_heads"], c["window"], c["sinks"]
    q_start, ctx, starts = s["q_start"].long(), s["ctx_len"].long(), s["blk_start"].long()
    n_new = q_start[1:] - q_start[:-1]
    lo = (ctx - n_new - window + 1).clamp_min(0)                # the first key in any row's window
    kept = lo.clamp_max(sinks)                                  # first tokens in front of it
    i = torch.arange(s["max_seen"], device=DEV)[None, :]
    j = torch.where(i < kept[:, None], i, lo[:, None] + i - kept[:, None])          # [seq, key]: its position
    there = j < ctx[:, None]
    blk = s["block_ids"].long()[torch.where(there, starts[:-1, None] + j // bs, starts[:-1, None] + (ctx[:, None] - 1) // bs)]
    row = torch.where(there, j % bs, 0)
    keys, values = (_token_major(p, c)[blk, row].float() for p in s["pool"])        # [seq, key, kv head, dim]
    if c["cache"] == "8":
        keys *= s["scales"][0][blk][..., None]
        values *= s["scales"][1][blk][..., None]
    r = torch.arange(s["max_q"], device=DEV)
    q = s["q"][torch.where(r[None, :] < n_new[:, None], q_start[:-1, None] + r, 0)].float()
    q = q.unflatten(2, (hk, g)).permute(0, 2, 3, 1, 4).flatten(2, 3)                # [seq, kv head, (query head, new token), dim]
    scores = (q * c["dim"] ** -0.5) @ keys.permute(0, 2, 3, 1)
    pos = ((ctx - n_new)[:, None] + r)[:, :, None]                                  # [seq, new token, 1]
    seen = (j[:, None] <= pos) & ((j[:, None] < sinks) | (j[:, None] > pos - window)) & there[:, None]
    # rows behind a sequence's last one see its last key: they are left out below
    seen |= (r[None, :, None] >= n_new[:, None, None]) & (j[:, None] == ctx[:, None, None] - 1)
    scores = scores.unflatten(2, (g, -1)).masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ values.transpose(1, 2)).unflatten(2, (g, -1)) / total
    lse = (top + total.log()).squeeze(-1)
    t = torch.arange(s["n_tok"], device=DEV)
    seq = torch.bucketize(t, q_start[1:], right=True)
    at = t - q_start[seq]
    return {"out": out[seq, :, :, at].flatten(1, 2).to(s["q"].dtype), "lse": lse[seq, :, :, at].flatten(1, 2)}


def _copy_plain(s, pairs):
    pairs = pairs.long()
    pairs = pairs[pairs[:, 0] >= 0]
    pool = s["pool"].view(torch.uint8) if s["case"]["cache"] == "8" else s["pool"]
    pool[:, pairs[:, 1]] = pool[:, pairs[:, 0]]
    if "scales" in s:
        s["scales"][:, pairs[:, 1]] = s["scales"][:, pairs[:, 0]]
    return _moved(s)


def _counted(ids, n_blocks):
    """How often each block is in a table's held entries."""
    return torch.bincount(ids[ids >= 0].long(), minlength=n_blocks)[:n_blocks].to(torch.int32)


def _held(ids, length, bs):
    """[row, entry]: which entries belong to the row's tokens."""
    return torch.arange(ids.shape[1], device=DEV)[None, :] < ((length + bs - 1) // bs)[:, None]


def _extend_plain(ids, length, refs, n_new, bs):
    """New blocks, the lowest free ones first, in the order of the rows: where a row's next token goes into a block that
    others share, and for the tokens behind it.  Of rows that share the block they write to, the last keeps it if nobody else has it."""
    n_seq, cap = ids.shape
    row = torch.arange(n_seq, device=DEV)
    after = length + n_new
    partial = (n_new > 0) & (length % bs != 0)
    at = (length // bs).long().clamp_max(cap - 1)
    tail = torch.where(partial, ids[row, at], -1).long()                            # the block that is written to and has tokens
    spot = tail.clamp_min(0)
    writers = torch.zeros_like(refs).index_add_(0, spot, partial.to(refs.dtype))
    last = torch.full_like(refs, -1, dtype=torch.int64).scatter_reduce_(0, spot, torch.where(partial, row, -1), "amax")
    share = partial & (refs[spot] > 1)
    copied = share & ~((writers[spot] >= refs[spot]) & (last[spot] == row))
    more = (after + bs - 1) // bs - (length + bs - 1) // bs
    need = copied + more
    end = need.cumsum(0)
    free = (refs == 0).nonzero().squeeze(1)[:int(end[-1])]
    refs = refs.index_add(0, spot, -copied.to(refs.dtype))
    refs[free] = 1
    ids = ids.clone()
    begin = end - need
    ids[row[copied], at[copied]] = free[begin[copied]].to(torch.int32)
    pairs = torch.where(copied[:, None], torch.stack([tail, free[begin.clamp_max(len(free) - 1)] if len(free) else tail], 1), -1).to(torch.int32)
    k = torch.arange(int(more.sum()), device=DEV)                                   # the blocks behind
    owner = torch.bucketize(k, more.cumsum(0), right=True)
    nth = k - (more.cumsum(0) - more)[owner]
    ids[owner, ((length + bs - 1) // bs)[owner] + nth] = free[begin[owner] + copied[owner] + nth].to(torch.int32)
    return ids, after.to(torch.int32), refs, pairs


def _beams_plain(s):
    bs = s["case"]["block"]
    old, length, refs, parent = s["ids0"].view(s["parent"].numel(), -1), s["len0"], s["refs0"], s["parent"].long()
    new, new_len = old[parent], length[parent]
    held = _held(new, new_len, bs)
    new = torch.where(held, new, -1)
    refs = refs + _counted(new, s["n_blocks"]) - _counted(torch.where(_held(old, length, bs), old, -1), s["n_blocks"])
    ids, after, refs, pairs = _extend_plain(new, new_len, refs, s["n_new"], bs)
    return {"ids": ids.view(-1), "len": after, "refs": refs, "pairs": pairs, **_copy_plain(s, pairs)}


def _slide_plain(s):
    c, bs = s["case"], s["case"]["block"]
    ids, length = s["ids0"].view(s["n_new"].numel(), -1), s["len0"]
    first = torch.arange(ids.shape[1], device=DEV)[None, :] * bs
    gone = _held(ids, length, bs) & (first >= c["sinks"]) & (first + bs - 1 <= (length - c["window"])[:, None]) & (ids >= 0)
    refs = s["refs0"] - _counted(ids[gone], s["n_blocks"])
    ids, after, refs, pairs = _extend_plain(torch.where(gone, -1, ids), length, refs, s["n_new"], bs)
    return {"ids": ids.view(-1), "len": after, "refs": refs, "pairs": pairs}


def _compact_plain(s):
    bs, n = s["case"]["block"], s["n_blocks"]
    ids, length, which = s["ids0"].view(s["which"].numel(), -1), s["len0"], s["which"]
    gone = _held(ids, length, bs) & which[:, None]
    refs = s["refs0"] - _counted(ids[gone], n)
    ids, length = torch.where(gone, -1, ids), torch.where(which, 0, length)
    live = refs > 0
    low = torch.arange(n, device=DEV) < live.sum()
    source, to = (live & ~low).nonzero().squeeze(1).flip(0), (~live & low).nonzero().squeeze(1)
    place = torch.arange(n, device=DEV)
    place[source] = to
    held = _held(ids, length, bs) & (ids >= 0)
    ids = torch.where(held, place[ids.clamp_min(0).long()].to(torch.int32), ids)
    refs = refs.clone()
    refs[to] = refs[source]
    refs[source] = 0
    pairs = torch.full_like(s["pairs"], -1)
    pairs[:len(to), 0], pairs[:len(to), 1] = source.to(torch.int32), to.to(torch.int32)
    n_pairs = (live & ~low).sum().to(torch.int32)[None]
    return {"ids": ids.view(-1), "len": length, "refs": refs, "pairs": pairs, "n_pairs": n_pairs, **_copy_plain(s, pairs)}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "copy":
        return _copy_plain(state, state["pairs"])
    return {"attend": _attend_plain, "beams": _beams_plain, "slide": _slide_plain, "compact": _compact_plain}[op](state)


# ---------------------------------------------------------------------------- cost and the statement in 64 bits

def work(case):
    c, lens = case, lengths(case) if case["op"] != "copy" else []
    size = 1 if c["cache"] == "8" else 2
    row = c["kv_heads"] * c["dim"] * size
    block = 2 * (c["block"] * row + (4 * c["kv_heads"] if size == 1 else 0))        # keys and values of a block, and their scales
    if c["op"] == "attend":
        w, sinks = c["window"], c["sinks"]
        lo = [max(0, p - w + 1) for p, _ in lens]
        seen = sum(p + n - a + min(sinks, a) for (p, n), a in zip(lens, lo))        # keys that any row sees
        pairs = 0
        for p, n in lens:
            at = np.arange(p, p + n, dtype=np.int64)
            a = np.maximum(0, at - w + 1)
            pairs += int((at + 1 - a + np.minimum(sinks, a)).sum())
        tokens = sum(n for _, n in lens)
        return {"bytes": seen * 2 * row + seen // c["block"] * (4 + (8 * c["kv_heads"] if size == 1 else 0)) + tokens * c["heads"] * (4 * c["dim"] + 4),
                "flops": 4 * c["heads"] * c["dim"] * pairs}
    if c["op"] == "copy":
        return {"bytes": c["pairs"] * (8 + 2 * c["layers"] * block), "flops": 0}
    if c["op"] == "beams":
        b, ids, copies = c["beams"], 0, 0.0
        for p, a in lens:
            ids += b * -(-(p + a) // c["block"])
            if (p + a) % c["block"]:
                copies += b - b * (1 - (1 - 1 / b) ** b)        # beams less the beams that are chosen, on average
        return {"bytes": 8 * ids + copies * 2 * c["layers"] * block, "flops": 0}
    held = [-(-p // c["block"]) for p, _ in lens]
    if c["op"] == "slide":                                      # entries that have just left the window, counts, new entries
        gone = sum(max(0, min(h, (p - c["window"] + 1) // c["block"]) - -(-c["sinks"] // c["block"])) if c["new"] > 1 else 1 for (p, _), h in zip(lens, held))
        return {"bytes": 16 * gone + 32 * len(lens), "flops": 0}
    n_blocks = int(sum(held) / 0.8) + 8
    live = sum(held) * (1 - c["gone"])
    return {"bytes": 8 * n_blocks + 8 * sum(held) + live * (1 - live / n_blocks) * 2 * c["layers"] * block, "flops": 0}


def exact(case, seed):
    return _attend_exact(case, prepare(case, seed)) if case["op"] == "attend" else None


def _attend_exact(c, s):
    hk, g, bs, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["block"], c["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    row = blk = 0
    for p, n in lengths(c):
        nb = -(-(p + n) // bs)
        ids = s["block_ids"][blk:blk + nb].long().clamp_min(0)  # blocks that are gone are masked below
        step = 1024
        for h in range(hk):
            for a in range(0, n, step):
                b = min(n, a + step)
                lo = max(0, p + a - c["window"] + 1)
                key = torch.cat([torch.arange(min(c["sinks"], lo)), torch.arange(lo, p + b)]).to(DEV)
                kv = []
                for x in range(2):
                    t = (s["pool"][x][ids[key // bs], h, key % bs] if c["hnd"] else s["pool"][x][ids[key // bs], key % bs, h]).double()
                    if c["cache"] == "8":
                        t = t * s["scales"][x][ids[key // bs], h].double()[:, None]
                    kv.append(t)
                at = torch.arange(p + a, p + b, device=DEV)[:, None]
                far = at - key[None, :]
                hidden = (far < 0) | ((far >= c["window"]) & (key[None, :] >= c["sinks"]))
                for x in range(h * g, (h + 1) * g):
                    w = s["q"][row + a:row + b, x].double() @ kv[0].T / math.sqrt(d)
                    w.masked_fill_(hidden, -math.inf)
                    lse[row + a:row + b, x] = torch.logsumexp(w, -1)
                    out[row + a:row + b, x] = torch.softmax(w, -1) @ kv[1]
        row, blk = row + n, blk + nb
    return {"out": out, "lse": lse}
