"""A paged pool and one step of tokens for the operators on the pool, with a plain statement of
append and attend in 64 bits (numpy loops over sequences, blocks and heads)."""
from __future__ import annotations

import numpy as np
import torch

from paper_2605_03375_b200 import tutti as T

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
#: half a step of a type relative to the value, and half its smallest step
HALF = {"bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25), "e4m3": (2.0 ** -4, 2.0 ** -10)}
F32 = 2.0 ** -24


def rotate64(x, pos, table, style):
    """x [rows, heads, dim] float64, rotated by positions; also the sum of magnitudes behind every element."""
    r = table.shape[1]
    c, s = table[pos, None, : r // 2].astype(np.float64), table[pos, None, r // 2:].astype(np.float64)
    one = np.arange(r // 2) if style == "half" else np.arange(0, r, 2)
    two = one + (r // 2 if style == "half" else 1)
    y, mag = x.copy(), np.abs(x)
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    mag[..., one] = mag[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    return y, mag


def pow2_scale(amax):
    """Smallest power of two s with amax / s <= 448, at least 2^-100."""
    if amax == 0:
        return 2.0 ** -100
    m, e = np.frexp(amax)
    return max(2.0 ** (int(e) - 9 + (m > 0.875)), 2.0 ** -100)


class OpCase:
    """lens: (tokens in the pool before the step, new tokens) of every sequence."""

    def __init__(self, lens, *, heads=8, kv_heads=2, dim=128, block=16, dtype="bf16", cache="16", hnd=False, pad=0,
                 interleaved=False, seed=0, spare_rows=3, packed=True, spread=0.3, spare_ids=1, share=None):
        self.lens, self.heads, self.hk, self.dim, self.bs = lens, heads, kv_heads, dim, block
        self.dtype, self.cache, self.hnd, self.dev = dtype, cache, hnd, torch.device("cuda", 0)
        rng = np.random.default_rng(seed)
        self.rng = rng
        dt = DTYPES[dtype]
        n_seq = len(lens)
        news = [n for _, n in lens]
        self.ctx_len = np.array([p + n for p, n in lens], dtype=np.int32)
        self.q_start = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        rows = [-(-int(c) // block) + spare_ids for c in self.ctx_len]
        self.blk_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n_blocks = int(sum(rows) * 1.3) + 2
        self.block_ids = rng.permutation(self.n_blocks)[: sum(rows)].astype(np.int32)
        if share:                                   # leading blocks of sequence 0 in every other sequence's row
            for s in range(1, n_seq):
                self.block_ids[self.blk_start[s]:self.blk_start[s] + share] = self.block_ids[:share]
        self.n_tok = int(self.q_start[-1]) + spare_rows
        self.max_new = max(news + [1])
        # pool: every byte 0xff (NaN in all the types) but the rows that sequences hold already
        size = 1 if cache == "8" else 2
        self.size = size
        bb = block * kv_heads * dim * size
        self.stride = (2 if interleaved else 1) * bb + pad
        self.k_off, self.v_off = 0, bb if interleaved else self.n_blocks * self.stride
        raw = torch.full(((1 if interleaved else 2) * self.n_blocks * self.stride,), 0xFF, dtype=torch.uint8)
        self.raw = raw
        self.scale = None
        if cache == "8":
            self.scale = [torch.from_numpy(np.exp2(rng.integers(-8, -5, (self.n_blocks, kv_heads))).astype(np.float32)) for _ in range(2)]
        for s, (p, n) in enumerate(lens):
            for b in range(-(-p // block)):
                m = min(block, p - b * block)
                for half in range(2):
                    v = rng.standard_normal((m, kv_heads, dim))
                    t = torch.from_numpy(v * 60).clamp(-448, 448).to(torch.float8_e4m3fn) if size == 1 else torch.from_numpy(v).to(dt)
                    self.block(raw, half, self.block_ids[self.blk_start[s] + b])[:m] = t
        # projections, side by side in one packed row
        w = (heads + 2 * kv_heads) * dim
        x = torch.from_numpy(rng.standard_normal((self.n_tok, w)) * np.exp(rng.standard_normal(w) * spread)).to(dt)
        self.host_q, self.host_k, self.host_v = (x[:, a * dim:b * dim].reshape(self.n_tok, b - a, dim) for a, b in
                                                 ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads)))
        if packed:
            x = x.to(self.dev)
            self.q, self.k, self.v = (x[:, a * dim:b * dim].unflatten(1, (b - a, dim)) for a, b in
                                      ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads)))
        else:
            self.q, self.k, self.v = (y.contiguous().to(self.dev) for y in (self.host_q, self.host_k, self.host_v))
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(self.dev)  # noqa: E731
        self.t_q_start, self.t_ctx, self.t_blk_start, self.t_ids = up(self.q_start), up(self.ctx_len), up(self.blk_start), up(self.block_ids)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.dev)
        self.pool = raw.to(self.dev)
        self.scale_dev = [s.to(self.dev) for s in self.scale] if self.scale else None
        self.ctx = T.Context(T.Geom(2, kv_heads, dim, size, block, block, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
        if hnd:
            self.ctx.tutti_set_option(T.OPT_POOL_LAYOUT, T.POOL_HND)
        self.register(1)
        self.attn = T.Attn(self.ctx)
        self.step = self.make_step()

    def register(self, layer):
        self.ctx.tutti_pool_register(layer, self.pool.data_ptr() + self.k_off, self.pool.data_ptr() + self.v_off, self.stride, self.n_blocks)
        if self.scale:
            self.ctx.tutti_scales_register(layer, self.scale_dev[0].data_ptr(), self.scale_dev[1].data_ptr(), self.n_blocks)

    def make_step(self):
        return T.make_step(self.t_q_start, self.t_ctx, self.t_blk_start, self.t_ids, self.n_tok, self.max_new, self.status)

    def close(self):
        torch.cuda.synchronize()
        self.attn.close()
        self.ctx.close()

    def block(self, raw, half, b):
        """Block b of the key (0) or value (1) plane in `raw` as a [token, head, dim] view."""
        o = (self.v_off if half else self.k_off) + int(b) * self.stride
        t = raw[o:o + self.bs * self.hk * self.dim * self.size]
        t = t.view(torch.float8_e4m3fn if self.size == 1 else DTYPES[self.dtype])
        return t.view(self.hk, self.bs, self.dim).transpose(0, 1) if self.hnd else t.view(self.bs, self.hk, self.dim)

    def keys(self, raw, scale, half, s, n):
        """The first n keys or values of sequence s in float64, [n, head, dim]."""
        out = np.zeros((n, self.hk, self.dim))
        for b in range(-(-n // self.bs)):
            i = int(self.block_ids[self.blk_start[s] + b])
            x = self.block(raw, half, i).float().double().numpy()
            if scale is not None:
                x = x * scale[half][i].double().numpy()[None, :, None]
            m = min(self.bs, n - b * self.bs)
            out[b * self.bs:b * self.bs + m] = x[:m]
        return out

    def key_scales(self, scale, half, s, n):
        """The scales behind keys(), [n, head]."""
        ids = self.block_ids[self.blk_start[s] + np.arange(n) // self.bs]
        return scale[half].double().numpy()[ids] if scale is not None else np.ones((n, self.hk))

    def attend64(self, q, raw, scale, sm):
        """(out, lse, bound of |out error| for a 16-bit kernel, bound of |lse error|) for rows [0, q_start[-1])."""
        half_step, tiny = HALF[self.dtype]
        g = self.heads // self.hk
        n_rows = int(self.q_start[-1])
        out, lse = np.zeros((n_rows, self.heads, self.dim)), np.full((n_rows, self.heads), -np.inf)
        tol, ltol = np.zeros_like(out), np.zeros_like(lse)
        q = q.float().double().cpu().numpy()
        for s, (p, n) in enumerate(self.lens):
            total = int(self.ctx_len[s])
            first = total - n
            k, v = (self.keys(raw, scale, h, s, total) for h in range(2))
            vs = self.key_scales(scale, 1, s, total)
            for i in range(n):
                seen = first + i + 1
                if seen <= 0:
                    continue
                row = int(self.q_start[s]) + i
                for h in range(self.heads):
                    kk, vv = k[:seen, h // g], v[:seen, h // g]
                    x = kk @ q[row, h] * sm
                    # 32-bit products and sums of a score; its exponential's argument and result
                    d = (self.dim * F32 * (np.abs(kk) @ np.abs(q[row, h]))).max() * abs(sm) + 4 * F32 * (np.abs(x).max() + 16)
                    # fp16 over an 8-bit pool: keys and values may be rounded to f16 at half their size,
                    # which is off by 2^-24 at most where that is below the normal range
                    low = 2.0 ** -24 if self.cache == "8" and self.dtype == "fp16" else 0.0
                    d += low * np.abs(q[row, h]).sum() * abs(sm)
                    m = x.max()
                    e = np.exp(x - m)
                    l = e.sum()
                    w = e / l
                    out[row, h] = w @ vv
                    lse[row, h] = m + np.log(l)
                    size = w @ np.abs(vv)
                    # Products of probability and value scale that are rounded to f16 are also off by half
                    # its smallest step, 2^-25, in units that make the row's largest such product 2^6 at
                    # least (2^14 where the rows of a step are few): 2^-31 of that product a key, times its code.
                    f16 = self.dtype == "fp16" or self.cache == "8"
                    floor = 2.0 ** -31 * (w * vs[:seen, h // g]).max() * (np.abs(vv) / vs[:seen, h // g, None]).sum(0) if f16 else 0.0
                    # the result rounded once, the probabilities rounded to 16 bits, the scores off by
                    # d, and 32-bit sums over the keys
                    tol[row, h] = half_step * np.abs(out[row, h]) + tiny + low + floor + (half_step + 2 * d + (seen + 64) * F32 + 2 ** -20) * size
                    ltol[row, h] = 2 * d + (seen + 64) * F32 + 2 ** -20 + 4 * F32 * abs(lse[row, h])
        return out, lse, tol, ltol


def check(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, bound {tol[bad][0]}"
