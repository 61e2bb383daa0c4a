"""Tables of block ids and counts of a pool, with the operators on pages stated row by row in plain Python, and a window's
attention in 64 bits over an OpCase."""
from __future__ import annotations

import numpy as np
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import F32, HALF, OpCase

MAX_TOKENS = (1 << 31) - 1


def blocks_of(tokens, bs):
    return -(-tokens // bs)


class Book:
    """blk_start, ids, lens and refs as lists; every call is one sequence of plain steps.  status: the codes that came up."""

    def __init__(self, blk_start, ids, lens, bs, n_blk=None):
        self.blk_start, self.ids, self.lens, self.bs = [int(x) for x in blk_start], [int(x) for x in ids], [int(x) for x in lens], bs
        self.n_blk = len(self.ids) if n_blk is None else n_blk
        self.status = set()

    def room(self, s):
        a, b = self.blk_start[s], self.blk_start[s + 1]
        return (a, b - a) if 0 <= a <= b <= self.n_blk else None

    def row(self, s):
        """First entry, room, tokens and held entries; None for a row that is refused."""
        r, n = self.room(s), self.lens[s]
        if r is None or n > MAX_TOKENS or n < 0 or blocks_of(n, self.bs) > r[1]:
            return None
        return r[0], r[1], n, blocks_of(n, self.bs)


def drop(refs, i, status):
    if not 0 <= i < len(refs):
        status.add(T.EFAULT)
    elif refs[i] <= 0:
        status.add(T.EINVAL)
    else:
        refs[i] -= 1


def fork(frm, parent, to, refs, move):
    for s in range(len(to.lens)):
        f, r = int(parent[s]), to.room(s)
        ok = r is not None
        if f != -1:
            p = frm.row(f) if 0 <= f < len(frm.lens) else None
            ok = ok and p is not None and p[3] <= r[1]
        to.lens[s] = 0
        if not ok:
            to.status.add(T.EINVAL)
        elif f != -1:
            to.lens[s] = p[2]
            for k in range(p[3]):
                i = to.ids[r[0] + k] = frm.ids[p[0] + k]
                if 0 <= i < len(refs):
                    refs[i] += 1
                elif i != -1:
                    frm.status.add(T.EFAULT)
    for f in range(len(frm.lens)):
        p = frm.row(f)
        if p is None:
            frm.status.add(T.EINVAL)
        elif move:
            for k in range(p[3]):
                if frm.ids[p[0] + k] != -1:
                    drop(refs, frm.ids[p[0] + k], frm.status)


def extend(t, refs, n_new):
    n_seq = len(t.lens)
    pairs = [(-1, -1)] * n_seq
    rows, writers = [None] * n_seq, {}
    for s in range(n_seq):
        r, add = t.row(s), int(n_new[s])
        if r is None or add < 0 or r[2] + add > MAX_TOKENS or blocks_of(r[2] + add, t.bs) > r[1]:
            t.status.add(T.EINVAL)
            continue
        tail = -1
        if add and r[2] % t.bs:
            tail = t.ids[r[0] + r[2] // t.bs]
            if tail != -1:
                if not 0 <= tail < len(refs) or refs[tail] <= 0:
                    t.status.add(T.EFAULT if not 0 <= tail < len(refs) else T.EINVAL)
                    continue
                writers.setdefault(tail, []).append(s)
        rows[s] = (*r, add, tail)
    need = []
    for s in range(n_seq):
        if rows[s] is None:
            continue
        b0, _, n, held, add, tail = rows[s]
        if tail >= 0 and refs[tail] > 1 and not (s == writers[tail][-1] and len(writers[tail]) >= refs[tail]):
            need.append((s, b0 + held - 1, True))
        need += [(s, b0 + k, False) for k in range(held, blocks_of(n + add, t.bs))]
    free = [i for i, x in enumerate(refs) if x == 0]
    if len(need) > t.n_blk:                                     # rows that lie over each other
        t.status.add(T.EINVAL)
        return pairs
    if len(need) > len(free):
        t.status.add(T.EAGAIN)
        return pairs
    for b, w in writers.items():
        if refs[b] > 1:
            refs[b] = max(1, refs[b] - len(w))
    for (s, at, copies), i in zip(need, free):
        if copies:
            pairs[s] = (t.ids[at], i)
        t.ids[at] = i
        refs[i] = 1
    for s in range(n_seq):
        if rows[s] is not None:
            t.lens[s] += rows[s][4]
    return pairs


def release(t, refs, which):
    for s in range(len(t.lens)):
        if which is not None and not which[s]:
            continue
        r = t.row(s)
        if r is None:
            t.status.add(T.EINVAL)
            continue
        for k in range(r[0], r[0] + r[3]):
            if t.ids[k] != -1:
                drop(refs, t.ids[k], t.status)
                t.ids[k] = -1
        t.lens[s] = 0


def trim(t, refs, window, sinks):
    for s in range(len(t.lens)):
        r = t.row(s)
        if r is None:
            t.status.add(T.EINVAL)
            continue
        for k in range(r[3]):
            first, last = k * t.bs, (k + 1) * t.bs - 1
            # a later row is at position len at least
            if first >= sinks and last <= r[2] - window and t.ids[r[0] + k] != -1:
                drop(refs, t.ids[r[0] + k], t.status)
                t.ids[r[0] + k] = -1


def compact(t, refs, max_pairs):
    n = sum(x != 0 for x in refs)
    source = [i for i in range(len(refs) - 1, n - 1, -1) if refs[i] != 0]
    to = [i for i in range(n) if refs[i] == 0]
    moves = list(zip(source, to))[:max_pairs]
    place = dict(moves)
    for a, b in moves:
        refs[b], refs[a] = refs[a], 0
    for s in range(len(t.lens)):
        r = t.row(s)
        if r is None:
            t.status.add(T.EINVAL)
            continue
        for k in range(r[0], r[0] + r[3]):
            if t.ids[k] < -1 or t.ids[k] >= len(refs):
                t.status.add(T.EFAULT)
            t.ids[k] = place.get(t.ids[k], t.ids[k])
    return moves


class Bound:
    """Tables and counts on the GPU."""

    def __init__(self, ctx, books, refs, device=0):
        self.dev = torch.device("cuda", device)
        self.books = books
        up = lambda a: torch.tensor(a, dtype=torch.int32, device=self.dev)  # noqa: E731
        self.refs = up(refs)
        self.t = []
        for b in books:
            x = [up(b.blk_start), up(b.ids), torch.tensor(np.array(b.lens, np.int64).astype(np.uint32).view(np.int32), device=self.dev), up([0])]
            self.t.append((T.make_tables(*x[:3], status=x[3]), *x))
        self.pages = T.Pages(ctx, self.refs)

    def tables(self, k=0):
        return self.t[k][0]

    def same(self, refs, k=0):
        """Counts, entries (spare ones too), lengths and the status of table k are what the book says."""
        b, (_, _, ids, lens, status) = self.books[k], self.t[k]
        assert self.refs.tolist() == [int(x) for x in refs], "counts"
        assert ids.tolist() == b.ids, "entries"
        assert [x & 0xffffffff for x in lens.tolist()] == [x & 0xffffffff for x in b.lens], "lengths"
        code = int(status)
        assert (code in b.status) if b.status else code == T.OK, (code, b.status)

    def close(self):
        torch.cuda.synchronize()
        self.pages.close()


def random_book(rng, n_seq, bs, n_blocks, most, *, share=0.3, spare=3, trimmed=0.0, gaps=False):
    """A book with consistent counts: rows of random lengths, some of which begin like the row before them."""
    free, rows, lens = list(rng.permutation(n_blocks)), [], []
    for s in range(n_seq):
        n = int(rng.integers(0, most + 1))
        h = blocks_of(n, bs)
        if s and rng.random() < share and rows[-1]:
            # all of the row before, its partly filled block too, or a part of it
            k = len(rows[-1]) if rng.random() < 0.5 else int(rng.integers(0, len(rows[-1]) + 1))
            n = lens[-1] if k == len(rows[-1]) else max(n, k * bs)
            h = blocks_of(n, bs)
            row = rows[-1][:k]
        else:
            row = []
        while len(row) < h and free:
            row.append(int(free.pop()))
        n = min(n, len(row) * bs)
        rows.append(row[:blocks_of(n, bs)])
        lens.append(n)
    start, ids = [0], []
    for row in rows:
        if gaps and rng.random() < 0.3:
            ids += [12345] * 2                                  # a row that nobody uses lies in between
        ids += row + [-7] * int(rng.integers(0, spare + 1))
        start.append(len(ids))
    book = Book(start, ids, lens, bs)
    if trimmed:
        for s, row in enumerate(rows):
            for k in range(len(row) - 1):
                if rng.random() < trimmed:
                    book.ids[start[s] + k] = -1
    refs = [0] * n_blocks
    for s in range(n_seq):
        a, _, _, h = book.row(s)
        for i in book.ids[a:a + h]:
            if i >= 0:
                refs[i] += 1
    return book, refs


class WindowCase(OpCase):
    """An OpCase whose blocks behind the window are gone: their ids are no block's (`gone`), their bytes NaN."""

    def __init__(self, lens, window, sinks, *, gone=-1, **kw):
        super().__init__(lens, **kw)
        self.window, self.sinks, self.gone = window, sinks, gone

    def clear(self):
        for s, (p, n) in enumerate(self.lens):
            total = int(self.ctx_len[s])
            for b in range(-(-total // self.bs)):
                if b * self.bs >= self.sinks and (b + 1) * self.bs <= total - n - self.window + 1:
                    at = self.blk_start[s] + b
                    if self.gone is not None:
                        for half in range(2):
                            self.block(self.raw, half, self.block_ids[at]).view(torch.uint8).fill_(0xFF)
                        self.block_ids[at] = self.gone
        self.pool.copy_(self.raw)
        self.t_ids.copy_(torch.from_numpy(self.block_ids))

    def seen(self, pos):
        """The keys of a row."""
        j = np.arange(pos + 1)
        return j[(j < self.sinks) | (pos - j < self.window)]

    def attend64(self, q, raw, scale, sm):
        """As OpCase.attend64, whose bounds hold for any set of keys."""
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
                if first + i < 0:
                    continue
                at = self.seen(first + i)
                row = int(self.q_start[s]) + i
                for h in range(self.heads):
                    kk, vv, sc = k[at, h // g], v[at, h // g], vs[at, h // g]
                    x = kk @ q[row, h] * sm
                    d = (self.dim * F32 * (np.abs(kk) @ np.abs(q[row, h]))).max() * abs(sm) + 4 * F32 * (np.abs(x).max() + 16)
                    low = 2.0 ** -24 if self.cache == "8" and self.dtype == "fp16" else 0.0
                    d += low * np.abs(q[row, h]).sum() * abs(sm)
                    m = x.max()
                    e = np.exp(x - m)
                    l = e.sum()
                    w = e / l
                    out[row, h] = w @ vv
                    lse[row, h] = m + np.log(l)
                    size = w @ np.abs(vv)
                    f16 = self.dtype == "fp16" or self.cache == "8"
                    floor = 2.0 ** -31 * (w * sc).max() * (np.abs(vv) / sc[:, None]).sum(0) if f16 else 0.0
                    tol[row, h] = half_step * np.abs(out[row, h]) + tiny + low + floor + (half_step + 2 * d + (len(at) + 64) * F32 + 2 ** -20) * size
                    ltol[row, h] = 2 * d + (len(at) + 64) * F32 + 2 ** -20 + 4 * F32 * abs(lse[row, h])
        return out, lse, tol, ltol

    def keys(self, raw, scale, half, s, n):
        """Blocks that are gone read as zeros: no row sees them."""
        out = np.zeros((n, self.hk, self.dim))
        for b in range(-(-n // self.bs)):
            i = int(self.block_ids[self.blk_start[s] + b])
            if not 0 <= i < self.n_blocks:
                continue
            x = self.block(raw, half, i).float().double().numpy()
            if scale is not None:
                x = x * scale[half][i].double().numpy()[None, :, None]
            m = min(self.bs, n - b * self.bs)
            out[b * self.bs:b * self.bs + m] = x[:m]
        return out

    def key_scales(self, scale, half, s, n):
        ids = np.clip(self.block_ids[self.blk_start[s] + np.arange(n) // self.bs], 0, self.n_blocks - 1)
        return scale[half].double().numpy()[ids] if scale is not None else np.ones((n, self.hk))
