"""The operators on the pool together, as a generating program runs them: steps under a window whose blocks are freed and taken
again, beams that share their blocks and go on in others, blocks moved together in between, graphs that are replayed."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HEADS, HK, DIM, BS, LAYERS = 8, 2, 64, 16, 2


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Model:
    """A pool of LAYERS layers whose keys, values and queries are drawn from a sequence's history, so that a sequence gives
    the same rows wherever its blocks lie."""

    def __init__(self, cache, n_blocks, n_seq, cap, dtype=torch.bfloat16):
        size = 1 if cache == "8" else 2
        self.cache, self.dtype, self.n_seq, self.cap, self.n_blocks = cache, dtype, n_seq, cap, n_blocks
        self.ctx = T.Context(T.Geom(LAYERS, HK, DIM, size, BS, BS, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
        self.pool = torch.full((LAYERS, 2, n_blocks, BS * HK * DIM * size), 0xFF, dtype=torch.uint8, device=DEV)
        self.scales = torch.zeros(LAYERS, 2, n_blocks, HK, device=DEV)
        for l in range(LAYERS):
            self.ctx.tutti_pool_register(l, self.pool[l, 0].data_ptr(), self.pool[l, 1].data_ptr(), self.pool.shape[-1], n_blocks)
            if cache == "8":
                self.ctx.tutti_scales_register(l, self.scales[l, 0].data_ptr(), self.scales[l, 1].data_ptr(), n_blocks)
        self.attn = T.Attn(self.ctx)
        self.refs = torch.zeros(n_blocks, dtype=torch.int32, device=DEV)
        self.pages = T.Pages(self.ctx, self.refs)
        self.status = ints([0])
        self.tables = [self._table() for _ in range(2)]
        self.pairs = torch.zeros(n_seq, 2, dtype=torch.int32, device=DEV)
        self.now = 0
        at = torch.arange(512)[:, None] * 10000.0 ** (-torch.arange(DIM // 2) * 2 / DIM)
        self.rope = T.make_rope(torch.cat([at.cos(), at.sin()], 1).float().to(DEV))

    def _table(self):
        x = ints([s * self.cap for s in range(self.n_seq + 1)]), torch.full((self.n_seq * self.cap,), -1, dtype=torch.int32, device=DEV), ints([0] * self.n_seq)
        return T.make_tables(*x, status=self.status), *x

    def rows(self, keys, n):
        """Rows [sequences * n, q | k | v] from an integer that says what each sequence has come from."""
        out = []
        for k in keys:
            g = torch.Generator().manual_seed(int(k) % (1 << 40))
            out.append(torch.randn(n, (HEADS + 2 * HK) * DIM, generator=g))
        return torch.cat(out).to(self.dtype).to(DEV)

    def step(self, x, n, window=None, stream=None):
        """Append and attend n tokens of every sequence, for which the tables have room."""
        _, start, ids, lens = self.tables[self.now]
        q, k, v = (x[:, a * DIM:b * DIM].unflatten(1, (b - a, DIM)) for a, b in ((0, HEADS), (HEADS, HEADS + HK), (HEADS + HK, HEADS + 2 * HK)))
        step = T.make_step(ints([s * n for s in range(self.n_seq + 1)]) if stream is None else self.q_start, lens, start, ids, len(x), n, self.status)
        outs = []
        for l in range(LAYERS):
            qr, out = torch.empty(len(x), HEADS, DIM, dtype=self.dtype, device=DEV), torch.empty(len(x), HEADS, DIM, dtype=self.dtype, device=DEV)
            self.ctx.tutti_kv_append_layer(l, step, T.make_tokens(k, v, q, qr), self.rope, stream)
            io = T.make_attend(qr, out)
            if window is None:
                self.attn.tutti_kv_attend_layer(l, step, io, DIM ** -0.5, stream)
            else:
                self.attn.tutti_kv_attend_window_layer(l, step, io, DIM ** -0.5, window, stream)
            outs.append(out)
        return outs

    def extend(self, n, stream=None):
        n_new = ints([n] * self.n_seq) if stream is None else self.n_new
        self.pages.tutti_pages_extend(self.tables[self.now][0], n_new, self.pairs, stream)
        self.ctx.tutti_kv_copy_blocks(0, LAYERS, self.pairs, status=self.status, stream=stream)

    def fork(self, parent, stream=None):
        self.pages.tutti_pages_fork(self.tables[self.now][0], ints(parent), self.tables[1 - self.now][0], T.FORK_MOVE, stream)
        self.now = 1 - self.now

    def counted(self):
        """The counts are what the tables say."""
        _, _, ids, lens = self.tables[self.now]
        held = torch.arange(self.cap, device=DEV)[None] < ((lens + BS - 1) // BS)[:, None]
        ids = ids.view(self.n_seq, self.cap)[held]
        return torch.equal(torch.bincount(ids[ids >= 0].long(), minlength=self.n_blocks).int(), self.refs)

    def close(self):
        torch.cuda.synchronize()
        self.pages.close()
        self.attn.close()
        self.ctx.close()


@pytest.mark.parametrize("cache,dtype", [("16", torch.bfloat16), ("8", torch.bfloat16), ("8", torch.float16)])
def test_steps_under_a_window_with_blocks_freed_and_taken_again(cache, dtype):
    """A prompt and many tokens in a pool that holds little more than the windows, against a pool where nothing is freed: the same bits."""
    w, n_seq, prompt, tokens = T.make_window(40, 5), 3, 90, 150
    whole, small = Model(cache, 60, n_seq, 20, dtype), Model(cache, 30, n_seq, 20, dtype)
    try:
        for m in (whole, small):
            m.extend(prompt)
        x = small.rows(range(n_seq), prompt)
        for a, b in zip(whole.step(x, prompt, w), small.step(x, prompt, w)):
            assert torch.equal(a, b)
        for i in range(tokens):
            small.pages.tutti_pages_trim(small.tables[0][0], w)
            for m in (whole, small):
                m.extend(1)
            x = small.rows([1000 * i + s for s in range(n_seq)], 1)
            for a, b in zip(whole.step(x, 1, w), small.step(x, 1, w)):
                assert torch.equal(a, b), i
            if i % 40 == 17:
                # what has been freed holds another's bytes by the time that it is looked for
                free = (small.refs == 0).nonzero().flatten()
                small.pool[:, :, free] = 0xFF
        assert int(small.status) == int(whole.status) == T.OK and small.counted() and whole.counted()
        assert int((small.refs > 0).sum()) <= n_seq * 5
    finally:
        whole.close()
        small.close()


@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("compact", [False, True])
def test_beams_share_blocks_and_go_on_as_if_each_had_its_own(cache, compact):
    """Beams of two requests that are chosen again and again, against sequences that were computed from the start with blocks of
    their own: the same bits."""
    rng = np.random.default_rng(1)
    beams, n_seq, prompt, tokens = 4, 8, 37, 40
    m = Model(cache, 120, n_seq, 8)
    lone = Model(cache, 80, n_seq, 8)
    try:
        # one row of each request has the prompt, its beams fork from it
        m.extend(0)
        m.pages.tutti_pages_extend(m.tables[0][0], ints([prompt if s % beams == 0 else 0 for s in range(n_seq)]), m.pairs)
        x = m.rows([0, 1], prompt)
        history = [[("prompt", s // beams)] for s in range(n_seq)]
        _, start, ids, lens = m.tables[0]
        q, k, v = (x[:, a * DIM:b * DIM].unflatten(1, (b - a, DIM)) for a, b in ((0, HEADS), (HEADS, HEADS + HK), (HEADS + HK, HEADS + 2 * HK)))
        step = T.make_step(ints([0] + [prompt * (1 + s // beams) for s in range(n_seq)]), lens, start, ids, 2 * prompt, prompt, m.status)
        for l in range(LAYERS):
            m.ctx.tutti_kv_append_layer(l, step, T.make_tokens(k, v), m.rope)
        m.fork([s // beams * beams for s in range(n_seq)])
        assert m.counted() and int(m.refs.max()) == beams
        outs, pairs, moved = [], torch.zeros(60, 2, dtype=torch.int32, device=DEV), ints([0])
        for i in range(tokens):
            m.extend(1)
            for s in range(n_seq):
                history[s].append(7 + 1000 * i + s)
            outs = m.step(m.rows([h[-1] for h in history], 1), 1)
            parent = [int(s // beams * beams + rng.integers(0, beams)) for s in range(n_seq)]
            if i < tokens - 1:
                m.fork(parent)
                history = [list(history[p]) for p in parent]
                assert m.counted(), i
                if compact and i % 7 == 3:
                    m.pages.tutti_pages_compact(m.tables[m.now][0], pairs, moved)
                    m.ctx.tutti_kv_copy_blocks(0, LAYERS, pairs, moved)
                    used = int((m.refs > 0).sum())
                    assert m.counted() and not m.refs[used:].any()
                    m.pool[:, :, used:] = 0xFF
        assert int(m.status) == T.OK
        # the same histories alone
        lone.extend(prompt)
        lone.step(lone.rows([s // beams for s in range(n_seq)], prompt), prompt)
        for i in range(1, tokens + 1):
            lone.extend(1)
            want = lone.step(lone.rows([h[i] for h in history], 1), 1)
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
        m.pages.tutti_pages_release(m.tables[m.now][0])
        assert not m.refs.any()
    finally:
        m.close()
        lone.close()


def test_captured_steps_are_replayed():
    """A step under a window in a graph: trim, extend, copy, append, attend, again and again, against the same calls one by one."""
    w, n_seq, tokens = T.make_window(24, 3), 4, 60
    eager, graph = Model("16", 40, n_seq, 12), Model("16", 40, n_seq, 12)
    try:
        for m in (eager, graph):
            m.extend(30)
            m.step(m.rows(range(n_seq), 30), 30, w)
        st = torch.cuda.Stream()
        graph.q_start, graph.n_new = ints(list(range(n_seq + 1))), ints([1] * n_seq)
        x = torch.zeros(n_seq, (HEADS + 2 * HK) * DIM, dtype=graph.dtype, device=DEV)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            graph.pages.tutti_pages_trim(graph.tables[0][0], w, torch.cuda.current_stream())
            graph.extend(1, torch.cuda.current_stream())
            outs = graph.step(x, 1, w, torch.cuda.current_stream())
        for i in range(tokens):
            rows = eager.rows([50 * i + s for s in range(n_seq)], 1)
            x.copy_(rows)
            g.replay()
            eager.pages.tutti_pages_trim(eager.tables[0][0], w)
            eager.extend(1)
            for a, b in zip(outs, eager.step(rows, 1, w)):
                assert torch.equal(a, b), i
            assert torch.equal(eager.refs, graph.refs) and torch.equal(eager.tables[0][2], graph.tables[0][2])
        assert int(graph.status) == T.OK and graph.counted()
    finally:
        eager.close()
        graph.close()


def test_handles_on_streams_of_their_own():
    """Two pools worked on at once, on side streams, give what each gives alone."""
    def run(m, stream, seed):
        rng = np.random.default_rng(seed)
        st = stream
        got = []
        with torch.cuda.stream(st):
            m.q_start, m.n_new = ints(list(range(m.n_seq + 1))), ints([1] * m.n_seq)
            n30 = ints([30] * m.n_seq)
            m.pages.tutti_pages_extend(m.tables[0][0], n30, m.pairs, st)
            for i in range(25):
                parent = ints([int(x) for x in rng.integers(0, m.n_seq, m.n_seq)])
                m.pages.tutti_pages_fork(m.tables[m.now][0], parent, m.tables[1 - m.now][0], T.FORK_MOVE, st)
                m.now = 1 - m.now
                m.extend(1, st)
                got.append(m.step(m.rows([i], m.n_seq), 1, T.make_window(20, 2), st)[-1])
        return got

    alone = []
    for seed in (1, 2):
        m = Model("16", 60, 5, 8)
        try:
            m.pool.zero_()
            alone.append([x.clone() for x in run(m, torch.cuda.Stream(), seed)])
            torch.cuda.synchronize()
        finally:
            m.close()
    both = [Model("16", 60, 5, 8) for _ in range(2)]
    try:
        for m in both:
            m.pool.zero_()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = [run(m, st, seed) for m, st, seed in zip(both, streams, (1, 2))]
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    finally:
        for m in both:
            m.close()


def test_rows_of_two_tables_share_counts():
    """A prompt's table and a batch's over the same counts: forked without giving the prompt up, then both freed."""
    m = Model("16", 40, 3, 6)
    try:
        m.extend(70)
        prompts, batch = m.tables
        m.pages.tutti_pages_fork(prompts[0], ints([2, 2, 0]), batch[0], T.FORK_KEEP)
        assert sorted(set(m.refs.tolist())) == [0, 1, 2, 3]
        m.now = 1
        m.extend(3)                                             # every row writes to a block that its prompt holds, too
        assert all(b >= 0 for _, b in m.pairs.tolist())
        m.pages.tutti_pages_release(batch[0])
        m.now = 0
        assert m.counted()
        m.pages.tutti_pages_release(prompts[0], torch.tensor([True, False, True], device=DEV))
        assert m.counted() and int(m.refs.sum()) == 5
        assert int(m.status) == T.OK
    finally:
        m.close()


def test_a_save_behind_a_copy_sees_what_was_copied():
    """The kernels of a save may start while the kernel in front of them runs, if that one lets them: it does not."""
    n, bs, hk, dim = 3000, 16, 8, 128
    bb = bs * hk * dim * 2
    ctx = T.Context(T.Geom(1, hk, dim, 2, bs, bs, 1, T.LAYOUT_LAYER_MAJOR, n // 2), 0)
    pool, store = torch.empty(2, n, bb, dtype=torch.uint8, device=DEV), torch.empty(int(ctx.layout.dev_bytes), dtype=torch.uint8, device=DEV)
    ring = T.Ring(ctx, 16, 2048, n, n)
    try:
        ctx.tutti_pool_register(0, pool[0].data_ptr(), pool[1].data_ptr(), bb, n)
        ctx.tutti_store_register(0, store.data_ptr(), store.numel())
        half = n // 2
        to = list(range(half, n))
        batch = T.make_batch(ints([half * bs]), ints([0, half]), ints(list(range(half))), ints([0, half]), ints(to))
        pairs = ints([[i, half + i] for i in range(half)])
        for i in range(5):
            pool.fill_(0)
            store.fill_(0)
            pool[:, :half] = torch.arange(half, device=DEV).remainder(200).add(1 + i).to(torch.uint8)[None, :, None]
            _, first, k = ring.tutti_build_sqes(batch, 0, T.OP_WRITE)
            torch.cuda.synchronize()
            ctx.tutti_kv_copy_blocks(0, 1, pairs)
            ring.tutti_kv_save_layer(first, k)
            rc, _, err, _ = ring.tutti_ring_poll_range(first, k, 5_000_000_000)
            assert rc == T.OK and err == T.OK
            assert torch.equal(store.view(half, 2, bb), pool[:, :half].transpose(0, 1))
    finally:
        torch.cuda.synchronize()
        ring.close()
        ctx.close()
