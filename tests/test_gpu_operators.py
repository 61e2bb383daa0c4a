"""The operators on the pool together, as a serving program uses them, and where they can go wrong:
append, attend, save, restore into other blocks, attend again; long pools, unusual blocks and groups,
codes and scales at the ends of their ranges, handles and graphs side by side."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import DTYPES, OpCase
from tests.test_gpu_append import append, table_of, verify as append_verify
from tests.test_gpu_attend import attend, fill_new, verify

pytestmark = pytest.mark.gpu


class Served:
    """One layer of a model over a pool with a store: two contexts, the second one for the scales of an 8-bit pool."""

    def __init__(self, cache, hk=4, dim=64, bs=16, n_blocks=64, obj=32, n_slots=8, heads=8):
        self.hk, self.dim, self.bs, self.heads, self.size = hk, dim, bs, heads, 1 if cache == "8" else 2
        self.dev = torch.device("cuda", 0)
        bb = bs * hk * dim * self.size
        self.pool = torch.full((2, n_blocks * bb), 0xFF, dtype=torch.uint8, device=self.dev)
        self.parts = [self._part(T.Geom(1, hk, dim, self.size, bs, obj, 1, T.LAYOUT_LAYER_MAJOR, n_slots), self.pool, bb, n_blocks)]
        self.ctx = self.parts[0][0]
        if cache == "8":
            self.scales = torch.zeros((2, n_blocks, hk), dtype=torch.float32, device=self.dev)
            self.ctx.tutti_scales_register(0, self.scales[0].data_ptr(), self.scales[1].data_ptr(), n_blocks)
            # a block's scales as one token of hk 4-byte elements; an object has a scale row for each of its blocks
            self.parts.append(self._part(T.Geom(1, hk, 1, 4, 1, obj // bs, 1, T.LAYOUT_LAYER_MAJOR, n_slots), self.scales, 4 * hk, n_blocks))
        self.attn = T.Attn(self.ctx)
        a = np.arange(512)[:, None] * 10000.0 ** (-np.arange(dim // 2) * 2 / dim)
        self.table = torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).to(self.dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.dev)

    def _part(self, geom, pool, block_bytes, n_blocks):
        ctx = T.Context(geom, 0)
        store = torch.zeros(int(ctx.layout.dev_bytes), dtype=torch.uint8, device=self.dev)
        ctx.tutti_store_register(0, store.data_ptr(), store.numel())
        ctx.tutti_pool_register(0, pool[0].data_ptr(), pool[1].data_ptr(), block_bytes, n_blocks)
        return ctx, store, T.Ring(ctx, 8, 64, 256, 64)

    def ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device=self.dev)

    def run(self, x, ctx, ids):
        """Append and attend rows x [n, q | k | v] as the last of `ctx` tokens in blocks ids."""
        n, d = len(x), self.dim
        q, k, v = (x[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in
                   ((0, self.heads), (self.heads, self.heads + self.hk), (self.heads + self.hk, self.heads + 2 * self.hk)))
        step = T.make_step(self.ints([0, n]), self.ints([ctx]), self.ints([0, len(ids)]), self.ints(ids), n, n, self.status)
        qr = torch.empty(n, self.heads, d, dtype=x.dtype, device=self.dev)
        out = torch.empty_like(qr)
        self.ctx.tutti_kv_append_layer(0, step, T.make_tokens(k, v, q, qr), T.make_rope(self.table))
        self.attn.tutti_kv_attend_layer(0, step, T.make_attend(qr, out), d ** -0.5)
        assert int(self.status) == T.OK
        return out

    def move(self, op, ids, slots, tokens):
        """Save (WRITE) or restore (READ) the blocks `ids` that hold `tokens` tokens: codes and scales alike."""
        for ctx, _, ring in self.parts:
            per = int(ctx.layout.blocks_per_obj)
            unit = tokens if ctx is self.ctx else len(ids)
            batch = T.make_batch(self.ints([unit]), self.ints([0, len(slots)]), self.ints(slots), self.ints([0, len(ids)]), self.ints(ids))
            assert len(slots) * per >= len(ids)
            _, first, n = ring.tutti_build_sqes(batch, 0, op)
            (ring.tutti_kv_save_layer if op == T.OP_WRITE else ring.tutti_kv_restore_layer)(first, n)
            rc, _, err, _ = ring.tutti_ring_poll_range(first, n, 5_000_000_000)
            assert rc == T.OK and err == T.OK

    def close(self):
        torch.cuda.synchronize()
        self.attn.close()
        for ctx, _, ring in self.parts:
            ring.close()
            ctx.close()


@pytest.mark.parametrize("cache,dtype", [("16", torch.bfloat16), ("8", torch.float16), ("8", torch.bfloat16)])
def test_a_prompt_is_computed_saved_restored_elsewhere_and_continued(cache, dtype):
    s = Served(cache)
    try:
        g = torch.Generator(device=s.dev).manual_seed(1)
        x = torch.randn(160, (s.heads + 2 * s.hk) * s.dim, generator=g, device=s.dev).to(dtype)
        here, there = list(range(3, 30, 2)), list(range(40, 60))
        prompt = s.run(x[:96], 96, here)
        s.move(T.OP_WRITE, here[:6], [5, 1, 6], 96)
        chunk = s.run(x[96:131], 131, here)                     # goes on in the same blocks
        tokens = [s.run(x[i:i + 1], i + 1, here) for i in range(131, 140)]
        s.move(T.OP_READ, there[:6], [5, 1, 6], 96)             # another request with the same prefix
        assert torch.equal(chunk, s.run(x[96:131], 131, there))
        for i, want in zip(range(131, 140), tokens):
            assert torch.equal(want, s.run(x[i:i + 1], i + 1, there))
        # the prompt in two chunks gives what it gives at once, up to the order of sums and, in an 8-bit
        # pool, nothing at all (a chunk ends with a block, so no scale depends on the cut)
        again = torch.cat([s.run(x[:48], 48, there), s.run(x[48:96], 96, there)])
        d = (again.double() - prompt.double()).abs().max() / prompt.double().abs().max()
        assert d <= (2.0 ** -7 if dtype is torch.bfloat16 else 2.0 ** -10)
    finally:
        s.close()


@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("block,dim,hnd,interleaved", [(8, 128, False, False), (128, 128, True, False), (24, 64, False, False),
                                                       (256, 64, False, True), (32, 128, True, True)])
def test_attend_other_block_sizes(cache, block, dim, hnd, interleaved):
    c = OpCase([(300, 70), (5, 1), (255, 40)], heads=8, kv_heads=2, dim=dim, block=block, cache=cache, hnd=hnd, interleaved=interleaved, seed=40 + block)
    try:
        fill_new(c)
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache,dtype", [("16", "bf16"), ("8", "bf16"), ("8", "fp16")])
@pytest.mark.parametrize("heads,kv_heads,new", [(9, 1, 1), (12, 1, 1), (16, 1, 1), (17, 1, 1), (64, 1, 1), (4, 1, 2), (4, 1, 4), (4, 1, 5), (2, 2, 16), (300, 1, 1)])
def test_attend_groups_and_rows_around_the_tiles(cache, dtype, heads, kv_heads, new):
    """8, 16 and 128 rows are where the kernels' tiles end."""
    c = OpCase([(200, new), (3, new)], heads=heads, kv_heads=kv_heads, dim=128, cache=cache, dtype=dtype, seed=heads + new)
    try:
        fill_new(c)
        verify(c, attend(c))
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend8_codes_and_scales_at_the_ends(dtype, new, dim):
    """Subnormal codes, zero and largest codes; scales from where f16 ends to where bf16 goes on."""
    c = OpCase([(100, new), (60, new)], heads=4, kv_heads=2, dim=dim, cache="8", dtype=dtype, seed=50)
    try:
        fill_new(c)
        for s, e in ((0, [-30, -26, -20, -9, 0, 3, 5, 7, 7]), (1, [-9] * 9)):
            for half in range(2):
                for b in range(-(-int(c.ctx_len[s]) // c.bs)):
                    i = int(c.block_ids[c.blk_start[s] + b])
                    x = c.block(c.raw, half, i)
                    codes = torch.randint(0, 127, x.shape, generator=torch.Generator().manual_seed(b + 2 * half), dtype=torch.uint8)
                    sign = torch.randint(0, 2, x.shape, generator=torch.Generator().manual_seed(b), dtype=torch.uint8) * 128
                    small = b % 3 == 2                          # codes 0..7 are zero and the subnormal ones
                    n = min(c.bs, int(c.ctx_len[s]) - b * c.bs)
                    x[:n] = (codes % (8 if small else 127) + sign).view(torch.float8_e4m3fn)[:n]
                    c.scale[half][i] = 2.0 ** e[b % 9]
        c.pool.copy_(c.raw)
        for a, b in zip(c.scale, c.scale_dev):
            b.copy_(a)
        # scores of a few at most, so that no single key decides
        for scale in (1e-5, 1e-3):
            verify(c, attend(c, scale), scale)
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [1, 40])
def test_attend8_nan_codes_stay_in_their_sequence(dtype, new):
    c = OpCase([(100, new), (60, new)], heads=4, kv_heads=2, dim=128, cache="8", dtype=dtype, seed=51)
    try:
        fill_new(c)
        i = int(c.block_ids[1])                                 # keys 16..31 of sequence 0
        for code in (0x7F, 0xFF):
            for half in range(2):
                raw = c.raw.clone()
                c.block(raw, half, i).view(torch.uint8)[3, 1, 77] = code
                c.pool.copy_(raw)
                out = attend(c)
                verify(c, out, skip=(0,))
                got = torch.isnan(out[:new].float())
                assert not got[:, :2].any()                     # query heads 0 and 1 read KV head 0
                assert got[:, 2:].all() if half == 0 else got[:, 2:, 77].all() and int(got[:, 2:].sum()) == 2 * new
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 40])
def test_operators_behind_four_gigabytes(new):
    """Block offsets that pass 32 bits: a 6 GB pool of which the last blocks are used."""
    c = OpCase([(50, new), (20, new)], heads=8, kv_heads=8, dim=128, block=16, seed=52)
    try:
        fill_new(c)
        shift = (3 << 30) // c.stride                            # of each of the two planes
        n = c.n_blocks + shift
        big = torch.empty(2, n * c.stride, dtype=torch.uint8, device=c.dev)
        big[:, -c.n_blocks * c.stride:] = c.pool.view(2, -1)
        c.ctx.tutti_pool_register(1, big[0].data_ptr(), big[1].data_ptr(), c.stride, n)
        c.t_ids += shift
        verify(c, attend(c))
        assert int(c.status) == T.OK
        tail = big[:, -c.n_blocks * c.stride:].clone()
        q = torch.empty_like(c.q)
        c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k, c.v, c.q, q))
        small = c.pool.clone()
        c.register(0)
        c.t_ids -= shift
        c.ctx.tutti_kv_append_layer(0, c.step, T.make_tokens(c.k, c.v, c.q, q))
        assert not torch.equal(small, c.pool)
        assert torch.equal(big[:, -c.n_blocks * c.stride:].reshape(-1), c.pool) and not torch.equal(tail.reshape(-1), c.pool)
    finally:
        c.close()


def test_two_graphs_with_a_handle_each_run_side_by_side():
    a, b = (OpCase([(5000, n), (1000, n)], heads=8, kv_heads=2, seed=53 + n) for n in (1, 30))
    try:
        graphs, outs = [], []
        for c in (a, b):
            fill_new(c)
            c.lse = None
            out = torch.zeros((c.n_tok, c.heads, c.dim), dtype=DTYPES[c.dtype], device=c.dev)
            io = T.make_attend(c.q, out)
            g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=s):
                for _ in range(8):
                    c.attn.tutti_kv_attend_layer(1, c.step, io, c.dim ** -0.5, s)
            graphs.append((g, s))
            outs.append(out)
        torch.cuda.synchronize()
        for _ in range(3):
            for g, s in graphs:
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for c, out in zip((a, b), outs):
            out[int(c.q_start[-1]):] = 7.5
            verify(c, out)
    finally:
        a.close()
        b.close()


def test_handle_is_reusable_over_all_kinds_of_calls():
    """The workspace is left as the next call needs it, whichever kernel that is."""
    cases = [OpCase([(2000, n), (900, n)], heads=h, kv_heads=2, dim=d, cache=k, seed=60 + n, dtype="fp16")
             for n, h, d, k in ((1, 8, 128, "16"), (1, 24, 128, "16"), (50, 8, 128, "16"), (1, 8, 64, "8"), (60, 4, 128, "8"))]
    try:
        for c in cases:
            fill_new(c)
        for _ in range(2):
            for c in cases:
                # a handle belongs to a context, so a context takes the others' pools in turn only where the geometry agrees
                verify(c, attend(c))
                verify(c, attend(c))
        same = [c for c in cases if c.cache == "16"]
        for c in same[1:]:
            c.own_ctx, c.ctx = c.ctx, same[0].ctx
            c.register(1)
            verify(c, attend(c, attn=same[0].attn))
            c.ctx = c.own_ctx
        same[0].register(1)
        verify(same[0], attend(same[0]))
    finally:
        for c in cases:
            c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_steps_with_nothing_to_do(cache):
    c = OpCase([(20, 0), (0, 0)], cache=cache, seed=70, spare_rows=5)
    try:
        before = c.pool.clone()
        out = attend(c)
        q = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k, c.v, c.q, q))
        empty = T.make_step(c.t_q_start[:1], c.t_ctx[:0], c.t_blk_start[:1], c.t_ids[:0], 0, 0)
        c.ctx.tutti_kv_append_layer(1, empty, T.make_tokens(c.k, c.v))
        c.attn.tutti_kv_attend_layer(1, empty, T.make_attend(c.q, out), 1.0)
        torch.cuda.synchronize()
        assert (out == 7.5).all() and (c.lse == 7.5).all() and (q == 7.5).all() and torch.equal(before, c.pool)
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 64])
def test_many_sequences_some_of_them_empty(new):
    rng = np.random.default_rng(71)
    lens = [(int(p), new if rng.random() < 0.6 else 0) for p in rng.integers(0, 80, 700)]
    c = OpCase(lens, heads=2, kv_heads=1, dim=64, seed=72)
    try:
        fill_new(c)
        verify(c, attend(c))
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_decode_and_prompt_rows_in_one_step(cache):
    c = OpCase([(600, 1), (0, 300), (1000, 1), (130, 7), (90, 1), (700, 128)], heads=8, kv_heads=2, cache=cache, seed=73)
    try:
        fill_new(c)
        verify(c, attend(c))
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_a_step_in_two_calls_over_slices_of_its_tables(cache):
    """Decoding and prompt sequences of one step apart: the second call's first row is not row 0."""
    c = OpCase([(600, 1), (1000, 1), (90, 1), (0, 300), (130, 7), (700, 128)], heads=8, kv_heads=2, cache=cache, seed=74)
    try:
        steps = [T.make_step(c.t_q_start[a:b + 1], c.t_ctx[a:b], c.t_blk_start[a:b + 1], c.t_ids, c.n_tok, new, c.status)
                 for a, b, new in ((3, 6, 300), (0, 3, 1))]
        qr = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        c.table = table_of(1001, c.dim)
        for st in steps:
            c.ctx.tutti_kv_append_layer(1, st, T.make_tokens(c.k, c.v, c.q, qr), T.make_rope(c.table))
            assert int(c.status) == T.OK
            if st is steps[0]:
                assert (qr[:3] == 7.5).all()
        append_verify(c, qr)
        fill_new(c)
        out = torch.full_like(qr, 7.5)
        c.lse = torch.full((c.n_tok, c.heads), 7.5, dtype=torch.float32, device=c.dev)
        for st in steps:
            c.attn.tutti_kv_attend_layer(1, st, T.make_attend(c.q, out, c.lse), c.dim ** -0.5)
            assert int(c.status) == T.OK
            if st is steps[0]:
                assert (out[:3] == 7.5).all() and (c.lse[:3] == 7.5).all()
        verify(c, out)
    finally:
        c.close()


def random_case(seed):
    rng = np.random.default_rng(seed)
    kv_heads = int(rng.choice([1, 2, 3, 4]))
    new = int(rng.choice([1, 1, 3, 20, 150]))
    lens = [(int(rng.integers(0, rng.choice([5, 60, 700]))), int(rng.integers(0, new + 1)) if new > 1 else 1) for _ in range(rng.integers(1, 7))]
    block = int(rng.choice([1, 2, 7, 8, 16, 16, 33, 64, 100, 128]))
    cache = str(rng.choice(["16", "8"]))
    return OpCase(lens, heads=kv_heads * int(rng.choice([1, 2, 4, 5, 8, 13])), kv_heads=kv_heads, dim=int(rng.choice([64, 128])), block=block,
                  dtype=str(rng.choice(["bf16", "fp16"])), cache=cache, hnd=bool(rng.random() < 0.4), interleaved=bool(rng.random() < 0.3),
                  pad=16 * int(rng.integers(0, 5)), packed=bool(rng.random() < 0.5), spare_rows=int(rng.integers(0, 4)), seed=seed)


@pytest.mark.parametrize("seed", range(24))
def test_random_steps(seed):
    c = random_case(1000 + seed)
    try:
        style = "half" if seed % 2 else "pairs"
        append_verify(c, append(c, style, c.dim // (1 + seed % 3 // 2)), style)
        fill_new(c)
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()
