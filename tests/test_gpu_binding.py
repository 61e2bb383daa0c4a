"""The binding of the operators on the pool with tensors on the GPU and in pinned host memory."""
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import DTYPES, OpCase
from tests.test_gpu_append import append, table_of, verify as append_verify
from tests.test_gpu_attend import attend, fill_new, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 30])
def test_tables_and_status_in_pinned_host_memory(new):
    c = OpCase([(40, new), (200, new)], seed=90)
    try:
        tables = [t.cpu().pin_memory() for t in (c.t_q_start, c.t_ctx, c.t_blk_start, c.t_ids)]
        status = torch.zeros(1, dtype=torch.int32).pin_memory()
        c.step = T.make_step(*tables, c.n_tok, c.max_new, status)
        append_verify(c, append(c))
        fill_new(c)
        verify(c, attend(c))
        torch.cuda.synchronize()
        assert int(status) == T.OK
        tables[3][1] = -1                                   # a block that is attended to
        attend(c)
        torch.cuda.synchronize()
        assert int(status) == T.EFAULT
    finally:
        c.close()


def test_tensors_that_are_refused():
    c = OpCase([(40, 2), (200, 2)], seed=91)
    try:
        out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        before = c.pool.clone()
        tok, io = T.make_tokens(c.k, c.v, c.q, out), T.make_attend(c.q, out)
        few = c.n_tok - 1
        host = T.make_step(c.t_q_start.cpu(), c.t_ctx, c.t_blk_start, c.t_ids, c.n_tok, c.max_new)
        for call in (lambda: c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k[:few], c.v[:few], c.q[:few], out[:few])),
                     lambda: c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k.cpu(), c.v)),
                     lambda: c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k[:, :1], c.v[:, :1])),
                     lambda: c.ctx.tutti_kv_append_layer(1, c.step, tok, T.make_rope(table_of(300, 128).cpu())),
                     lambda: c.ctx.tutti_kv_append_layer(1, host, tok),
                     lambda: c.attn.tutti_kv_attend_layer(1, host, io, 1.0),
                     lambda: c.attn.tutti_kv_attend_layer(1, c.step, T.make_attend(c.q[:few], out[:few]), 1.0),
                     lambda: c.attn.tutti_kv_attend_layer(1, c.step, T.make_attend(c.q, out.cpu()), 1.0),
                     lambda: c.attn.tutti_kv_attend_layer(1, c.step, T.make_attend(c.q, out, torch.zeros(c.n_tok, c.heads)), 1.0)):
            with pytest.raises(T.TuttiError):
                call()
        torch.cuda.synchronize()
        assert (out == 7.5).all() and torch.equal(before, c.pool)
        attn = T.Attn(c.ctx)
        attn.close()
        with pytest.raises(T.TuttiError):
            attn.tutti_kv_attend_layer(1, c.step, io, 1.0)
    finally:
        c.close()
