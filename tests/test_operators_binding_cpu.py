"""What the binding of the operators on the pool refuses before the library is called: tensors that do not fit each
other, the step, the geometry or the context's GPU."""
import ctypes as C

import pytest
import torch

from paper_2605_03375_b200 import tutti as T

HALF = torch.float16


def ints(n, dtype=torch.int32):
    return torch.zeros(n, dtype=dtype)


def rows(n, heads, dim=64, dtype=HALF):
    return torch.zeros(n, heads, dim, dtype=dtype)


def handles(device, kv_heads=2, dim=64):
    """A context and an attention handle whose calls reach the library with a null pointer: it answers EINVAL."""
    ctx = T.Context.__new__(T.Context)
    ctx.lib, ctx.h, ctx.device, ctx._row = T.load(), C.c_void_p(None), device, (kv_heads, dim)
    attn = T.Attn.__new__(T.Attn)
    attn.lib, attn.h, attn.ctx = ctx.lib, C.c_void_p(None), ctx
    return ctx, attn


def refused(call, *words):
    with pytest.raises(T.TuttiError) as e:
        call()
    assert e.value.code == T.EINVAL and all(w in str(e.value) for w in words), str(e.value)


def test_tensors_of_different_shapes():
    k, q = rows(4, 2), rows(4, 8)
    assert T.make_tokens(k, k, q, q).n_q_heads == 8
    refused(lambda: T.make_tokens(k, rows(3, 2)), "one shape")
    refused(lambda: T.make_tokens(k, rows(4, 1)), "one shape")
    refused(lambda: T.make_tokens(k, rows(4, 2, 128)), "one shape")
    refused(lambda: T.make_tokens(k, k, q, rows(4, 4)), "one shape")
    refused(lambda: T.make_tokens(k, k, q, rows(3, 8)), "one shape")
    refused(lambda: T.make_tokens(k, k, rows(3, 8), rows(3, 8)), "one shape")
    refused(lambda: T.make_tokens(k, k, q), "one shape")
    refused(lambda: T.make_attend(q, rows(3, 8)), "one shape")
    refused(lambda: T.make_attend(q, rows(4, 4)), "one shape")
    refused(lambda: T.make_attend(q, rows(4, 8), torch.zeros(3, 8)), "lse")
    refused(lambda: T.make_attend(q, rows(4, 8), torch.zeros(4, 4)), "lse")
    refused(lambda: T.make_attend(q, rows(4, 8), torch.zeros(32)), "lse")
    refused(lambda: T.make_attend(q, rows(4, 8), torch.zeros(4, 8, dtype=torch.float64)), "lse")
    refused(lambda: T.make_attend(q, rows(4, 8), torch.zeros(8, 4).t()), "lse")
    refused(lambda: T.make_attend(q, rows(4, 8, dtype=torch.bfloat16)), "type")


def test_tables_of_a_step():
    ok = T.make_step(ints(3), ints(2), ints(3), ints(5), 4, 2, ints(1))
    assert ok.n_seq == 2 and ok.n_blk == 5 and ok.status
    longer = T.make_step(ints(9), ints(2), ints(9), ints(5), 4, 2)      # tables of a larger batch are fine
    assert longer.n_seq == 2 and not longer.status
    assert T.make_step(ints(0), ints(0), ints(0), ints(0), 0, 0).n_seq == 0
    refused(lambda: T.make_step(ints(2), ints(2), ints(3), ints(5), 4, 2), "entry more")
    refused(lambda: T.make_step(ints(3), ints(2), ints(2), ints(5), 4, 2), "entry more")
    refused(lambda: T.make_step(ints(3), ints(2, torch.float32), ints(3), ints(5), 4, 2), "int32")
    refused(lambda: T.make_step(ints(3), ints(2), ints(3), ints(5, torch.int64), 4, 2), "int32")
    refused(lambda: T.make_step(ints(3), ints(2), ints(3), ints(10)[::2], 4, 2), "int32")
    refused(lambda: T.make_step(ints(3), ints(2), ints(3), ints(5), 4, 2, ints(0)), "status")
    refused(lambda: T.make_step(ints(3), ints(2), ints(3), ints(5), 4, 2, ints(1, torch.int64)), "status")


def test_calls_compare_the_structs_with_each_other_and_the_geometry():
    ctx, attn = handles(-1)                     # the "GPU" of tensors in host memory
    step = T.make_step(ints(3), ints(2), ints(3), ints(5), 4, 2)
    append = lambda t, s=step, r=None: ctx.tutti_kv_append_layer(0, s, t, r, allow=(T.EINVAL,))  # noqa: E731
    attend = lambda a, s=step: attn.tutti_kv_attend_layer(0, s, a, 1.0, allow=(T.EINVAL,))  # noqa: E731
    k, q = rows(4, 2), rows(4, 8)
    assert append(T.make_tokens(k, k)) == T.EINVAL                       # these reach the library
    assert append(T.make_tokens(rows(9, 2), rows(9, 2)), r=T.make_rope(torch.zeros(9, 32))) == T.EINVAL
    assert append(T.Tokens(), T.Step(), T.Rope()) == T.EINVAL            # structs made by hand are not looked into
    assert attend(T.make_attend(q, rows(4, 8), torch.zeros(4, 8))) == T.EINVAL and attend(T.Attend(), T.Step()) == T.EINVAL
    refused(lambda: append(T.make_tokens(rows(3, 2), rows(3, 2))), "n_tok")
    refused(lambda: append(T.make_tokens(rows(4, 1), rows(4, 1))), "n_kv_heads")
    refused(lambda: append(T.make_tokens(rows(4, 2, 128), rows(4, 2, 128))), "head_dim")
    refused(lambda: attend(T.make_attend(rows(3, 8), rows(3, 8))), "n_tok")
    refused(lambda: attend(T.make_attend(rows(4, 8, 128), rows(4, 8, 128))), "head_dim")


def test_calls_want_their_tensors_where_the_gpu_reaches_them():
    ctx, attn = handles(0)
    k, q = rows(4, 2), rows(4, 8)
    step = T.make_step(ints(3), ints(2), ints(3), ints(5), 4, 2)
    refused(lambda: ctx.tutti_kv_append_layer(0, step, T.Tokens()), "cpu", "GPU 0")
    refused(lambda: ctx.tutti_kv_append_layer(0, T.Step(), T.make_tokens(k, k)), "cpu", "GPU 0")
    refused(lambda: ctx.tutti_kv_append_layer(0, T.Step(), T.make_tokens(k, k, q, q)), "cpu", "GPU 0")
    refused(lambda: ctx.tutti_kv_append_layer(0, T.Step(), T.Tokens(), T.make_rope(torch.zeros(9, 32))), "cpu", "GPU 0")
    refused(lambda: attn.tutti_kv_attend_layer(0, step, T.Attend(), 1.0), "cpu", "GPU 0")
    refused(lambda: attn.tutti_kv_attend_layer(0, T.Step(), T.make_attend(q, rows(4, 8)), 1.0), "cpu", "GPU 0")


def test_closed_handles():
    ctx, attn = handles(-1)
    ctx.h = None
    refused(lambda: attn.tutti_kv_attend_layer(0, T.Step(), T.Attend(), 1.0), "closed")
    ctx.h, attn.h = C.c_void_p(None), None
    refused(lambda: attn.tutti_kv_attend_layer(0, T.Step(), T.Attend(), 1.0), "closed")


def test_structs_keep_their_tensors():
    import weakref
    t = T.make_rope(torch.zeros(9, 32))
    k = rows(4, 2)
    there = weakref.ref(k)
    tokens, io = T.make_tokens(k, k), T.make_attend(k, rows(4, 2))
    del k
    assert there() is not None and t._of[1].data_ptr() == t.table
    del tokens
    assert there() is not None
    del io
    assert there() is None


def test_scale_rows_of_no_context():
    lib = T.load()
    assert lib.tutti_scales_register_rows(None, 0, None, None, 0, 4) == T.EINVAL
