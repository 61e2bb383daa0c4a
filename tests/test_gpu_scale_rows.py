"""8-bit pools whose scales lie in rows longer than the number of KV heads, so that they can be saved and restored for
any number of heads."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import OpCase
from tests.test_gpu_append import append, verify as append_verify
from tests.test_gpu_attend import attend, fill_new, verify
from tests.test_gpu_operators import Served

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("kv_heads,row", [(1, 4), (2, 4), (3, 4), (5, 8), (2, 2), (2, 7)])
def test_operators_with_rows_of_scales(kv_heads, row, new):
    c = OpCase([(40, new), (200, new), (7, new)], heads=2 * kv_heads, kv_heads=kv_heads, cache="8", seed=95 + row)
    try:
        wide = [torch.full((c.n_blocks, row), float("nan"), device=c.dev) for _ in range(2)]
        for half in range(2):
            wide[half][:, :kv_heads] = c.scale_dev[half]
            c.scale_dev[half].fill_(float("nan"))
        c.ctx.tutti_scales_register_rows(1, wide[0].data_ptr(), wide[1].data_ptr(), c.n_blocks, row)
        c.scale_dev = [w[:, :kv_heads] for w in wide]
        append_verify(c, append(c))
        fill_new(c)
        verify(c, attend(c))
        assert all(torch.isnan(w[:, kv_heads:]).all() for w in wide)
        assert int(c.status) == T.OK
    finally:
        c.close()


def test_rows_that_are_refused():
    c = OpCase([(40, 1)], heads=4, kv_heads=4, cache="8", seed=96)
    try:
        k, v = (s.data_ptr() for s in c.scale_dev)
        c.ctx.tutti_scales_register_rows(1, k, v, c.n_blocks, 4)
        for layer, a, b, n, row in ((1, k, v, c.n_blocks, 3), (1, k, v, c.n_blocks, 0), (1, k, v, c.n_blocks - 1, 4), (1, k + 2, v, c.n_blocks, 4),
                                    (1, k, 0, c.n_blocks, 4), (0, k, v, c.n_blocks, 4), (2, k, v, c.n_blocks, 4)):
            with pytest.raises(T.TuttiError):
                c.ctx.tutti_scales_register_rows(layer, a, b, n, row)
    finally:
        c.close()


class ServedRows(Served):
    """Served over an 8-bit pool with a padded row of scales for each block."""

    def __init__(self, hk, dim=64, bs=16, n_blocks=64, obj=32, n_slots=8, heads=6):
        self.hk, self.dim, self.bs, self.heads, self.size = hk, dim, bs, heads, 1
        self.dev = torch.device("cuda", 0)
        bb, row = bs * hk * dim, -(-hk // 4) * 4
        self.pool = torch.full((2, n_blocks * bb), 0xFF, dtype=torch.uint8, device=self.dev)
        self.scales = torch.full((2, n_blocks, row), float("nan"), device=self.dev)
        self.parts = [self._part(T.Geom(1, hk, dim, 1, bs, obj, 1, T.LAYOUT_LAYER_MAJOR, n_slots), self.pool, bb, n_blocks),
                      self._part(T.Geom(1, row, 1, 4, 1, obj // bs, 1, T.LAYOUT_LAYER_MAJOR, n_slots), self.scales, 4 * row, n_blocks)]
        self.ctx = self.parts[0][0]
        self.ctx.tutti_scales_register_rows(0, self.scales[0].data_ptr(), self.scales[1].data_ptr(), n_blocks, row)
        self.attn = T.Attn(self.ctx)
        a = np.arange(512)[:, None] * 10000.0 ** (-np.arange(dim // 2) * 2 / dim)
        self.table = torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).to(self.dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.dev)


@pytest.mark.parametrize("hk", [1, 2, 3, 6])
def test_a_prompt_is_saved_and_restored_for_any_number_of_heads(hk):
    s = ServedRows(hk)
    try:
        g = torch.Generator(device=s.dev).manual_seed(hk)
        x = torch.randn(110, (s.heads + 2 * hk) * s.dim, generator=g, device=s.dev).to(torch.bfloat16)
        here, there = list(range(3, 30, 2)), list(range(40, 60))
        s.run(x[:96], 96, here)
        s.move(T.OP_WRITE, here[:6], [5, 1, 6], 96)
        want = [s.run(x[96:109], 109, here), s.run(x[109:110], 110, here)]
        s.move(T.OP_READ, there[:6], [5, 1, 6], 96)
        got = [s.run(x[96:109], 109, there), s.run(x[109:110], 110, there)]
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[0].float()).all()
    finally:
        s.close()
