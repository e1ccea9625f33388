"""Rows of C inside wider rows, of every length against a 16-byte boundary: nothing behind them is written."""
import pytest
import torch

from tests.dense_util import ACTS, check, ctx, gen, linear64, operand, status
from tests.test_linear_variant import B, variant

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("c_t", [F32, F16, BF16])
@pytest.mark.parametrize("m,n,k", [(66, 142, 41), (66, 1000, 41), (134, 130, 41), (272, 134, 40), (3961, 530, 200), (1, 26000, 4096), (70, 142, 1500)])
@pytest.mark.parametrize("gated,residual", [(False, True), (True, False)])
def test_nothing_behind_a_row(m, n, k, c_t, gated, residual):
    g = gen(m + n)
    a, w = operand(g, m, k, F16), operand(g, n, k, F16, 0.05)
    for short in range(0, 8, 3 if n < 5000 else 7):
        cols = (n - 2 * short) // (2 if gated else 1)
        rows = cols * (2 if gated else 1)
        per = 16 // torch.empty(0, dtype=c_t).element_size()
        pitch = (cols + per - 1) // per * per        # rows on 16-byte boundaries
        whole = torch.full(((m + 2) * pitch,), 9.0, device="cuda", dtype=c_t)
        out = whole[pitch:].as_strided((m, cols), (pitch, 1))
        r = None if not residual else torch.randn(m, cols, generator=g, device="cuda").to(c_t)
        ctx().linear(a, w[:rows], out, act=ACTS["silu" if gated else "none"], gated=gated, residual=r)
        check(out, *linear64(a, w[:rows], act="silu" if gated else "none", gated=gated, residual=r, c_dtype=c_t))
        out.fill_(9.0)
        assert bool((whole == 9.0).all())
    assert status() == 0


def test_the_sizes_take_tiles():
    """All but the last take kernels whose blocks of results leave by copies; one row among them."""
    for m, n, k in ((66, 142, 41), (134, 130, 41), (272, 134, 40), (3961, 530, 200), (1, 26000, 4096)):
        tokens, share, _ = variant(m, n, k, B.DTYPE_F16, B.DTYPE_F16)
        assert tokens >= 32 and share == 1, (m, n, k, tokens, share)
