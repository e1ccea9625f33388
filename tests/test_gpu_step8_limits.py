"""hb_mixed_step8: sizes that it refuses, and what its status says of values that do not fit fp16."""

import numpy as np
import pytest
import torch

from paper_2609_25405_b200 import binding as B
from paper_2609_25405_b200 import synth
from paper_2609_25405_b200.engine import Engine, Request
from tests.dense_util import E4M3

pytestmark = pytest.mark.gpu


def _codes_weights(shape, gain=1.0, emb=None, **scales):
    """DeviceWeights8 of constant codes, made without hb_quant_rows: a caller's own."""
    dw = B.DeviceWeights8(shape.L)
    ones = torch.full((shape.d,), gain, device="cuda", dtype=torch.bfloat16)
    for l in range(shape.L):
        dw.layers[l].attn_norm = dw.layers[l].ffn_norm = dw._keep(ones)
        for name, scale, r, c in (("wqkv", "wqkv_scale", shape.n_qkv, shape.d), ("wo", "wo_scale", shape.d, shape.Hq * shape.Dh),
                                  ("w_gate_up", "gate_up_scale", 2 * shape.F, shape.d), ("w_down", "down_scale", shape.d, shape.F)):
            setattr(dw.layers[l], name, dw._keep(torch.ones((r, c), device="cuda").to(E4M3)))
            setattr(dw.layers[l], scale, dw._keep(torch.full((r,), scales.get(name, 2.0 ** -9), device="cuda")))
    if emb is None:
        emb = torch.rand(shape.V, shape.d, device="cuda")
    return dw._rest(emb.bfloat16(), ones, torch.zeros(shape.V, shape.d, device="cuda", dtype=torch.float16))


@pytest.mark.parametrize("shape", [synth.ModelShape("step8-long-ffn", 1, 64, 1, 1, 64, 40960, 64),
                                   synth.ModelShape("step8-long-ffn-1", 1, 64, 1, 1, 64, 32832, 64),
                                   synth.ModelShape("step8-many-heads", 1, 64, 272, 272, 128, 64, 64)])
def test_rows_too_long_for_codes_are_refused(shape):
    """Inner rows or attention rows of more than 32768 elements, with a caller's own codes."""
    dw = _codes_weights(shape)
    eng = Engine(shape, dw, n_pages=8, n_slots=1, max_tokens=16, max_segs=2, max_pos=64, kv_dtype="e4m3")
    with pytest.raises(B.HbError, match="TOO_LARGE"):
        eng.step([(Request("gen", np.array([1, 2, 3], dtype=np.int32)), 3)])
    torch.cuda.synchronize()
    assert eng.ctx.status_poll() == 0
    eng.close()


def _status(dw, shape):
    eng = Engine(shape, dw, n_pages=8, n_slots=1, max_tokens=16, max_segs=2, max_pos=64, kv_dtype="e4m3")
    eng.step([(Request("gen", np.arange(1, 9, dtype=np.int32)), 8)])
    torch.cuda.synchronize()
    got = eng.ctx.status_poll()
    eng.close()
    return got


@pytest.mark.parametrize("layers", [1, 2])
def test_status_of_values_beyond_fp16(layers):
    """Rows of one sign, so that every product is positive: a row's normed values are 0.9 in the mean, its 64 products about 55, times the scale."""
    shape = synth.ModelShape("step8-range", layers, 64, 1, 1, 64, 128, 64)
    assert _status(_codes_weights(shape), shape) == 0
    # gate = up = 55 x 16: their product passes 65504
    assert _status(_codes_weights(shape, w_gate_up=16.0), shape) == 64
    # a gain whose normed rows would not fit fp16, but do fit codes; everything behind it is small
    assert _status(_codes_weights(shape, gain=1e6, wqkv=2.0 ** -30, w_gate_up=2.0 ** -30), shape) == 0
    # v = 55 x 4096: the projection saturates, and so does the attention's output
    assert _status(_codes_weights(shape, wqkv=4096.0), shape) == 64
    emb = torch.rand(shape.V, shape.d, device="cuda")
    emb[3, 5] = float("nan")
    assert _status(_codes_weights(shape, emb=emb), shape) == 64
