"""hb_mixed_step8 at the 7B class's widths: long sums onto the residual stream, codes in place by several warps a row, pairs of CTAs."""
import numpy as np
import pytest
import torch

from paper_2609_25405_b200 import binding as B
from paper_2609_25405_b200 import synth
from paper_2609_25405_b200.engine import Engine, Request
from tests.dense_util import E4M3, check, linear64
from tests.test_linear_variant import variant

SHAPE = synth.ModelShape("step8-7b-widths", 2, 4096, 32, 8, 128, 14336, 1024)


def test_the_steps_take_long_sums_and_pairs():
    """Of the steps below: projections onto the residual stream leave in segments, a full step's by pairs."""
    for m, tokens in ((1700, 256), (401, 128)):
        for k in (4096, 14336):
            assert variant(m, 4096, k, B.DTYPE_E4M3, B.DTYPE_F32) == (tokens, 1, 1)
        assert variant(m, 28672, 4096, B.DTYPE_E4M3) == (256, 1, 0)
    assert variant(2, 4096, 14336, B.DTYPE_E4M3, B.DTYPE_F32)[0] == 8


def _rows_of_product(a, a_scale, w, w_scale, got, was, rows, act="none", gated=False):
    """Sampled rows of a product against the definition; `was`: the residual before it."""
    check(got[rows], *linear64(a[rows], w, a_scale[rows], w_scale, None, act, gated, None if was is None else was[rows], got.dtype))


def _by_hand(eng, dw, emb, batch, kv):
    """The residual stream after the layers, by the public operators, each product of the first layer held to its definition."""
    s, ctx = eng.shape, eng.ctx
    T, n_q = batch.n_tokens, s.Hq * s.Dh
    rows = B.SegRows.from_batch(batch)
    rope = B.Rope.table(eng.cfg.max_pos, s.Dh, s.rope_theta)
    x = emb[torch.from_numpy(np.asarray(batch.token_ids)).long().cuda()].float()
    new = lambda n, t: torch.empty(T, n, device="cuda", dtype=t)   # noqa: E731
    scale, ones = torch.empty(T, device="cuda"), torch.ones(s.d, device="cuda", dtype=torch.bfloat16)
    some = torch.unique(torch.linspace(0, T - 1, 5).long()).cuda()
    for l in range(s.L):
        c = dw.codes[l]
        first = _rows_of_product if l == 0 else lambda *a, **k: None
        h = new(s.d, E4M3)
        ctx.norm(x, ones, h, y_scale=scale)
        qkv, q, o = new(s.n_qkv, torch.float16), new(n_q, torch.float16), new(n_q, torch.float16)
        ctx.linear(h, c["wqkv"][0], qkv, a_scale=scale, w_scale=c["wqkv"][1])
        first(h, scale, *c["wqkv"], qkv, None, some)
        ctx.kv8_append(kv, l, rows, qkv, q, rope=rope)
        ctx.kv8_attention(kv, l, rows, q, o)
        oc = new(n_q, E4M3)
        ctx.quant_rows(o, oc, scale)
        was = x.clone()
        ctx.linear(oc, c["wo"][0], x, a_scale=scale, w_scale=c["wo"][1], residual=x)
        first(oc, scale, *c["wo"], x, was, some)
        ctx.norm(x, ones, h, y_scale=scale)
        act, ac = new(s.F, torch.float16), new(s.F, E4M3)
        ctx.linear(h, c["w_gate_up"][0], act, a_scale=scale, w_scale=c["w_gate_up"][1], act=B.ACT_SILU, gated=True)
        first(h, scale, *c["w_gate_up"], act, None, some, "silu", True)
        ctx.quant_rows(act, ac, scale)
        was = x.clone()
        ctx.linear(ac, c["w_down"][0], x, a_scale=scale, w_scale=c["w_down"][1], residual=x)
        first(ac, scale, *c["w_down"], x, was, some)
    return x


@pytest.mark.gpu
def test_step_is_its_operators_at_7b_widths():
    """Full steps and a decode step: cache bytes equal bit by bit, logits and embeddings by the tail's definition from the residual stream."""
    dw = B.DeviceWeights8.random_on_device(SHAPE, seed=3)
    emb, head = dw.tensors[-3], dw.tensors[-1].double()
    eng = Engine(SHAPE, dw, n_pages=256, n_slots=4, max_tokens=2048, max_segs=8, max_pos=2048, kv_fill=0x7F, kv_dtype="e4m3")
    kv2 = B.KvCache8(eng.cfg, 256, fill=0x7F)
    rng = np.random.default_rng(6)
    gen = [Request("gen", synth.token_ids(rng, n, SHAPE.V)) for n in (200, 1)]
    text = Request("embed", synth.token_ids(rng, 1900, SHAPE.V), B.POOL_LAST)
    for work in ([(gen[0], 200), (text, 1500)], [(gen[1], 1), (text, 400)], None):
        if work is None:
            for r in gen:
                r.tokens.append(7)
            work = [(r, 1) for r in gen]
        batch, _, _ = eng.step(work)
        x = _by_hand(eng, dw, emb, batch, kv2)
        torch.cuda.synchronize()
        assert torch.equal(eng.kv.arena, kv2.arena)
        y = x.double()
        y = y / (y.square().mean(dim=1, keepdim=True) + SHAPE.rms_eps).sqrt()
        for seg in batch.segs:
            last = int(seg["q_start"] + seg["q_len"]) - 1
            if seg["logits_row"] >= 0:
                want, bound = linear64(torch.cat([y[last:last + 1]] * 2, 1) / 2, torch.cat([head, head], 1))
                check(eng.out_logits[int(seg["logits_row"])][None], want, bound + want.abs().max() * 2.0 ** -18)
            if seg["emb_row"] >= 0:
                e = y[last] / y[last].norm()
                assert float((eng.out_emb[int(seg["emb_row"])].double() - e).abs().max()) <= 2.0 ** -18
    assert eng.ctx.status_poll() == 0
    eng.close()
