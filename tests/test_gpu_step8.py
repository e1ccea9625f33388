"""hb_mixed_step8, the step with 8-bit projection weights: against the operators called one by one (bit by bit), against the
64-bit definition of its tail, and against the step with 16-bit weights."""
import numpy as np
import pytest
import torch

from paper_2609_25405_b200 import binding as B
from paper_2609_25405_b200 import synth
from paper_2609_25405_b200.engine import Engine, Request
from tests.dense_util import E4M3, check, linear64

pytestmark = pytest.mark.gpu

TINY = synth.SHAPES["tiny"]
WIDE = synth.ModelShape("step8-wide", 2, 512, 4, 1, 128, 1024, 1024)


@pytest.fixture(scope="module", params=["tiny", "wide"])
def model(request):
    shape = TINY if request.param == "tiny" else WIDE
    W = synth.Weights(shape, 0)
    return shape, W, B.DeviceWeights8.from_synth(W)


def _engine(shape, dw, **kw):
    args = dict(n_pages=64, n_slots=4, max_tokens=512, max_segs=16, max_pos=256, kv_fill=0x7F, kv_dtype="e4m3")
    return Engine(shape, dw, **dict(args, **kw))


def _by_hand(eng, dw, W, batch, kv):
    """The residual stream [T, d] after the layers, by the public operators."""
    s, ctx = eng.shape, eng.ctx
    T, n_q = batch.n_tokens, s.Hq * s.Dh
    rows = B.SegRows.from_batch(batch)
    rope = B.Rope.table(eng.cfg.max_pos, s.Dh, s.rope_theta)
    x = torch.from_numpy(np.asarray(W.tok_emb, dtype=np.float32)[batch.token_ids]).cuda()
    new = lambda n, t: torch.empty(T, n, device="cuda", dtype=t)   # noqa: E731
    scale = torch.empty(T, device="cuda")
    for l in range(s.L):
        gain = lambda n: B.bf16_from_f32(W.layer(l)[n])   # noqa: E731
        c = dw.codes[l]
        h = new(s.d, E4M3)
        ctx.norm(x, gain("attn_norm"), h, y_scale=scale)
        qkv, q, o = new(s.n_qkv, torch.float16), new(n_q, torch.float16), new(n_q, torch.float16)
        ctx.linear(h, c["wqkv"][0], qkv, a_scale=scale, w_scale=c["wqkv"][1])
        ctx.kv8_append(kv, l, rows, qkv, q, rope=rope)
        ctx.kv8_attention(kv, l, rows, q, o)
        oc = new(n_q, E4M3)
        ctx.quant_rows(o, oc, scale)
        ctx.linear(oc, c["wo"][0], x, a_scale=scale, w_scale=c["wo"][1], residual=x)
        ctx.norm(x, gain("ffn_norm"), h, y_scale=scale)
        act, ac = new(s.F, torch.float16), new(s.F, E4M3)
        ctx.linear(h, c["w_gate_up"][0], act, a_scale=scale, w_scale=c["w_gate_up"][1], act=B.ACT_SILU, gated=True)
        ctx.quant_rows(act, ac, scale)
        ctx.linear(ac, c["w_down"][0], x, a_scale=scale, w_scale=c["w_down"][1], residual=x)
    return x


def test_step_is_its_operators(model):
    """Prompt chunks, decode rows and embedding chunks: cache bytes equal bit by bit, logits and embeddings by the tail's definition
    from the operators' residual stream."""
    shape, W, dw = model
    eng = _engine(shape, dw)
    rng = np.random.default_rng(5)
    reqs = [Request("gen", synth.token_ids(rng, n, shape.V)) for n in (70, 33)]
    emb = [Request("embed", synth.token_ids(rng, n, shape.V), m) for n, m in ((90, B.POOL_LAST), (40, B.POOL_LAST))]
    kv2 = B.KvCache8(eng.cfg, 64, fill=0x7F)
    plan = [[(reqs[0], 50), (emb[0], 64)], [(reqs[0], 20), (reqs[1], 33), (emb[1], 40)], None]
    gain = torch.from_numpy(np.asarray(W.final_norm, dtype=np.float64)).cuda()
    head = torch.from_numpy(np.asarray(W.lm_head, dtype=np.float64)).cuda()
    for step, work in enumerate(plan):
        if work is None:
            for r in reqs:
                r.tokens.append(7)
            work = [(reqs[0], 1), (reqs[1], 1), (emb[0], 26)]
        batch, lrows, erows = eng.step(work)
        x = _by_hand(eng, dw, W, batch, kv2)
        torch.cuda.synchronize()
        assert torch.equal(eng.kv.arena, kv2.arena)
        y = x.double()
        y = y / (y.square().mean(dim=1, keepdim=True) + shape.rms_eps).sqrt() * gain
        for seg in batch.segs:
            last = int(seg["q_start"] + seg["q_len"]) - 1
            if seg["logits_row"] >= 0:
                # hi + lo of the final rows: 2^-22 of each; their products over 2 d columns
                want, bound = linear64(torch.cat([y[last:last + 1]] * 2, 1) / 2, torch.cat([head, head], 1))
                check(eng.out_logits[int(seg["logits_row"])][None], want, bound + want.abs().max() * 2.0 ** -18)
            if seg["emb_row"] >= 0:
                e = y[last] / y[last].norm()
                assert float((eng.out_emb[int(seg["emb_row"])].double() - e).abs().max()) <= 2.0 ** -18
        if step == 1:
            assert len(lrows) == 2 and len(erows) == 1
    assert eng.ctx.status_poll() == 0
    eng.close()


def test_close_to_the_step_with_16_bit_weights(model):
    """Each projection's operands are rounded to e4m3, off by at most 2^-4 and so 2^-4 / sqrt(3) in the mean, two operands and four
    projections a layer: sqrt(2 * 4 * L) * 0.036 of the result in all if nothing of it cancels, 15 % for two layers, a cosine of
    0.99.  Demanded: 0.98."""
    shape, W, dw = model
    ref = B.DeviceWeights.from_synth(W)
    rng = np.random.default_rng(9)
    prompt, text = synth.token_ids(rng, 60, shape.V), synth.token_ids(rng, 100, shape.V)
    got = []
    for weights in (dw, ref):
        eng = _engine(shape, weights)
        g, e = Request("gen", prompt), Request("embed", text, B.POOL_MEAN)
        _, lrows, erows = eng.step([(g, 60), (e, 100)])
        torch.cuda.synchronize()
        assert eng.ctx.status_poll() == 0
        got.append((eng.out_logits[lrows[g]].double().clone(), eng.out_emb[erows[e]].double().clone()))
        eng.close()
    for a, b in zip(*got):
        assert float(torch.nn.functional.cosine_similarity(a, b, dim=0)) >= 0.98


def test_refusals(model):
    shape, W, dw = model
    with pytest.raises(ValueError):
        _engine(shape, dw, kv_dtype="f16")
    eng = _engine(shape, dw)
    r = Request("gen", [1, 2, 3])
    batch, _, _ = eng.step([(r, 3)])
    kv16 = B.KvCache(eng.cfg, 64)
    with pytest.raises(ValueError):
        eng.ctx.mixed_step(batch, dw, kv16, eng.pool, eng.out_logits, eng.out_emb)
    import ctypes as C
    call = lambda w, kv: B.lib.hb_mixed_step8(eng.ctx.handle, C.byref(batch.desc), C.byref(w), kv.handle, eng.pool.handle,   # noqa: E731
                                              C.c_void_p(eng.out_logits.data_ptr()), C.c_void_p(eng.out_emb.data_ptr()), None)
    assert call(dw.struct, kv16) == -1
    bad = B.Weights8(dw.struct.tok_emb, None, dw.struct.final_norm, dw.struct.lm_head)
    assert call(bad, eng.kv) == -1
    layers = (B.LayerWeights8 * shape.L)(*dw.layers)
    bad.layers = C.cast(layers, C.POINTER(B.LayerWeights8))
    for name, value in (("wo", None), ("wo", layers[1].wo + 8), ("down_scale", None), ("ffn_norm", layers[1].ffn_norm + 2)):
        was = getattr(layers[1], name)
        setattr(layers[1], name, value)
        assert call(bad, eng.kv) == -1
        setattr(layers[1], name, was)
    assert call(bad, eng.kv) == 0
    torch.cuda.synchronize()
    eng.close()
