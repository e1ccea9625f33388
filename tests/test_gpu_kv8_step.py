"""hb_mixed_step over an 8-bit cache: the whole path against a float64 forward whose keys and values go through the
same cache (oracle.kv8), and against itself (batch composition, adapters, captures of memory)."""
import numpy as np
import pytest
import torch

from oracle import kv8 as O
from oracle import method as M
from oracle.transformer import apply_rope, l2_normalise, rmsnorm, rope_cos_sin, silu
from paper_2609_25405_b200 import synth

pytestmark = pytest.mark.gpu

TINY = synth.SHAPES["tiny"]
# 4 query heads on 1 KV head of 128, two layers
WIDE = synth.ModelShape("kv8-wide", 2, 512, 4, 1, 128, 1024, 1024)
# the step's own tolerances: logits max-abs 5e-2, embeddings cosine 0.9995 and max-abs 2e-2.  On top of the fp16
# path a key or value that lands next to a rounding border of e4m3 may take the neighbouring code (fp16 rounding of
# the projection, 2^-11, against steps of 2^-3 .. 2^-4: about one element in a hundred, by a sixteenth)
EMB_COS, EMB_ABS, LOGIT_ABS = 0.9995, 2e-2, 5e-2


class Ref:
    """One request: its tokens so far and an 8-bit cache of its own, layer by layer."""

    def __init__(self, shape, W, n_pages=24, lora=None):
        self.s, self.W, self.n, self.lora = shape, W, 0, lora
        self.cache = [O.Cache([np.zeros((n_pages, shape.Hkv, 16, shape.Dh)) for _ in range(2)],
                              [np.full((n_pages, shape.Hkv), O.E_MIN) for _ in range(2)]) for _ in range(shape.L)]
        self.H = np.zeros((0, shape.d))

    def rows(self, tokens):
        """Final hidden states of `tokens`, the next rows of the request."""
        s, W = self.s, self.W
        c, p0 = len(tokens), self.n
        x = np.asarray(W.tok_emb)[np.asarray(tokens)].astype(np.float64)
        cos, sin = rope_cos_sin(s.Dh, s.rope_theta, np.arange(p0, p0 + c), np.float64)
        for l in range(s.L):
            w = W.layer(l)
            proj = lambda h, n: M._proj(h, w, n, self.lora, l, np.float64)  # noqa: E731
            h = rmsnorm(x, w["attn_norm"].astype(np.float64), s.rms_eps)
            q = apply_rope(proj(h, "wq").reshape(c, s.Hq, s.Dh), cos, sin)
            k = apply_rope(proj(h, "wk").reshape(c, s.Hkv, s.Dh), cos, sin)
            v = proj(h, "wv").reshape(c, s.Hkv, s.Dh)
            for b in range(p0 // 16, (p0 + c + 15) // 16):
                lo, hi = max(p0, b * 16), min(p0 + c, b * 16 + 16)
                self.cache[l].append(0, b, lo - b * 16, k[lo - p0:hi - p0])
                self.cache[l].append(1, b, lo - b * 16, v[lo - p0:hi - p0])
            pages = np.arange((p0 + c + 15) // 16)
            o, _ = O.attend(q, *(self.cache[l].rows(i, pages, p0 + c) for i in range(2)), p0, s.Dh ** -0.5)
            x = x + proj(o.reshape(c, -1), "wo")
            h = rmsnorm(x, w["ffn_norm"].astype(np.float64), s.rms_eps)
            x = x + proj(silu(proj(h, "wg")) * proj(h, "wu"), "wd")
        self.n += c
        H = rmsnorm(x, np.asarray(W.final_norm).astype(np.float64), s.rms_eps)
        self.H = np.concatenate([self.H, H])
        return H

    def logits(self, tokens):
        return self.rows(tokens)[-1] @ np.asarray(self.W.lm_head).astype(np.float64).T


def _engine(shape, dw, **kw):
    from paper_2609_25405_b200.engine import Engine
    args = dict(n_pages=64, n_slots=4, max_tokens=512, max_segs=16, max_pos=256, kv_fill=0x7F, kv_dtype="e4m3")
    return Engine(shape, dw, **dict(args, **kw))


@pytest.fixture(scope="module", params=["tiny", "wide"])
def model(request):
    from paper_2609_25405_b200 import binding as B
    shape = TINY if request.param == "tiny" else WIDE
    W = synth.Weights(shape, 0)
    return shape, W, B.DeviceWeights.from_synth(W)


def test_mixed_workload(model):
    """Prompts in chunks, teacher-forced decode, embedding chunks in the same steps; last token and mean pooling."""
    from paper_2609_25405_b200 import binding as B
    from paper_2609_25405_b200.engine import Request
    shape, W, dw = model
    eng = _engine(shape, dw)
    r = np.random.default_rng(4)
    gens = [Request("gen", synth.token_ids(r, n, shape.V)) for n in (20, 33)]
    texts = [synth.token_ids(r, n, shape.V) for n in (70, 45)]
    embs = [Request("embed", texts[0], B.POOL_MEAN), Request("embed", texts[1], B.POOL_LAST)]
    ref_g, ref_e = [Ref(shape, W) for _ in gens], [Ref(shape, W) for _ in embs]
    plan = [[(gens[0], 20), (gens[1], 16), (embs[0], 32)], [(gens[0], 1), (gens[1], 17), (embs[0], 7), (embs[1], 45)]]
    plan += [[(gens[0], 1), (gens[1], 1), (embs[0], 31)], [(gens[0], 1), (gens[1], 1)]]
    worst, emb_rows = 0.0, {}
    for work in plan:
        for q, n in work:
            while q.kind == "gen" and q.remaining() < n:
                q.tokens.append(int(r.integers(shape.V)))          # teacher-forced
        at = {q: q.n_done for q, _ in work}
        _, lrows, erows = eng.step(work)
        torch.cuda.synchronize()
        assert eng.ctx.status_poll() == 0
        for q, n in work:
            toks = q.tokens[at[q]:at[q] + n]
            if q.kind == "gen":
                lg = ref_g[gens.index(q)].logits(toks)
                if q in lrows:
                    err = np.max(np.abs(eng.out_logits[lrows[q]].cpu().numpy() - lg))
                    worst = max(worst, err)
                    assert err <= LOGIT_ABS
            else:
                ref_e[embs.index(q)].rows(toks)
                if q in erows:
                    emb_rows[q] = eng.out_emb[erows[q]].cpu().numpy().astype(np.float64)
    for q, ref in zip(embs, ref_e):
        want = l2_normalise(ref.H.mean(axis=0) if q.pool_mode == B.POOL_MEAN else ref.H[-1])
        cos = float(emb_rows[q] @ want / np.linalg.norm(emb_rows[q]))
        assert cos >= EMB_COS and np.max(np.abs(emb_rows[q] - want)) <= EMB_ABS, cos
    print(f"\n  {shape.name}: worst logits error {worst:.2e}, launches of the last step {eng.ctx.last_launch_count()}")
    # what is in the cache is the definition's, up to neighbouring codes
    for q, ref in zip(gens, ref_g):
        for l in range(shape.L):
            for i in range(2):
                n = q.n_done
                pos = np.arange(n)
                got = eng.kv.rows(l, np.asarray(q.pages)[pos // 16], pos % 16, i).cpu().numpy().astype(np.float64)
                if i == 0:   # stored pair-interleaved inside a head
                    back = np.argsort(B.rope_pair_order(shape.Dh))
                    got = got[..., back]
                want = ref.cache[l].rows(i, np.arange((n + 15) // 16), n)
                if l == 0:   # a neighbouring code at most (the projection's fp16 rounding is far below a step)
                    assert np.all(np.abs(got - want) <= 2.0 ** -3 * np.abs(want) + 2.0 ** -7 * np.abs(want).max())
                # An input off by d (relative, root mean square) crosses a rounding border with probability d / s and
                # then moves by s, the spacing of the codes (at most 2^-3 of the value): root mean square
                # sqrt(d s).  Layer 0: d = 2^-11, the projection's rounding to fp16: 2^-7.  Layer 1: its rows
                # carry layer 0's difference, d <= 2^-7: 2^-5.
                assert np.sqrt(np.mean((got - want) ** 2)) <= (2.0 ** -7 if l == 0 else 2.0 ** -5) * np.sqrt(np.mean(want ** 2))
    eng.close()


def test_a_requests_result_does_not_depend_on_its_batch(model):
    """A prompt over several pages and decode steps, alone and among others: the same bits."""
    from paper_2609_25405_b200 import binding as B
    from paper_2609_25405_b200.engine import Request
    shape, W, dw = model
    r = np.random.default_rng(9)
    prompt, others = synth.token_ids(r, 150, shape.V), [synth.token_ids(r, n, shape.V) for n in (40, 99)]
    feed = synth.token_ids(r, 3, shape.V)
    got = []
    for crowd in (False, True):
        eng = _engine(shape, dw)
        q = Request("gen", prompt)
        e = [Request("embed", t, B.POOL_MEAN) for t in others] if crowd else []
        for step in range(5):
            work = [(q, 100 if step == 0 else 50 if step == 1 else 1)]
            work += [(x, min(x.remaining(), 30)) for x in e if x.remaining()]
            if step >= 2:
                q.tokens.append(int(feed[step - 2]))
            _, lrows, _ = eng.step(work)
            if q in lrows:
                got.append(eng.out_logits[lrows[q]].clone())
        assert eng.ctx.status_poll() == 0
        eng.close()
    assert len(got) == 8 and all(torch.equal(a, b) for a, b in zip(got[:4], got[4:]))


def test_long_context_with_splits(model):
    """Decode over 1500 tokens (several key splits) after a prompt in large chunks: the logits of the 16-bit cache up to
    the 8-bit cache's error, and the bits of a second run."""
    from paper_2609_25405_b200.engine import Engine, Request
    shape, W, dw = model
    r = np.random.default_rng(11)
    prompt = synth.token_ids(r, 1500, shape.V)
    out = {}
    for kind in ("f16", "e4m3", "e4m3 again"):
        eng = Engine(shape, dw, n_pages=200, n_slots=2, max_tokens=512, max_segs=4, max_pos=2048, kv_dtype=kind.split()[0])
        q = Request("gen", prompt)
        for n in (500, 500, 500):
            eng.step([(q, n)])
        rows = []
        for t in range(3):
            q.tokens.append(int(prompt[t]))
            _, lrows, _ = eng.step([(q, 1)])
            rows.append(eng.out_logits[lrows[q]].clone())
        assert eng.ctx.status_poll() == 0
        out[kind] = torch.stack(rows)
        eng.close()
    assert torch.equal(out["e4m3"], out["e4m3 again"])
    # keys and values move by 2^-4 at most, 2.6 % root mean square: so do the hidden states that attention adds to
    d = (out["e4m3"] - out["f16"]).double()
    rel = float(d.norm() / out["f16"].double().norm())
    print(f"\n  {shape.name}: 8-bit against 16-bit cache, logits rel {rel:.2e}, max {float(d.abs().max()):.2e}")
    assert 0 < rel <= 2.0 ** -4


def test_adapters_over_an_8_bit_cache():
    """Embedding rows with low-rank adapters next to decode rows without."""
    from paper_2609_25405_b200 import binding as B
    from paper_2609_25405_b200.engine import Request
    W = synth.Weights(TINY, 0)
    ad = synth.LoraAdapters(TINY, 16, seed=5)
    eng = _engine(TINY, B.DeviceWeights.from_synth(W), lora=B.DeviceLora.from_synth(ad))
    r = np.random.default_rng(3)
    text, prompt = synth.token_ids(r, 50, TINY.V), synth.token_ids(r, 18, TINY.V)
    e, g = Request("embed", text, B.POOL_MEAN), Request("gen", prompt)
    eng.step([(g, 18), (e, 20)])
    g.tokens.append(7)
    _, lrows, erows = eng.step([(g, 1), (e, 30)])
    assert eng.ctx.status_poll() == 0
    re, rg = Ref(TINY, W, lora=ad), Ref(TINY, W)
    re.rows(text[:20]); re.rows(text[20:])
    rg.rows(prompt)
    assert np.max(np.abs(eng.out_logits[lrows[g]].cpu().numpy() - rg.logits([7]))) <= LOGIT_ABS
    got, want = eng.out_emb[erows[e]].cpu().numpy().astype(np.float64), l2_normalise(re.H.mean(axis=0))
    assert float(got @ want) >= EMB_COS and np.max(np.abs(got - want)) <= EMB_ABS
    eng.close()


def test_logprobs_of_a_steps_logits(model):
    """Step, greedy token, its score and alternatives: the serving loop's calls one after the other."""
    from paper_2609_25405_b200.engine import Request
    shape, W, dw = model
    eng = _engine(shape, dw)
    r = np.random.default_rng(2)
    gens = [Request("gen", synth.token_ids(r, n, shape.V)) for n in (17, 40)]
    tok = torch.empty(2, dtype=torch.int32, device="cuda")
    lp, ent = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    ids, top = torch.empty(2, 5, dtype=torch.int32, device="cuda"), torch.empty(2, 5, device="cuda")
    for step in range(3):
        _, lrows, _ = eng.step([(g, g.remaining()) for g in gens])
        eng.ctx.argmax(eng.out_logits, 2, tok)
        eng.ctx.logprobs(eng.out_logits[:2], tok, lp, ent, ids, top)
        ref = torch.log_softmax(eng.out_logits[:2].double(), dim=-1)
        assert torch.equal(ids[:, 0], tok) and torch.equal(top[:, 0], lp)
        assert float((lp - ref.gather(1, tok.long()[:, None])[:, 0]).abs().max()) <= 2.0 ** -19
        assert float((ent + (ref.exp() * ref).sum(dim=-1)).abs().max()) <= 2.0 ** -17
        for g in gens:
            g.tokens.append(int(tok[lrows[g]]))
    eng.close()


def test_a_16_bit_call_refuses_an_8_bit_cache_of_another_model():
    from paper_2609_25405_b200 import binding as B
    from paper_2609_25405_b200.engine import Engine, Request
    W = synth.Weights(TINY, 0)
    dw = B.DeviceWeights.from_synth(W)
    eng = _engine(TINY, dw)
    other = B.KvCache8(B.model_cfg(TINY, 128), 8)          # another max_pos
    eng.kv, keep = other, eng.kv
    with pytest.raises(B.HbError) as e:
        eng.step([(Request("gen", [1, 2, 3]), 3)])
    assert e.value.code == -1
    eng.kv = keep
    with pytest.raises(ValueError):
        Engine(TINY, dw, 8, 1, 16, 2, 64, kv_dtype="int8")
    eng.close()
