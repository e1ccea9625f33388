"""What is measured of the operators around the 8-bit KV cache and of the scoring of logits: the cases, their
inputs, the operators in their plain form, the calls a user makes, and the definitions in 64 bits.

Operators ("op" of a case):
  append    head norms and rotation of new query / key rows, keys and values appended to the 8-bit paged cache
  attend    causal attention with grouped heads over that cache: decode rows, prompt chunks, and both mixed
  logprobs  log probability of one given token per row, entropy, and the k best alternatives

The 8-bit cache.  A block is (layer, page of 16 tokens, KV head): 16 * Dh codes (e4m3) of K, 16 * Dh of V, then
32 bytes whose first two floats are the scales of K and of V, powers of two.  A code c stands for c * scale.
  K of (token t, dim d) at byte (d / 64) * 1024 + t * 64 + d % 64
  V of (token t, dim d) at byte (d / 32) * 512 + (d % 8 * 4 + t % 8 / 2) * 16 + d % 32 / 8 * 4 + t / 8 * 2 + t % 2
The scale of a block is the smallest power of two 2^e, -32 <= e <= 24, with max |x| <= 448 * 2^e over the rows that
were appended to it; a later append to the same page may raise it, and then the codes that are there are rounded
again to the new scale.
"""
import math
import random

import torch

own = False

PAGE = 16
E_MIN, E_MAX = -32, 24
DECODE, PREFILL = 0, 1


# ---- cases -------------------------------------------------------------------------------------------------------


def listed():
    return [
        # one request decodes over a short prompt: the smallest call, latency counts
        _attend("attend-decode-1x600", 32, 8, 128, 1, 600, 600),
        # the 7B-class step's decode rows: 64 requests, contexts U[512, 4096]
        _attend("attend-decode-64-7b", 32, 8, 128, 64, 512, 4096),
        # the 1B-class step's decode rows: head dimension 64, contexts U[128, 1024]
        _attend("attend-decode-32-1b", 32, 8, 64, 32, 128, 1024),
        # few requests over very long contexts: the long axis has to be split
        _attend("attend-decode-4-long", 32, 8, 128, 4, 40000, 65536),
        # prompt chunks of 512 rows over earlier chunks, lengths that end anywhere: 7B-class prefill
        _attend("attend-chunks-7b", 32, 8, 128, 0, 0, 0, 8, 257, 512, 0, 2048),
        # a mixed step: decode rows and prompt / embedding chunks together
        _attend("attend-mixed-7b", 32, 8, 128, 64, 512, 4096, 6, 33, 512, 0, 1024),
        # the append of 64 decode rows: one new token in each request's page
        _append("append-decode-64-7b", 32, 8, 128, 64, 512, 4096, rot=128, layout="pairs", norm=False),
        # the append of a whole 4096-row step of prompt chunks, with head norms and the half layout
        _append("append-chunks-7b", 32, 8, 128, 0, 0, 0, 8, 512, 512, 0, 2048, rot=128, layout="halves", norm=True),
        # scoring the 64 decode rows of a 7B-class step with 20 alternatives
        _logprobs("logprobs-64x32000", 64, 32000, 20, "float32"),
        # one row over the 1B-class vocabulary
        _logprobs("logprobs-1x128256", 1, 128256, 5, "float32"),
        # a decode-heavy step over the 1B-class vocabulary
        _logprobs("logprobs-400x128256", 400, 128256, 20, "float32"),
        # scoring a whole prompt: 16-bit logits, no alternatives
        _logprobs("logprobs-2048x32000-f16", 2048, 32000, 0, "float16"),
    ]


def _attend(name, hq, hkv, dh, n_dec, ctx_lo, ctx_hi, n_chunk=0, q_lo=0, q_hi=0, past_lo=0, past_hi=0, lens=1):
    return dict(name=name, op="attend", hq=hq, hkv=hkv, dh=dh, n_dec=n_dec, ctx_lo=ctx_lo, ctx_hi=ctx_hi, n_chunk=n_chunk,
                q_lo=q_lo, q_hi=q_hi, past_lo=past_lo, past_hi=past_hi, lens=lens)


def _append(name, hq, hkv, dh, n_dec, ctx_lo, ctx_hi, n_chunk=0, q_lo=0, q_hi=0, past_lo=0, past_hi=0, lens=1, rot=128,
            layout="pairs", norm=False):
    c = _attend(name, hq, hkv, dh, n_dec, ctx_lo, ctx_hi, n_chunk, q_lo, q_hi, past_lo, past_hi, lens)
    return dict(c, op="append", rot=rot, layout=layout, norm=norm)


def _logprobs(name, rows, vocab, k, dtype):
    return dict(name=name, op="logprobs", rows=rows, vocab=vocab, k=k, dtype=dtype)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attend", "attend", "append", "logprobs"))
    if op == "logprobs":
        vocab = _log_int(rng, 100, 130000)
        rows = _log_int(rng, 1, max(2, min(2048, 40000000 // vocab)))
        return {k: v for k, v in _logprobs("", rows, vocab, min(rng.choice((0, 1, 5, 20, 32)), vocab),
                                           rng.choice(("float32", "float16"))).items() if k != "name"}
    dh = rng.choice((64, 128))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 4, 8, 16)) if hkv < 8 else hkv * rng.choice((1, 2, 4))
    n_dec = n_chunk = ctx_hi = q_hi = past_hi = 0
    kind = rng.choice(("decode", "chunks", "mixed"))
    if kind != "chunks":
        ctx_hi = _log_int(rng, 1, 40000 if kind == "decode" else 4096)
        n_dec = _log_int(rng, 1, max(1, min(96, 200000 // ctx_hi)))
    if kind != "decode":
        n_chunk = rng.randint(1, 6)
        q_hi = _log_int(rng, 2, 512)
        past_hi = rng.choice((0, _log_int(rng, 1, 1500)))
    c = _attend("", hq, hkv, dh, n_dec, max(1, ctx_hi // 4) if n_dec else 0, ctx_hi, n_chunk, max(1, q_hi // 3) if n_chunk else 0,
                q_hi, 0, past_hi, rng.randrange(1 << 20))
    if op == "append":
        c = dict(c, op="append", rot=rng.choice((dh, dh // 2, dh // 4)), layout=rng.choice(("pairs", "halves")),
                 norm=rng.choice((True, False)))
    return {k: v for k, v in c.items() if k != "name"}


def _segments(case):
    """[(tokens already cached, new rows, kind)]: decode rows first, then chunks."""
    r = random.Random(case["lens"])
    segs = [(r.randint(case["ctx_lo"], case["ctx_hi"]), 1, DECODE) for _ in range(case["n_dec"])]
    return segs + [(r.randint(case["past_lo"], case["past_hi"]), r.randint(case["q_lo"], case["q_hi"]), PREFILL)
                   for _ in range(case["n_chunk"])]


def work(case):
    if case["op"] == "logprobs":
        n, v, k = case["rows"], case["vocab"], case["k"]
        size = 4 if case["dtype"] == "float32" else 2
        # per logit: subtract, exp, two additions and a product for the entropy, a comparison
        return {"bytes": n * v * size + n * (4 + 8 + 8 * k), "flops": 6 * n * v}
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    segs = _segments(case)
    rows = sum(q for _, q, _ in segs)
    if case["op"] == "append":
        # qkv in, q out (16 bits), k and v out (8 bits), two scales a block, tables and gains
        blocks = sum((p + q + PAGE - 1) // PAGE - p // PAGE for p, q, _ in segs) * hkv
        byte = rows * ((hq + 2 * hkv) * dh * 2 + hq * dh * 2 + 2 * hkv * dh + case["rot"] * 4) + blocks * 8
        return {"bytes": byte, "flops": rows * ((hq + hkv) * (case["rot"] * 3 + (dh * 4 if case["norm"] else 0)) + 2 * hkv * dh * 2)}
    # the cache once for each request (8 bits and two scales a block), q in and the output out
    keys = sum(p + q for p, q, _ in segs)
    blocks = sum((p + q + PAGE - 1) // PAGE for p, q, _ in segs)
    pairs = sum(q * p + q * (q + 1) // 2 for p, q, _ in segs)
    return {"bytes": keys * hkv * 2 * dh + blocks * (hkv * 8 + 4) + rows * hq * dh * 4, "flops": 4 * dh * hq * pairs}


# ---- inputs ------------------------------------------------------------------------------------------------------


def _exponent(amax):
    """Smallest e with amax <= 448 * 2^e, clamped; float32 tensor -> int32 tensor."""
    m, p = torch.frexp(amax)   # amax = m * 2^p, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = p - 9 + (m > 0.875).to(p.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _pow2(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _views(arena, n_pages, hkv, dh):
    """(codes [page, head, 32 * Dh] float8, scales [page, head, 2] float32) of a one-layer arena."""
    a = arena.view(n_pages, hkv, 32 * dh + 32)
    return a[..., :32 * dh].view(torch.float8_e4m3fn), a[..., 32 * dh:32 * dh + 8].view(torch.float32)


def _k_codes(codes, dh):
    """K codes as [page, head, 16, Dh] (a copy)."""
    k = codes[..., :16 * dh].unflatten(-1, (dh // 64, 16, 64))
    return k.transpose(-3, -2).flatten(-2)


def _v_codes(codes, dh):
    """V codes as [page, head, 16, Dh] (a copy): stored [Dh/32][d % 8][t % 8 / 2][d % 32 / 8][t / 8][t % 2]."""
    v = codes[..., 16 * dh:].unflatten(-1, (dh // 32, 8, 4, 4, 2, 2))
    # -> page, head, (t/8, t%8/2, t%2), (d/32, d%32/8, d%8)
    return v.permute(0, 1, 6, 4, 7, 2, 5, 3).reshape(*codes.shape[:2], 16, dh)


def _store_k(codes, k, dh):
    codes[..., :16 * dh] = k.unflatten(-1, (dh // 64, 64)).transpose(-3, -2).flatten(-3)


def _store_v(codes, v, dh):
    # page, head, t/8, t%8/2, t%2, d/32, d%32/8, d%8
    v = v.unflatten(-1, (dh // 32, 4, 8)).unflatten(2, (2, 4, 2))
    codes[..., 16 * dh:] = v.permute(0, 1, 5, 7, 3, 6, 2, 4).flatten(2)


_contexts = {}


def _context(case):
    """The program's context for this geometry, opened once."""
    from paper_2609_25405_b200 import binding as B
    from paper_2609_25405_b200 import synth
    key = (case.get("hq", 1), case.get("hkv", 1), case.get("dh", 64))
    if key not in _contexts:
        cfg = B.model_cfg(synth.ModelShape("ops", 1, 64, key[0], key[1], key[2], 64, 64), 65552)
        _contexts[key] = (cfg, B.Context(cfg, 1, 1, 1))
    return _contexts[key]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    st = {"case": case}
    if case["op"] == "logprobs":
        n, v = case["rows"], case["vocab"]
        # logits of a language model: most mass on few tokens, rows of different sharpness
        x = torch.randn(n, v, generator=g, device=dev) * (1.0 + 2.0 * torch.rand(n, 1, generator=g, device=dev))
        st["logits"] = x.to(getattr(torch, case["dtype"]))
        st["tokens"] = torch.randint(v, (n,), generator=g, device=dev, dtype=torch.int32)
        st["out"] = (torch.empty(n, device=dev), torch.empty(n, device=dev))
        st["top"] = (torch.empty(n, case["k"], device=dev, dtype=torch.int32), torch.empty(n, case["k"], device=dev))
        if own:
            st["ctx"] = _context(case)[1]
        return st
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    segs = _segments(case)
    need = [(p + q + PAGE - 1) // PAGE for p, q, _ in segs]
    n_pages = sum(need) + 3
    T = sum(q for _, q, _ in segs)
    st["page_ids"] = torch.randperm(n_pages, generator=g, device=dev)[:sum(need)].to(torch.int32)
    rows, row_seg, q_at, pt_at = [], [], 0, 0
    for i, (p, q, kind) in enumerate(segs):
        rows.append([kind, q_at, q, p, pt_at, need[i], -1, 0, 1, -1, -1, 0])
        row_seg += [i] * q
        q_at += q
        pt_at += need[i]
    st["segs"] = torch.tensor(rows, dtype=torch.int32).to(dev)
    st["row_seg"] = torch.tensor(row_seg, dtype=torch.int32).to(dev)
    st["lens"] = [(p, q) for p, q, _ in segs]
    # the cache as appends have left it: keys and values around 1, channels with an offset of their own
    arena = torch.zeros(n_pages * hkv * (32 * dh + 32), dtype=torch.uint8, device=dev)
    codes, scales = _views(arena, n_pages, hkv, dh)
    for which, store in ((0, _store_k), (1, _store_v)):
        x = torch.randn(n_pages, hkv, 16, dh, generator=g, device=dev) + 0.5 * torch.randn(hkv, 1, dh, generator=g, device=dev)
        s = _pow2(_exponent(x.abs().amax(dim=(2, 3))))
        store(codes, (x / s[..., None, None]).to(torch.float8_e4m3fn), dh)
        scales[..., which] = s
        del x
    st["arena"], st["n_pages"] = arena, n_pages
    if case["op"] == "attend":
        st["q"] = torch.randn(T, hq * dh, generator=g, device=dev).half()
        st["out"] = torch.empty(T, hq * dh, device=dev, dtype=torch.float16)
    else:
        st["qkv"] = torch.randn(T, (hq + 2 * hkv) * dh, generator=g, device=dev).half()
        st["out"] = torch.empty(T, hq * dh, device=dev, dtype=torch.float16)
        top = max(p + q for p, q in st["lens"])
        half = case["rot"] // 2
        ang = torch.arange(top, dtype=torch.float64, device=dev)[:, None] * torch.pow(
            torch.tensor(1e4, dtype=torch.float64, device=dev), -torch.arange(half, dtype=torch.float64, device=dev) / half)
        st["cos"], st["sin"] = ang.cos().float(), ang.sin().float()
        st["gain"] = [(1 + 0.1 * torch.randn(dh, generator=g, device=dev)).bfloat16() for _ in range(2)] if case["norm"] else [None] * 2
    if own:
        from paper_2609_25405_b200 import binding as B
        cfg, st["ctx"] = _context(case)
        st["kv"] = B.KvCache8(cfg, n_pages, arena=arena)
        st["rows"] = B.SegRows(st["segs"], st["page_ids"], st["row_seg"], max_q_len=max(q for _, q in st["lens"]),
                               max_keys=max(p + q for p, q in st["lens"]))
        if case["op"] == "append":
            st["rope"] = B.Rope(st["cos"], st["sin"], B.ROPE_PAIRS if case["layout"] == "pairs" else B.ROPE_HALVES)
    return st


def run(st):
    return {"attend": _run_attend, "append": _run_append, "logprobs": _run_logprobs}[st["case"]["op"]](st)


# ---- attend ------------------------------------------------------------------------------------------------------


def _run_attend(st):
    if own:
        st["ctx"].kv8_attention(st["kv"], 0, st["rows"], st["q"], st["out"])
        return st["out"]
    n = st["case"]["n_dec"]
    if n:
        _plain_attend(st, 0, n, st["lens"][:n])
    if len(st["lens"]) > n:
        _plain_attend(st, n, len(st["lens"]), st["lens"][n:])
    return st["out"]


def _plain_attend(st, lo, hi, lens):
    """Segments lo .. hi, padded to their longest: gather pages, dequantise, softmax, weighted sum, in 32 bits."""
    hq, hkv, dh = (st["case"][n] for n in ("hq", "hkv", "dh"))
    dev = st["q"].device
    segs = st["segs"][lo:hi].long()
    max_q, max_k = max(q for _, q in lens), max(p + q for p, q in lens)
    n_pg = (max_k + PAGE - 1) // PAGE
    codes, scales = _views(st["arena"], st["n_pages"], hkv, dh)
    at = segs[:, 4, None] + torch.arange(n_pg, device=dev).minimum(segs[:, 5, None] - 1)
    pages = st["page_ids"].long()[at]                                            # [R, n_pg]
    j = torch.arange(max_q, device=dev)
    rows = (segs[:, 1, None] + j).clamp(max=st["q"].shape[0] - 1)                # [R, max_q]
    q = st["q"][rows].float().view(hi - lo, max_q, hkv, hq // hkv, dh)
    flat = pages.flatten()
    k = (_k_codes(codes[flat], dh).float() * scales[flat][..., 0, None, None]).view(hi - lo, n_pg, hkv, PAGE, dh)
    k = k.permute(0, 2, 1, 3, 4).reshape(hi - lo, hkv, n_pg * PAGE, dh)
    s = torch.einsum("rjhgd,rhkd->rhgjk", q, k) / math.sqrt(dh)
    del k
    seen = torch.arange(n_pg * PAGE, device=dev) <= segs[:, 3, None, None] + j[:, None]      # [R, max_q, keys]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    s = torch.exp(s - s.amax(dim=-1, keepdim=True))
    total = s.sum(dim=-1)
    v = (_v_codes(codes[flat], dh).float() * scales[flat][..., 1, None, None]).view(hi - lo, n_pg, hkv, PAGE, dh)
    v = v.permute(0, 2, 1, 3, 4).reshape(hi - lo, hkv, n_pg * PAGE, dh)
    o = torch.einsum("rhgjk,rhkd->rjhgd", s, v) / total.permute(0, 3, 1, 2)[..., None]
    valid = j < segs[:, 2, None]
    st["out"][rows[valid]] = o.reshape(hi - lo, max_q, hq * dh)[valid].half()


def _exact_attend(st):
    hq, hkv, dh = (st["case"][n] for n in ("hq", "hkv", "dh"))
    dev = st["q"].device
    arena = st["arena"].view(st["n_pages"], hkv, 32 * dh + 32)
    d, t = torch.arange(dh, device=dev)[None, :], torch.arange(PAGE, device=dev)[:, None]
    k_at = (d // 64 * 1024 + t * 64 + d % 64).flatten()
    v_at = (16 * dh + d // 32 * 512 + (d % 8 * 4 + t % 8 // 2) * 16 + d % 32 // 8 * 4 + t // 8 * 2 + t % 2).flatten()
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=dev)
    for p, n, at, pt in [(p, n, int(r[1]), int(r[4])) for (p, n), r in zip(st["lens"], st["segs"].tolist())]:
        ids = st["page_ids"][pt:pt + (p + n + PAGE - 1) // PAGE].long()
        blk = arena[ids]                                                        # [pages, head, bytes]
        sc = blk[..., 32 * dh:32 * dh + 8].contiguous().view(torch.float32).double()
        get = lambda where, s: (blk[..., where].contiguous().view(torch.float8_e4m3fn).double().view(len(ids), hkv, PAGE, dh) *  # noqa: E731
                                s[..., None, None]).transpose(0, 1).reshape(hkv, len(ids) * PAGE, dh)[:, :p + n]
        k, v = get(k_at, sc[..., 0]), get(v_at, sc[..., 1])
        q = st["q"][at:at + n].double().view(n, hkv, hq // hkv, dh)
        for h in range(hkv):
            x = (q[:, h].reshape(-1, dh) @ k[h].T).view(n, hq // hkv, p + n) * dh ** -0.5
            hide = torch.ones(n, p + n, dtype=torch.bool, device=dev).triu(p + 1)
            w = torch.softmax(x.masked_fill(hide[:, None], -math.inf), dim=-1)
            out[at:at + n].view(n, hkv, hq // hkv, dh)[:, h] = w @ v[h]
    return out


# ---- append ------------------------------------------------------------------------------------------------------


def _run_append(st):
    case = st["case"]
    if own:
        st["ctx"].kv8_append(st["kv"], 0, st["rows"], st["qkv"], st["out"], rope=st["rope"], q_norm=st["gain"][0],
                             k_norm=st["gain"][1], norm_eps=1e-6)
    else:
        _plain_append(st)
    codes, scales = _views(st["arena"], st["n_pages"], case["hkv"], case["dh"])
    return {"q": st["out"], "codes": codes, "scales": scales}


def _rotate(x, cos, sin, layout):
    """x [T, H, Dh], tables [T, rot / 2]: the first rot dimensions turn, the rest stay."""
    half = cos.shape[-1]
    c, s = cos[:, None], sin[:, None]
    if layout == "pairs":
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    return torch.cat((y, x[..., 2 * half:]), dim=-1)


def _normed(x, gain):
    return x if gain is None else x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + 1e-6) * gain.to(x.dtype)


def _plain_append(st):
    case = st["case"]
    hq, hkv, dh = (case[n] for n in ("hq", "hkv", "dh"))
    T, n_pages, dev = st["qkv"].shape[0], st["n_pages"], st["qkv"].device
    seg = st["segs"].long()[st["row_seg"].long()]
    pos = seg[:, 3] + torch.arange(T, device=dev) - seg[:, 1]
    page, slot = st["page_ids"].long()[seg[:, 4] + pos // PAGE], pos % PAGE
    x = st["qkv"].float().view(T, hq + 2 * hkv, dh)
    cos, sin = st["cos"][pos], st["sin"][pos]
    st["out"].copy_(_rotate(_normed(x[:, :hq], st["gain"][0]), cos, sin, case["layout"]).reshape(T, hq * dh))
    k = _rotate(_normed(x[:, hq:hq + hkv], st["gain"][1]), cos, sin, case["layout"])
    # the pages that get rows, and the first slot that each of them gets
    touched, page = torch.unique(page, return_inverse=True)
    first = torch.full(touched.shape, PAGE, device=dev).scatter_reduce_(0, page, slot, "amin")
    arena = st["arena"].view(n_pages, -1)
    part = arena[touched]
    codes, scales = _views(part, len(touched), hkv, dh)
    _plain_store(codes, scales, 0, k, _k_codes, _store_k, page, slot, first, dh)
    _plain_store(codes, scales, 1, x[:, hq + hkv:], _v_codes, _store_v, page, slot, first, dh)
    arena[touched] = part


def _plain_store(codes, scales, which, x, load, store, page, slot, first, dh):
    new = torch.zeros_like(scales[..., which]).index_reduce_(0, page, x.abs().amax(dim=-1), "amax")
    old = torch.frexp(scales[..., which])[1] - 1
    fresh = (first == 0)[:, None]
    e = torch.where(fresh, _exponent(new), torch.maximum(old, _exponent(new)))
    # what is there, under the new scale; a page that starts afresh is zero
    val = load(codes, dh).float() * torch.where(fresh, 0.0, _pow2(old - e))[..., None, None]
    val[page, :, slot] = x / _pow2(e)[page][..., None]
    store(codes, val.to(torch.float8_e4m3fn), dh)
    scales[..., which] = _pow2(e)


def _e4m3(x):
    """Nearest e4m3 value of x (|x| <= 448), ties to even, in 64 bits."""
    p = torch.frexp(x)[1].clamp(min=-5) - 1            # 2^p <= |x| < 2^(p+1); below 2^-6 the spacing stays 2^-9
    step = torch.ldexp(torch.ones_like(x), p - 3)
    return torch.round(x / step) * step


def _exact_append(st):
    case = st["case"]
    hq, hkv, dh = (case[n] for n in ("hq", "hkv", "dh"))
    dev, half, rot = st["qkv"].device, case["rot"] // 2, case["rot"]
    arena = st["arena"].view(st["n_pages"], hkv, 32 * dh + 32)
    codes = arena[..., :32 * dh].contiguous().view(torch.float8_e4m3fn).double()
    scales = arena[..., 32 * dh:32 * dh + 8].contiguous().view(torch.float32).double()
    d, t = torch.arange(dh, device=dev)[None, :], torch.arange(PAGE, device=dev)[:, None]
    at = [d // 64 * 1024 + t * 64 + d % 64,
          16 * dh + d // 32 * 512 + (d % 8 * 4 + t % 8 // 2) * 16 + d % 32 // 8 * 4 + t // 8 * 2 + t % 2]
    i = torch.arange(half, device=dev)
    a_at, b_at = (2 * i, 2 * i + 1) if case["layout"] == "pairs" else (i, i + half)
    q_out = []
    for (p, n), r in zip(st["lens"], st["segs"].tolist()):
        x = st["qkv"][r[1]:r[1] + n].double().view(n, hq + 2 * hkv, dh).clone()
        if case["norm"]:
            rms = (x[:, :hq + hkv].pow(2).sum(-1, keepdim=True) / dh + 1e-6).sqrt()
            x[:, :hq + hkv] /= rms
            x[:, :hq] *= st["gain"][0].double()
            x[:, hq:hq + hkv] *= st["gain"][1].double()
        c, s = st["cos"][p:p + n].double()[:, None], st["sin"][p:p + n].double()[:, None]
        a, b = x[:, :hq + hkv, a_at].clone(), x[:, :hq + hkv, b_at].clone()
        x[:, :hq + hkv, a_at] = a * c - b * s
        x[:, :hq + hkv, b_at] = a * s + b * c
        q_out.append(x[:, :hq].reshape(n, hq * dh))
        for pg in range(p // PAGE, (p + n - 1) // PAGE + 1):
            page = int(st["page_ids"][r[4] + pg])
            lo, hi = max(p, pg * PAGE), min(p + n, pg * PAGE + PAGE)
            for which in range(2):
                y = x[lo - p:hi - p, hq + which * hkv:hq + (which + 1) * hkv].transpose(0, 1)       # [head, new, Dh]
                top = y.abs().amax(dim=(1, 2))
                e = torch.ceil(torch.log2(top / 448.0)).clamp(E_MIN, E_MAX)
                e = torch.where(torch.ldexp(torch.full_like(e, 448.0), e - 1) >= top, e - 1, e).clamp(E_MIN, E_MAX)
                s_new = torch.exp2(e)
                blk = codes[page][:, at[which].flatten()].view(hkv, PAGE, dh)
                if lo > pg * PAGE:
                    s_new = torch.maximum(s_new, scales[page, :, which])
                    blk = _e4m3(blk * (scales[page, :, which] / s_new)[:, None, None])
                else:
                    blk = torch.zeros_like(blk)
                blk[:, lo - pg * PAGE:hi - pg * PAGE] = _e4m3(y / s_new[:, None, None])
                codes[page][:, at[which].flatten()] = blk.view(hkv, -1)
                scales[page, :, which] = s_new
    return {"q": torch.cat(q_out), "codes": codes, "scales": scales}


# ---- logprobs ----------------------------------------------------------------------------------------------------


def _run_logprobs(st):
    k = st["case"]["k"]
    if own:
        st["ctx"].logprobs(st["logits"], st["tokens"], *st["out"], *(st["top"] if k else ()))
        return st["out"] + st["top"]
    x = st["logits"].float()
    top, ids = x.max(dim=-1, keepdim=True)[0], None
    z = x - top
    e = torch.exp(z)
    total = e.sum(dim=-1)
    log_total = torch.log(total)
    given = z.gather(1, st["tokens"].long()[:, None])[:, 0] - log_total
    entropy = log_total - (e * z).sum(dim=-1) / total
    best, ids = torch.sort(z, dim=-1, descending=True, stable=True)   # equal logits: the lower token first
    return (given, entropy, ids[:, :k].to(torch.int32), best[:, :k] - log_total[:, None])


def _exact_logprobs(st):
    x, k = st["logits"].double(), st["case"]["k"]
    logp = torch.log_softmax(x, dim=-1)
    v = torch.arange(x.shape[1], device=x.device)
    ids, left = [], x.clone()
    for _ in range(k):
        best = left.amax(dim=-1, keepdim=True)
        i = torch.where(left == best, v, x.shape[1]).amin(dim=-1, keepdim=True)
        ids.append(i)
        left.scatter_(1, i, -math.inf)
    ids = torch.cat(ids, dim=1) if k else torch.empty(x.shape[0], 0, dtype=torch.int64, device=x.device)
    return (logp.gather(1, st["tokens"].long()[:, None])[:, 0], -(logp.exp() * logp).sum(dim=-1), ids.to(torch.int32), logp.gather(1, ids))


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"attend": _exact_attend, "append": _exact_append, "logprobs": _exact_logprobs}[case["op"]](st)
