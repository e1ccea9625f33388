"""What is measured of the dense operators: the cases, their inputs, the operators in their plain form, the calls a user
makes, and the definitions in 64 bits.

Operators ("op" of a case):
  norm     residual addition, root-mean-square norm and gain in one pass; 16 or 32 bits out, or 8 bits with a scale per row
  quant    rows to 8 bits with a scale per row, in order or gathered by an index
  linear   C = act((a_scale w_scale) A W^T + bias) + residual, A and W in 8 bits (with scales) or 16
  grouped  the same where each run of rows has a W of its own: experts, or one adapter per request

8 bits are e4m3 codes; a row's scale is its largest magnitude / 448, and a code c of the row stands for c * scale.
"gated": the rows of W come in pairs (gate, up), and C = act(gate) * up has half as many columns.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


# ---- cases -------------------------------------------------------------------------------------------------------


def listed():
    return [
        # one decode row of the 7B-class model before a projection: the smallest call, latency counts
        _norm("norm-1x4096-e4m3", 1, 4096, "f16", "f32", "e4m3"),
        # a whole 4096-row step of the 7B-class model: the norm before its 8-bit projections
        _norm("norm-4096x4096-e4m3", 4096, 4096, "f16", "f32", "e4m3"),
        # attention output of a 7B-class step's 64 decode rows, before the 8-bit output projection
        _quant("quant-64x4096", 64, 4096, "f16", 0),
        # inner activations of a whole step, gathered into another order (rows by expert)
        _quant("quant-4096x14336-gather", 4096, 14336, "f16", 1),
        # QKV projection with bias of one decode row, 8 bits
        _linear("linear-1x6144x4096-e4m3", 1, 6144, 4096, "e4m3", "f16", bias=True),
        # gate/up projection of 64 decode rows, 8 bits
        _linear("linear-64x28672x4096-e4m3-silu", 64, 28672, 4096, "e4m3", "f16", act="silu", gated=True),
        # the same of a whole 4096-row step: the largest
        _linear("linear-4096x28672x4096-e4m3-silu", 4096, 28672, 4096, "e4m3", "f16", act="silu", gated=True),
        # output projection of a 1B-class step onto the fp32 residual stream, 16 bits
        _linear("linear-2048x2048x2048-f16-res", 2048, 2048, 2048, "f16", "f32", residual="f32"),
        # an encoder's feed-forward layer, odd sizes, bf16 with bias and GELU
        _linear("linear-777x4100x1030-bf16-gelu", 777, 4100, 1030, "bf16", "bf16", act="gelu", bias=True),
        # 32 decode rows, two of eight experts each: gate/up, 8 bits
        _grouped("grouped-64x28672x4096-8-e4m3-silu", 64, 28672, 4096, 8, "e4m3", "f16", act="silu", gated=True, lens=1),
        # a 2048-row step, two of sixteen experts each, down projection, 8 bits
        _grouped("grouped-4096x2048x8192-16-e4m3", 4096, 2048, 8192, 16, "e4m3", "f16", lens=2),
        # up factors of 24 adapters of rank 64, added to the residual stream of a 4096-row step
        _grouped("grouped-4096x4096x64-24-f16-res", 4096, 4096, 64, 24, "f16", "f32", residual="f32", lens=3),
    ]


def _norm(name, rows, d, x, residual, out, gain=True):
    return dict(name=name, op="norm", rows=rows, d=d, x=x, residual=residual, out=out, gain=gain)


def _quant(name, rows, d, x, gather):
    return dict(name=name, op="quant", rows=rows, d=d, x=x, gather=gather)


def _linear(name, m, n, k, ab, out, act="none", gated=False, bias=False, residual=""):
    return dict(name=name, op="linear", m=m, n=n, k=k, ab=ab, out=out, act=act, gated=gated, bias=bias, residual=residual)


def _grouped(name, m, n, k, groups, ab, out, act="none", gated=False, bias=False, residual="", lens=1):
    return dict(_linear(name, m, n, k, ab, out, act, gated, bias, residual), op="grouped", groups=groups, lens=lens)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "quant", "linear", "linear", "grouped", "grouped"))
    if op == "norm":
        d = _log_int(rng, 8, 16384)
        c = _norm("", _log_int(rng, 1, min(8192, (1 << 24) // d)), d, rng.choice(("f32", "f16", "bf16")),
                  rng.choice(("", "f32", "f32", "f16", "bf16")), rng.choice(("e4m3", "e4m3", "f16", "bf16")), rng.random() < 0.8)
    elif op == "quant":
        d = _log_int(rng, 8, 16384)
        c = _quant("", _log_int(rng, 1, min(8192, (1 << 25) // d)), d, rng.choice(("f32", "f16", "bf16")), rng.randrange(2))
    else:
        ab = rng.choice(("e4m3", "e4m3", "f16", "bf16"))
        act = rng.choice(ACTS)
        gated = act != "none" and rng.random() < 0.5
        out = rng.choice(("f16", "bf16", "f32") if ab == "e4m3" else (ab, "f32"))
        args = dict(act=act, gated=gated, bias=rng.random() < 0.5, residual=rng.choice(("", "", out, "f32")))
        groups = rng.randint(1, 32) if op == "grouped" else 1
        n, k = _log_int(rng, 16, 28672), _log_int(rng, 16, 14336)
        if n * k * groups > 1 << 29:
            n = max(16, (1 << 29) // (k * groups))
        n += n % 2 if gated else 0
        m = _log_int(rng, 1, max(2, min(8192, (1 << 38) // (n * k))))
        if op == "linear":
            c = _linear("", m, n, k, ab, out, **args)
        else:
            c = _grouped("", m, n, k, groups, ab, out, lens=rng.randrange(1 << 20), **args)
    return {k: v for k, v in c.items() if k != "name"}


def _counts(case):
    """Rows of each group: uneven, and some groups without any."""
    if case["op"] == "linear":
        return [case["m"]]
    r = random.Random(case["lens"])
    share = [r.expovariate(1.0) for _ in range(case["groups"])]
    at = r.choices(range(case["groups"]), share, k=case["m"])
    return [at.count(e) for e in range(case["groups"])]


def _size(t):
    return {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1, "": 0}[t]


def work(case):
    if case["op"] == "norm":
        n = case["rows"] * case["d"]
        byte = n * (_size(case["x"]) + 2 * _size(case["residual"]) + _size(case["out"])) + (case["d"] * 2 if case["gain"] else 0)
        return {"bytes": byte + (case["rows"] * 4 if case["out"] == "e4m3" else 0), "flops": n * 6}
    if case["op"] == "quant":
        n = case["rows"] * case["d"]
        return {"bytes": n * (_size(case["x"]) + 1) + case["rows"] * (4 + 4 * case["gather"]), "flops": n * 3}
    m, n, k, ab = case["m"], case["n"], case["k"], _size(case["ab"])
    counts = _counts(case)
    cols = n // 2 if case["gated"] else n
    used = sum(c > 0 for c in counts)
    byte = m * k * ab + used * n * k * ab + m * cols * (_size(case["out"]) + _size(case["residual"]))
    byte += (m * 4 + used * n * 4 if case["ab"] == "e4m3" else 0) + (used * n * 4 if case["bias"] else 0) + 4 * len(counts)
    return {"bytes": byte, "flops": 2 * m * n * k}


# ---- inputs ------------------------------------------------------------------------------------------------------


_contexts = []


def _context():
    """The program's context, opened once."""
    from paper_2609_25405_b200 import binding as B
    from paper_2609_25405_b200 import synth
    if not _contexts:
        cfg = B.model_cfg(synth.ModelShape("ops", 1, 64, 1, 1, 64, 64, 64), 64)
        _contexts.append(B.Context(cfg, 1, 1, 1))
    return _contexts[0]


def _matrix(g, rows, cols, kind, std=1.0):
    """A matrix whose rows start on 16-byte boundaries, and the scales of its rows (8 bits) or None."""
    dev, step = torch.device("cuda"), 16 // _size(kind)
    x = torch.empty(rows, (cols + step - 1) // step * step, device=dev, dtype=TYPES[kind])[:, :cols]
    if kind != "e4m3":
        x.copy_(torch.empty(rows, cols, device=dev, dtype=TYPES[kind]).normal_(0.0, std, generator=g))
        return x, None
    part = max(1, (1 << 26) // cols)   # rows at a time, for the 16-bit values in between
    for i in range(0, rows, part):
        v = torch.empty(min(part, rows - i), cols, device=dev, dtype=torch.float16).normal_(0.0, 110.0, generator=g)
        x[i:i + part] = v.clamp_(-448, 448).to(torch.float8_e4m3fn)
    return x, std / 110 * (0.75 + 0.5 * torch.rand(rows, generator=g, device=dev))


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    st = {"case": case}
    if own:
        st["ctx"] = _context()
    if case["op"] in ("norm", "quant"):
        rows, d = case["rows"], case["d"]
        # a few channels are far larger than the others, as in a residual stream
        wide = 1 + 20 * (torch.rand(d, generator=g, device=dev) < 0.002).float()
        st["x"] = (torch.randn(rows, d, generator=g, device=dev) * wide).to(TYPES[case["x"]])
        out = case.get("out", "e4m3")
        st["y"] = torch.empty(rows, d, device=dev, dtype=TYPES[out])
        st["scale"] = torch.empty(rows, device=dev) if out == "e4m3" else None
        if case["op"] == "quant":
            st["index"] = torch.randperm(rows, generator=g, device=dev).to(torch.int32) if case["gather"] else None
            return st
        st["residual"] = st["sum"] = None
        if case["residual"]:
            st["residual"] = (2 * torch.randn(rows, d, generator=g, device=dev) * wide).to(TYPES[case["residual"]])
            st["sum"] = torch.empty_like(st["residual"])
        st["gain"] = (1 + 0.1 * torch.randn(d, generator=g, device=dev)).bfloat16() if case["gain"] else None
        return st
    m, n, k = case["m"], case["n"], case["k"]
    counts = _counts(case)
    st["a"], st["a_scale"] = _matrix(g, m, k, case["ab"])
    w, s = _matrix(g, n * len(counts), k, case["ab"], 0.02)
    cols = n // 2 if case["gated"] else n
    out = TYPES[case["out"]]
    if case["op"] == "grouped":
        w, s = w.unflatten(0, (len(counts), n)), None if s is None else s.view(len(counts), n)
        ends = [sum(counts[:e]) for e in range(len(counts) + 1)]
        st["start"] = torch.tensor(ends, dtype=torch.int32).to(dev)
        st["most"] = max(counts)
    st["w"], st["w_scale"] = w, s
    st["bias"] = torch.randn(w.shape[:-1], generator=g, device=dev) * 0.5 if case["bias"] else None
    st["residual"] = (2 * torch.randn(m, cols, generator=g, device=dev)).to(TYPES[case["residual"]]) if case["residual"] else None
    st["out"] = torch.empty(m, cols, device=dev, dtype=out)
    if own:
        from paper_2609_25405_b200 import binding as B
        st["act"] = getattr(B, "ACT_" + case["act"].upper())
    return st


def run(st):
    return {"norm": _run_norm, "quant": _run_quant, "linear": _run_linear, "grouped": _run_grouped}[st["case"]["op"]](st)


# ---- norm, quant -------------------------------------------------------------------------------------------------


def _codes(y):
    """(codes, scales) of fp32 rows."""
    scale = y.abs().amax(dim=-1) / 448
    return (y / scale[:, None]).to(torch.float8_e4m3fn), scale


def _run_norm(st):
    if own:
        st["ctx"].norm(st["x"], st["gain"], st["y"], residual=st["residual"], sum_out=st["sum"], y_scale=st["scale"], eps=1e-5)
        return {"y": st["y"], "scale": st["scale"], "sum": st["sum"]}
    s, total = st["x"].float(), None
    if st["residual"] is not None:
        s = s + st["residual"].float()
        total = s.to(st["residual"].dtype)
    y = s * torch.rsqrt(s.square().mean(dim=-1, keepdim=True) + 1e-5)
    if st["gain"] is not None:
        y = y * st["gain"].float()
    if st["scale"] is None:
        return {"y": y.to(st["y"].dtype), "scale": None, "sum": total}
    y, scale = _codes(y)
    return {"y": y, "scale": scale, "sum": total}


def _run_quant(st):
    if own:
        st["ctx"].quant_rows(st["x"], st["y"], st["scale"], index=st["index"])
        return {"y": st["y"], "scale": st["scale"]}
    x = st["x"].float()
    y, scale = _codes(x if st["index"] is None else x[st["index"].long()])
    return {"y": y, "scale": scale}


def _e4m3(x):
    """Nearest e4m3 value of x (|x| <= 448), ties to even, in 64 bits."""
    p = torch.frexp(x)[1].clamp(min=-5) - 1            # 2^p <= |x| < 2^(p+1); below 2^-6 the spacing stays 2^-9
    step = torch.ldexp(torch.ones_like(x), p - 3)
    return torch.round(x / step) * step


def _exact_rows(st):
    s, total = st["x"].double(), None
    if st["case"]["op"] == "quant":
        if st["index"] is not None:
            s = s[st["index"].long()]
    else:
        if st["residual"] is not None:
            total = s = s + st["residual"].double()
        s = s / (s.pow(2).sum(dim=-1, keepdim=True) / s.shape[1] + 1e-5).sqrt()
        if st["gain"] is not None:
            s = s * st["gain"].double()
    if st["scale"] is None:
        return {"y": s, "scale": None, "sum": total}
    scale = s.abs().max(dim=-1)[0] / 448
    got = {"y": _e4m3(s / scale[:, None]), "scale": scale}
    return got if st["case"]["op"] == "quant" else dict(got, sum=total)


# ---- linear, grouped ---------------------------------------------------------------------------------------------


def _act(x, kind):
    if kind == "relu":
        return x.clamp(min=0)
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu":
        return x * 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return x * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _tail(x, case):
    """Activation of what the product, its scales and the bias gave, pairs of columns joined where gated."""
    if case["gated"]:
        return _act(x[..., 0::2], case["act"]) * x[..., 1::2]
    return _act(x, case["act"])


def _args(st):
    return dict(a_scale=st["a_scale"], w_scale=st["w_scale"], bias=st["bias"], act=st["act"], gated=st["case"]["gated"],
                residual=st["residual"])


def _run_linear(st):
    if own:
        st["ctx"].linear(st["a"], st["w"], st["out"], **_args(st))
        return st["out"]
    x = torch.matmul(st["a"].float(), st["w"].float().T)
    if st["a_scale"] is not None:
        x = x * st["a_scale"][:, None] * st["w_scale"]
    if st["bias"] is not None:
        x = x + st["bias"]
    x = _tail(x, st["case"])
    return (x if st["residual"] is None else x + st["residual"].float()).to(st["out"].dtype)


def _run_grouped(st):
    if own:
        st["ctx"].linear_grouped(st["a"], st["w"], st["start"], st["out"], **_args(st))
        return st["out"]
    # every group padded to the longest
    start = st["start"].long()
    m = st["a"].shape[0]
    row = torch.arange(m, device=start.device)
    group = torch.searchsorted(start[1:], row, right=True)
    place = row - start[group]
    a = st["a"].float()
    if st["a_scale"] is not None:
        a = a * st["a_scale"][:, None]
    wide = torch.zeros(len(start) - 1, st["most"], a.shape[1], device=a.device)
    wide[group, place] = a
    x = torch.bmm(wide, st["w"].float().transpose(1, 2))[group, place]
    if st["w_scale"] is not None:
        x = x * st["w_scale"][group]
    if st["bias"] is not None:
        x = x + st["bias"][group]
    x = _tail(x, st["case"])
    return (x if st["residual"] is None else x + st["residual"].float()).to(st["out"].dtype)


def _exact_linear(st):
    case = st["case"]
    n, act, pieces, at = case["n"], case["act"], [], 0
    w = st["w"].reshape(-1, n, case["k"])
    for e, count in enumerate(_counts(case)):
        if not count:
            continue
        rows = slice(at, at + count)
        at += count
        a, b = st["a"][rows].double(), w[e].double()
        if st["a_scale"] is not None:
            a = a * st["a_scale"][rows].double()[:, None]
            b = b * st["w_scale"].view(-1, n)[e].double()[:, None]
        y = a @ b.T
        if st["bias"] is not None:
            y += st["bias"].view(-1, n)[e].double()
        gate, up = (y[:, 0::2], y[:, 1::2]) if case["gated"] else (y, None)
        if act == "relu":
            gate = torch.where(gate > 0, gate, 0.0)
        elif act == "silu":
            gate = gate * torch.sigmoid(gate)
        elif act == "gelu":
            gate = 0.5 * gate * torch.erfc(-gate / 2 ** 0.5)
        elif act == "gelu_tanh":
            gate = gate * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (gate + 0.044715 * gate ** 3))
        pieces.append(gate if up is None else gate * up)
    y = torch.cat(pieces)
    return y if st["residual"] is None else y + st["residual"].double()


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return _exact_rows(st) if case["op"] in ("norm", "quant") else _exact_linear(st)
