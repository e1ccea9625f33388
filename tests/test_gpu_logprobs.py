"""Logits scoring through the C-ABI against float64: log probability of the given token, entropy, the k best."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_25405_b200 import binding as B
from tests.kv8_util import context

pytestmark = pytest.mark.gpu


def _ctx():
    return context(2, 1, 64)[1]


def _run(x, tokens, k):
    n = x.shape[0]
    out = [torch.full((n,), 99.0, device="cuda"), torch.full((n,), 99.0, device="cuda"),
           torch.full((n, k), -7, dtype=torch.int32, device="cuda"), torch.full((n, k), 99.0, device="cuda")]
    _ctx().logprobs(x, tokens, out[0], out[1], *(out[2:] if k else ()))
    return [o.cpu().numpy() for o in out]


def _reference(x, tokens, k):
    """From the definition in float64: x numpy [n, V]."""
    x = x.astype(np.float64)
    m = x.max(axis=1, keepdims=True)
    z = x - m
    e = np.exp(z)
    s = e.sum(axis=1)
    with np.errstate(invalid="ignore"):
        ent = np.log(s) - np.where(e > 0, e * z, 0.0).sum(axis=1) / s
    lp = z[np.arange(len(x)), tokens] - np.log(s)
    ids = np.argsort(-x, axis=1, kind="stable")[:, :k]
    return lp, ent, ids, np.take_along_axis(z, ids, axis=1) - np.log(s)[:, None]


def _check(x, k, seed=0):
    r = np.random.default_rng(seed)
    tokens = r.integers(0, x.shape[1], x.shape[0]).astype(np.int32)
    got = _run(x, torch.from_numpy(tokens).cuda(), k)
    ref = _reference(x.float().cpu().numpy(), tokens, k)
    assert np.array_equal(got[2], ref[2])
    # x - m is rounded once (2^-24 |z|), log1p(T) carries the sum's relative error: terms e^d with d rounded
    # (|d| 2^-24 each, |d| e^d <= 0.37 of the largest), ex2 2^-22, tree additions of 16 + 15 levels 2^-24 each
    tol = lambda z: 2.0 ** -23 * np.abs(z) + 2.0 ** -19  # noqa: E731
    for a, b in ((got[0], ref[0]), (got[3], ref[3])):
        fin = np.isfinite(b)
        assert np.array_equal(np.isfinite(a), fin) and np.all(np.abs(a[fin] - b[fin]) <= tol(b[fin]))
    assert np.all(np.abs(got[1] - ref[1]) <= 2.0 ** -19 * (1 + np.abs(ref[1])))
    return got, ref


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("n,vocab", [(1, 1), (3, 2), (1, 31), (5, 1000), (2, 4095), (2, 4096), (2, 4097), (7, 32000), (1, 128256),
                                     (70, 8191), (700, 20011), (3, 262144)])
@pytest.mark.parametrize("k", [0, 1, 20, 32])
def test_rows_of_every_size(n, vocab, dtype, k):
    """Vocabularies on both sides of a tile, rows that are shared by clusters of every size and rows that are not."""
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab + n)
    _check((torch.randn(n, vocab, generator=g, device="cuda") * 3).to(dtype), min(k, vocab))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_strided_and_misaligned_rows(dtype):
    """Rows inside a wider matrix, at offsets and strides that are no multiple of 16 bytes; the columns beside the
    vocabulary hold larger logits and NaN and do not count."""
    for off, stride in ((0, 5008), (1, 5003), (3, 5009), (8, 5016)):
        wide = torch.full((9, stride), float("nan"), dtype=dtype, device="cuda")
        wide[:, :off] = 1000.0
        x = wide[:, off:off + 5000]
        x.copy_(torch.randn(9, 5000, device="cuda") * 3)
        a = _check(x, 20)[0]
        b = _check(x.contiguous(), 20)[0]
        assert all(np.array_equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("order", ["equal", "two values", "ascending", "descending", "top at the end", "one thread's elements"])
@pytest.mark.parametrize("vocab", [50, 9000, 40000])
def test_arrangements_that_are_hard_on_the_selection(order, vocab):
    """All equal (ties go to the lowest token), ascending (every tile beats the one before), the best ones all among one
    thread's elements."""
    i = torch.arange(vocab, dtype=torch.float32, device="cuda")
    x = {"equal": torch.full_like(i, 2.5), "two values": (i % 3 == 1).float(), "ascending": i / vocab * 8, "descending": -i / vocab * 8,
         "top at the end": (i > vocab - 30).float() * 5 + i * 1e-5,
         "one thread's elements": torch.where((i % 1024 < 4) | (i % 2048 < 8), 5 + i * 1e-5, -i * 1e-5)}[order]
    x = torch.stack([x, x.flip(0), torch.randn_like(x)])
    for k in (1, 7, 32):
        _check(x, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("n,vocab", [(1, 40), (5, 20000), (1, 128256), (40, 128256), (500, 33001)])
def test_zeros_of_either_sign_are_equal(n, vocab, dtype):
    """-0 and +0 are equal logits: the lower token comes first, inside a slice, across slices and across the blocks that share a
    row; as the best logits, between larger and smaller ones, and in rows of nothing else."""
    r = np.random.default_rng(vocab + n)
    x = -np.abs(r.standard_normal((n, vocab))) - 0.5
    for i in range(n):
        at = r.choice(vocab, min(vocab // 2, 30), replace=False)
        x[i, at] = np.where(r.integers(0, 2, len(at)) == 1, 0.0, -0.0)
        if i % 3 == 1:
            x[i, at[:3]] = 2.0
    x[0, np.argmax(x[0] == 0.0)] = -0.0                    # the first zero is a negative one
    if n > 2:
        x[2] = np.where(np.arange(vocab) % 2 == 0, -0.0, 0.0)
    t = torch.from_numpy(x).to(dtype).cuda()
    for k in (1, 7, min(32, vocab)):
        _check(t, k)


def test_zeros_of_either_sign_and_argmax():
    """The first alternative is hb_argmax's token in rows whose largest logits are zeros of both signs."""
    from paper_2609_25405_b200 import synth
    ctx = B.Context(B.model_cfg(synth.ModelShape("v", 1, 64, 1, 1, 64, 64, 32000), 16), 1, 1, 1)
    x = -torch.rand(4, 32000, device="cuda") - 0.1
    for i, (neg, pos) in enumerate(((5, 9), (9, 5), (100, 31000), (31000, 100))):
        x[i, neg], x[i, pos] = -0.0, 0.0
    tok, ids, top = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(4, 2, device="cuda")
    ctx.argmax(x, 4, tok)
    ctx.logprobs(x, None, None, None, ids, top)
    assert torch.equal(tok, ids[:, 0]) and tok.tolist() == [5, 5, 100, 100] and torch.equal(top[:, 0], top[:, 1])
    ctx.close()


def test_nearly_certain_rows_keep_their_entropy():
    """One logit 5 .. 60 above the rest: the entropy and -log p of the best are tiny and right to 2^-17 relative."""
    gap = torch.arange(5.0, 61.0, 5.0, device="cuda")
    x = torch.zeros(len(gap), 30000, device="cuda") + torch.linspace(0, 1, 30000, device="cuda")
    x[:, 777] = 1 + gap
    tokens = torch.full((len(gap),), 777, dtype=torch.int32, device="cuda")
    got = _run(x, tokens, 2)
    z = x.cpu().numpy().astype(np.float64) - (1 + gap.cpu().numpy().astype(np.float64))[:, None]
    z[:, 777] = 0
    e = np.exp(z)
    T = np.delete(e, 777, axis=1).sum(axis=1)
    ent = np.log1p(T) - (e * z).sum(axis=1) / (1 + T)
    assert np.all(np.abs(got[1] - ent) <= 2.0 ** -17 * ent)
    assert np.all(np.abs(got[0] + np.log1p(T)) <= 2.0 ** -17 * np.log1p(T))
    assert np.all(got[2][:, 0] == 777) and np.all(got[2][:, 1] == 29999) and np.array_equal(got[3][:, 0], got[0])


def test_masked_logits():
    """-inf has probability zero: any number of them, the given token too, down to one logit that is left; fewer
    unmasked logits than alternatives: the masked ones follow in order, at -inf."""
    V = 9001
    x = torch.randn(6, V, device="cuda")
    x[0, ::2] = -float("inf")
    x[1, 10:] = -float("inf")
    x[2] = -float("inf"); x[2, 8999] = -3.0
    x[3, 4096:] = -float("inf")                           # whole tiles
    x[4, :8192] = -float("inf")
    x[5] = -3.4e38; x[5, 5] = 3.0                          # masks of the type's lowest value
    tokens = torch.tensor([0, 5, 8999, 5000, 8999, 5], dtype=torch.int32, device="cuda")
    got = _run(x, tokens, 20)
    ref = _reference(x.cpu().numpy(), tokens.cpu().numpy(), 20)
    assert np.array_equal(got[2], ref[2])
    for a, b in ((got[0], ref[0]), (got[3], ref[3])):
        assert np.array_equal(np.isneginf(a), np.isneginf(b))
        fin = np.isfinite(b)
        assert np.all(np.abs(a[fin] - b[fin]) <= 2.0 ** -23 * np.abs(b[fin]) + 2.0 ** -19)
    assert np.all(np.abs(got[1] - ref[1]) <= 2.0 ** -19 * (1 + np.abs(ref[1])))
    assert got[0][2] == 0.0 and got[1][2] == 0.0 and got[0][5] == 0.0 and got[1][5] == 0.0


@pytest.mark.parametrize("vocab", [40, 20000])
def test_rows_without_probabilities(vocab):
    """NaN, +inf or nothing but -inf: floats are NaN, the alternatives are still ranked (NaN last), other rows unharmed."""
    x = torch.randn(5, vocab, device="cuda")
    clean = x[4].clone()
    x[0, 7] = float("nan")
    x[1, 9] = float("inf")
    x[2] = -float("inf")
    x[3] = float("nan"); x[3, 30] = 1.0
    tokens = torch.tensor([3, 9, 0, 30, 2], dtype=torch.int32, device="cuda")
    got = _run(x, tokens, 5)
    assert np.all(np.isnan(got[0][:4])) and np.all(np.isnan(got[1][:4])) and np.all(np.isnan(got[3][:4]))
    assert got[2][1, 0] == 9 and list(got[2][2]) == [0, 1, 2, 3, 4] and list(got[2][3]) == [30, 0, 1, 2, 3]
    keep = [i for i in np.argsort(-x[0].cpu().numpy(), kind="stable") if i != 7][:5]
    assert list(got[2][0]) == keep
    alone = _run(clean[None], tokens[4:], 5)
    assert all(np.array_equal(a[4:], b) for a, b in zip(got, alone))


def test_tokens_outside_the_vocabulary():
    x = torch.randn(3, 100, device="cuda")
    got = _run(x, torch.tensor([-1, 5, -2 ** 31], dtype=torch.int32, device="cuda"), 1)
    assert got[0][0] == 0 and got[0][2] == 0 and got[0][1] < 0 and _ctx().status_poll() == 0
    got2 = _run(x, torch.tensor([100, 5, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), 1)
    assert np.isnan(got2[0][0]) and np.isnan(got2[0][2]) and got2[0][1] == got[0][1]
    assert _ctx().status_poll() == 128 and _ctx().status_poll() == 0


def test_a_rows_bits_do_not_depend_on_the_other_rows():
    """Alone a row is shared by a cluster of eight, among 600 it has one block."""
    x = torch.randn(600, 33001, device="cuda") * 2
    tokens = torch.randint(33001, (600,), device="cuda", dtype=torch.int32)
    many = _run(x, tokens, 20)
    for n in (1, 3, 60, 200):
        few = _run(x[:n], tokens[:n], 20)
        assert all(np.array_equal(a[:n], b) for a, b in zip(many, few))


def test_outputs_that_are_not_asked_for():
    x = torch.randn(4, 5000, device="cuda")
    tokens = torch.arange(4, dtype=torch.int32, device="cuda")
    full = _run(x, tokens, 3)
    ctx = _ctx()
    ent, ids, top = torch.empty(4, device="cuda"), torch.empty(4, 3, dtype=torch.int32, device="cuda"), torch.empty(4, 3, device="cuda")
    ctx.logprobs(x, None, None, ent)
    assert np.array_equal(ent.cpu().numpy(), full[1])
    lp = torch.empty(4, device="cuda")
    ctx.logprobs(x, tokens, lp)
    assert np.array_equal(lp.cpu().numpy(), full[0])
    ctx.logprobs(x, None, None, None, ids, top)
    assert np.array_equal(ids.cpu().numpy(), full[2]) and np.array_equal(top.cpu().numpy(), full[3])
    ctx.logprobs(x[:0], tokens[:0], lp[:0])


def test_agrees_with_argmax_and_replays_in_a_graph():
    """Greedy decoding with scores: hb_argmax's token is the first alternative; captured and replayed over new logits."""
    from paper_2609_25405_b200 import synth
    cfg = B.model_cfg(synth.ModelShape("v", 1, 64, 1, 1, 64, 64, 32000), 16)
    ctx = B.Context(cfg, 1, 1, 1)
    x = torch.randn(6, 32000, device="cuda")
    tok, lp, ent = torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    ids, top = torch.empty(6, 4, dtype=torch.int32, device="cuda"), torch.empty(6, 4, device="cuda")

    def both():
        ctx.argmax(x, 6, tok)
        ctx.logprobs(x, tok, lp, ent, ids, top)
    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for seed in range(3):
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, ids[:, 0]) and torch.equal(lp, top[:, 0])
        got = [t.cpu().numpy() for t in (lp, ent, ids, top)]
        ref = _run(x, tok, 4)
        assert all(np.array_equal(a, b) for a, b in zip(got, ref))
    ctx.close()


def test_refusals():
    ctx, lib, P = _ctx(), B.lib, C.c_void_p
    x = torch.randn(4, 100, device="cuda")
    b = x.data_ptr()

    def call(h=ctx.handle, lo=b, dt=0, n=4, v=100, st=100, tok=b, k=2, lp=b, en=b, ids=b, top=b):
        return lib.hb_logprobs(h, P(lo), dt, n, v, st, P(tok), k, P(lp), P(en), P(ids), P(top), None)
    assert call(h=None) == -1 and call(lo=0) == -1 and call(dt=2) == -1 and call(n=-1) == -1 and call(v=0) == -1
    assert call(st=99) == -1 and call(k=-1) == -1 and call(k=33) == -1 and call(k=5, v=4) == -1
    assert call(lo=b + 2) == -1 and call(dt=1, lo=b + 1) == -1 and call(lp=b + 2) == -1 and call(ids=b + 1) == -1
    assert call(ids=0) == -1 and call(top=0) == -1 and call(tok=0) == -1 and call(lp=0) == -1
    assert call(v=(1 << 20) + 1, st=1 << 21) == -5
    assert call(n=0) == 0
    o = torch.empty(4, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in ((x.double(), t, o), (x, t.long(), o), (x, t, o[:3]), (x.t(), t, o), (x.cpu(), t, o), (x, t, o.half())):
        with pytest.raises(ValueError):
            ctx.logprobs(*bad)
