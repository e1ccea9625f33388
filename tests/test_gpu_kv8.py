"""The 8-bit KV cache operators through the C-ABI against the plain float64 statement: append (norms, rotation,
quantisation, scale growth) and attention (decode rows, key splits, chunks, grouped heads)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8 as O
from paper_2609_25405_b200 import binding as B
from tests.kv8_util import Rows, attend_bound, context, layer_bytes, oracle_layer, random_arena

pytestmark = pytest.mark.gpu

EPS = 1e-6


# ---- append ------------------------------------------------------------------------------------------------------


def _append_oracle(cache, rows, x, hq, hkv, dh, cos, sin, halves, gains):
    """(q in float64 [T, hq, dh], exact k, v before rounding per row); updates `cache`."""
    q = np.full((rows.T, hq, dh), np.nan)
    exact = []
    for (p, n), at, pages in zip(rows.segs, rows.start, rows.pages):
        y = x[at:at + n].reshape(n, hq + 2 * hkv, dh).copy()
        for j in range(n):
            for part, gain in ((slice(0, hq), gains[0]), (slice(hq, hq + hkv), gains[1])):
                if gain is not None:
                    y[j, part] = O.rmsnorm_head(y[j, part], gain, EPS)
                if cos is not None:
                    y[j, part] = O.rotate(y[j, part], cos[p + j], sin[p + j], halves)
        q[at:at + n] = y[:, :hq]
        for b in range(p // 16, (p + n + 15) // 16):
            lo, hi = max(p, b * 16), min(p + n, b * 16 + 16)
            if hi <= lo:
                continue
            for which in range(2):
                new = y[lo - p:hi - p, hq + which * hkv:hq + (which + 1) * hkv]
                cache.append(which, pages[b], lo - b * 16, new)
                exact.append((which, pages[b], lo - b * 16, new))
    return q, exact


@pytest.mark.parametrize("hq,hkv,dh,rot,halves,norm", [
    (4, 4, 64, 64, False, False), (8, 2, 64, 64, True, True), (16, 1, 64, 32, True, False), (6, 6, 64, 16, False, True),
    (32, 8, 128, 128, False, False), (32, 8, 128, 128, True, True), (5, 5, 128, 64, True, True), (16, 2, 128, 48, False, True),
    (16, 1, 128, 0, False, True), (2, 2, 128, 16, True, False)])
def test_append_matches_the_definition(hq, hkv, dh, rot, halves, norm):
    """Ragged segments (from mid-page, over page borders, empty, one row), padding rows between them, a strided
    qkv view, second of two layers: q within fp16 rounding, every code the rounding of the exact value, scales
    exact, everything else untouched."""
    cfg, ctx = context(hq, hkv, dh)
    segs = [(0, 1), (5, 3), (15, 1), (16, 16), (7, 40), (100, 0), (0, 33), (31, 1), (200, 2)]
    rows = Rows(segs, 40, seed=dh + hq, gap=2)
    kv = random_arena(cfg, 40, seed=3)
    before = [layer_bytes(kv, l).copy() for l in range(2)]
    r = np.random.default_rng(hq * dh + rot)
    w = (hq + 2 * hkv) * dh
    x16 = r.standard_normal((rows.T, w)).astype(np.float16) * np.exp2(r.integers(-3, 4, (rows.T, 1))).astype(np.float16)
    wide = torch.full((rows.T, w + 24), 7.0, dtype=torch.float16, device="cuda")
    wide[:, 8:8 + w] = torch.from_numpy(x16).cuda()
    gains = [(1 + 0.2 * torch.randn(dh, generator=torch.Generator().manual_seed(i))).bfloat16() if norm else None for i in range(2)]
    rope, cos, sin = None, None, None
    if rot:
        cos, sin = B.rope_table(256, rot, 1e4)
        rope = B.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), B.ROPE_HALVES if halves else B.ROPE_PAIRS)
    out = torch.full((rows.T, hq * dh + 8), -3.0, dtype=torch.float16, device="cuda")
    dg = [g.cuda() if g is not None else None for g in gains]
    ctx.kv8_append(kv, 1, rows.dev, wide[:, 8:8 + w], out[:, :hq * dh], rope=rope, q_norm=dg[0], k_norm=dg[1], norm_eps=EPS)
    torch.cuda.synchronize()
    assert ctx.status_poll() == 0
    ref = O.read_layer(before[1], dh)
    q, exact = _append_oracle(ref, rows, x16.astype(np.float64), hq, hkv, dh, cos, sin, halves,
                              [g.double().numpy() if g is not None else None for g in gains])
    got_q = out.cpu().numpy().astype(np.float64)
    real = np.repeat(True, rows.T)
    real[:] = ~np.isnan(q[:, 0, 0])
    # padding rows and the columns beside the view stay
    assert np.all(got_q[~real] == -3.0) and np.all(got_q[:, hq * dh:] == -3.0)
    ref_q = q[real].reshape(-1, hq * dh)
    # fp16 rounding of the result, and 2^-20 of the head's largest element for norm and rotation in fp32
    # (a 128-term sum of squares, one reciprocal root, two products each: under 12 units of 2^-24)
    top = np.repeat(np.abs(q[real]).max(axis=2), dh, axis=1)
    assert np.all(np.abs(got_q[real][:, :hq * dh] - ref_q) <= 2.0 ** -11 * np.abs(ref_q) + 2.0 ** -25 + 2.0 ** -20 * top)
    # the other layer is untouched, and so is every page nobody wrote
    after = layer_bytes(kv, 1)
    assert np.array_equal(layer_bytes(kv, 0), before[0])
    written = {int(pg) for _, pg, _, _ in exact}
    for pg in range(40):
        if pg not in written:
            assert np.array_equal(after[pg], before[1][pg])
    got = O.read_layer(after, dh)
    fresh = {}
    for which, pg, slot0, new in exact:
        assert np.array_equal(got.exps[which][pg], ref.exps[which][pg])
        fresh.setdefault((which, int(pg)), set()).update(range(slot0, slot0 + len(new)))
        s = np.exp2(ref.exps[which][pg].astype(np.float64))[None, :, None]
        val = got.codes[which][pg][:, slot0:slot0 + len(new)].transpose(1, 0, 2) * s
        slack = 2.0 ** -20 * np.abs(new).max(axis=2, keepdims=True) if which == 0 else 0.0
        assert np.all(np.abs(val - new) <= O.e4m3_half_step(np.abs(new / s) + slack / s) * s + slack)
    for (which, pg), slots in fresh.items():      # slots nobody appended to: as the definition leaves them, exactly
        keep = [t for t in range(16) if t not in slots]
        assert np.array_equal(got.codes[which][pg][:, keep], ref.codes[which][pg][:, keep])


@pytest.mark.parametrize("dh", [64, 128])
def test_scale_growth_stores_the_old_codes_again(dh):
    """One row at a time into a page, magnitudes going up and down by powers of two: after every append all
    sixteen slots are exactly what the definition says (k unrotated, so the values are fp16 numbers)."""
    cfg, ctx = context(4, 2, dh)
    kv = random_arena(cfg, 3, seed=1)
    r = np.random.default_rng(5)
    cache = oracle_layer(kv, 0)
    out = torch.empty(1, 4 * dh, dtype=torch.float16, device="cuda")
    for t, e in enumerate([0, -6, 3, 3, -14, 5, 9, 9, 1, 12, -20, 14, 15, 0, 15, 2]):
        x = (r.uniform(-1, 1, (1, 8 * dh)) * 2.0 ** e).astype(np.float16)
        rows = Rows([(t, 1)], 3, seed=2)
        ctx.kv8_append(kv, 0, rows.dev, torch.from_numpy(x).cuda(), out)
        for which in range(2):
            cache.append(which, rows.pages[0][0], t, x.astype(np.float64)[0].reshape(8, dh)[None, 4 + 2 * which:6 + 2 * which])
        got = oracle_layer(kv, 0)
        for which in range(2):
            assert np.array_equal(got.exps[which], cache.exps[which]), t
            assert np.array_equal(got.codes[which], cache.codes[which]), t
    assert ctx.status_poll() == 0


def test_append_of_zeros_extremes_and_nan():
    """Zeros take the smallest scale; 65504 and its like round in their block; infinities saturate at the largest
    scale; a NaN stays a NaN in its place and does not move the scale."""
    cfg, ctx = context(2, 1, 64)
    kv = B.KvCache8(cfg, 8, fill=0x7F)          # what is there before is NaN everywhere, scales included
    rows = Rows([(0, 4)] * 5, 8)
    x = torch.zeros(20, 4 * 64, dtype=torch.float16)
    x[4:8, 128:] = 65504.0
    x[8:12, 128:] = 1.0
    x[9, 130] = float("inf")
    x[9, 200] = -float("inf")
    x[12:16, 128:] = 1.0
    x[13, 131] = float("nan")
    x[14, 250] = float("nan")
    x[16:20, 128:] = 2.0 ** -24
    out = torch.empty(20, 128, dtype=torch.float16, device="cuda")
    ctx.kv8_append(kv, 0, rows.dev, x.cuda(), out)
    assert ctx.status_poll() == 0
    c = oracle_layer(kv, 0)
    pg = [int(p[0]) for p in rows.pages]
    for which in range(2):
        assert c.exps[which][pg[0], 0] == -32 and not c.codes[which][pg[0]].any()
        assert c.exps[which][pg[1], 0] == 8 and np.all(c.codes[which][pg[1], 0, :4] == 256.0)
        assert np.all(c.codes[which][pg[1], 0, 4:] == 0.0)
        big = c.codes[which][pg[2], 0, 1]
        assert c.exps[which][pg[2], 0] == 24 and big[2 if which == 0 else 8] == (448.0 if which == 0 else -448.0)
        nan = np.isnan(c.codes[which][pg[3], 0])
        assert c.exps[which][pg[3], 0] == O.exponent(1.0) and nan.sum() == 1 and nan[(1, 2)[which], (3, 58)[which]]
        assert c.exps[which][pg[4], 0] == -32 and np.all(c.codes[which][pg[4], 0, :4] == 256.0)


@pytest.mark.parametrize("dh,halves", [(64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("odd", ["no epsilon", "gain", "table"])
def test_unused_slots_of_a_fresh_block_become_zero(dh, halves, odd):
    """Whatever the norm and the rotation make of nothing: an epsilon of zero (0 / 0), a gain or a rotary factor that is not finite."""
    cfg, ctx = context(4, 2, dh)
    kv = B.KvCache8(cfg, 12, fill=0xFF)
    rows = Rows([(0, 1), (0, 3), (0, 4), (16, 11), (5, 20), (0, 16)], 12, seed=4)
    x = torch.randn(rows.T, 8 * dh, device="cuda").half()
    gain = torch.ones(dh, device="cuda").bfloat16()
    cos, sin = (torch.from_numpy(t).cuda() for t in B.rope_table(32, dh, 1e4))
    if odd == "gain":
        gain[3] = float("inf")
    if odd == "table":
        cos[:, 1] = float("nan")
    out = torch.empty(rows.T, 4 * dh, dtype=torch.float16, device="cuda")
    ctx.kv8_append(kv, 0, rows.dev, x, out, rope=B.Rope(cos, sin, B.ROPE_HALVES if halves else B.ROPE_PAIRS), q_norm=gain, k_norm=gain,
                   norm_eps=0.0 if odd == "no epsilon" else EPS)
    assert ctx.status_poll() == 0
    c = oracle_layer(kv, 0)
    for (p, n), pages in zip(rows.segs, rows.pages):
        for b in range(p // 16, (p + n + 15) // 16):
            lo, hi = max(p - b * 16, 0), min(p + n - b * 16, 16)
            for which in range(2):
                if lo == 0:
                    assert np.all(c.codes[which][pages[b]][:, hi:] == 0.0), (which, p, n, b)
                if odd == "no epsilon":
                    assert np.all(np.isfinite(c.codes[which][pages[b]][:, lo:hi]))


def test_append_in_place_of_the_qkv_rows():
    """q_out may be the q part of qkv."""
    cfg, ctx = context(8, 2, 128)
    rows = Rows([(3, 20), (0, 1)], 8)
    x = torch.randn(21, 12 * 128, device="cuda").half()
    rope = B.Rope.table(64, 128, 1e4, B.ROPE_HALVES)
    outs = []
    for place in (False, True):
        kv = random_arena(cfg, 8, seed=9)
        y = x.clone()
        out = y[:, :8 * 128] if place else torch.empty(21, 8 * 128, dtype=torch.float16, device="cuda")
        ctx.kv8_append(kv, 0, rows.dev, y, out, rope=rope)
        outs.append((out.clone(), kv.arena.clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


# ---- attention ---------------------------------------------------------------------------------------------------


def _check_attend(ctx, kv, layer, rows, hq, hkv, dh, seed, scale=0.0, gap_value=-3.0, q_scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = (torch.randn(rows.T, hq * dh + 16, generator=g, device="cuda") * q_scale).half()[:, 8:8 + hq * dh]
    out = torch.full((rows.T, hq * dh + 8), gap_value, dtype=torch.float16, device="cuda")
    ctx.kv8_attention(kv, layer, rows.dev, q, out[:, :hq * dh], scale=scale)
    torch.cuda.synchronize()
    assert ctx.status_poll() == 0
    cache = oracle_layer(kv, layer)
    got, qn = out.cpu().numpy().astype(np.float64), q.cpu().numpy().astype(np.float64)
    used = np.zeros(rows.T, dtype=bool)
    worst = 0.0
    for (p, n), at, pages in zip(rows.segs, rows.start, rows.pages):
        if n == 0:
            continue
        used[at:at + n] = True
        K, V = (cache.rows(w, pages, p + n) for w in range(2))
        ref, mass = O.attend(qn[at:at + n].reshape(n, hq, dh), K, V, p, scale or dh ** -0.5)
        err = np.abs(got[at:at + n, :hq * dh].reshape(n, hq, dh) - ref)
        tol = attend_bound(mass, p + n, np.abs(V).max())
        assert np.all(err <= tol), ((p, n), np.max(err / tol))
        worst = max(worst, np.max(err / tol))
    assert np.all(got[~used] == gap_value) and np.all(got[:, hq * dh:] == gap_value)
    return worst


LENS = [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (62, 1), (63, 1), (510, 1), (511, 1), (512, 1), (1023, 1), (1025, 1), (2047, 1)]


@pytest.mark.parametrize("hq,hkv,dh", [(4, 4, 64), (8, 4, 64), (8, 2, 64), (8, 1, 64), (16, 1, 64),
                                       (2, 2, 128), (4, 2, 128), (32, 8, 128), (16, 2, 128), (32, 2, 128)])
def test_decode_rows(hq, hkv, dh):
    """One row per segment, contexts on both sides of page, tile and split borders, every group size."""
    cfg, ctx = context(hq, hkv, dh)
    kv = random_arena(cfg, 480, seed=dh)
    rows = Rows(LENS, 480, seed=hq, gap=1)
    print("\n  worst error / bound:", _check_attend(ctx, kv, 1, rows, hq, hkv, dh, 11))


@pytest.mark.parametrize("hq,hkv,dh", [(4, 4, 64), (8, 1, 64), (16, 1, 64), (4, 1, 128), (32, 8, 128), (32, 2, 128)])
def test_chunks(hq, hkv, dh):
    """Chunks of 2 .. 300 rows (every remainder of the row tiles), with and without earlier tokens, next to decode
    rows, an empty segment and padding rows."""
    cfg, ctx = context(hq, hkv, dh)
    kv = random_arena(cfg, 400, seed=dh + 1)
    segs = [(40, 1), (0, 2), (3, 3), (600, 4), (0, 17), (9, 0), (16, 64), (5, 129), (1000, 127), (130, 300), (0, 1), (777, 33)]
    rows = Rows(segs, 400, seed=hq, gap=1)
    print("\n  worst error / bound:", _check_attend(ctx, kv, 0, rows, hq, hkv, dh, 12))


@pytest.mark.parametrize("hq,hkv,dh", [(32, 8, 128), (32, 8, 64), (8, 8, 128), (16, 1, 64)])
def test_many_chunks(hq, hkv, dh):
    """More items than SMs, so that every resident block of the chunk body walks through several: blocks of 256 rows with one
    and with two row tiles, key ranges of every length, one after the other."""
    cfg, ctx = context(hq, hkv, dh)
    r = np.random.default_rng(hq + dh)
    segs = [(int(r.integers(0, 600)), int(q)) for q in r.integers(17, 400, 40 if hkv == 1 else 14)]
    n_pages = sum((p + q + 15) // 16 for p, q in segs)
    kv = random_arena(cfg, n_pages, seed=dh + 1)
    rows = Rows(segs, n_pages, seed=hq)
    items = sum((q * (hq // hkv) + 255) // 256 for _, q in segs) * hkv
    print("\n ", items, "items, worst error / bound:", _check_attend(ctx, kv, 0, rows, hq, hkv, dh, 12))


@pytest.mark.parametrize("scale_lo,scale_hi", [(-32, -30), (-14, 10), (0, 0)])
def test_block_scales_far_apart(scale_lo, scale_hi):
    """Scales of neighbouring pages that differ by up to 2^24 (K's are kept small so that the scores stay finite)."""
    cfg, ctx = context(8, 2, 128)
    kv = random_arena(cfg, 150, 4, scale_lo, scale_hi)
    kv.scales()[..., 0] = kv.scales()[..., 0].clamp(max=2.0 ** -8)
    if scale_hi > 4:   # fp16 output
        kv.scales()[..., 1] = kv.scales()[..., 1].clamp(max=2.0 ** 6)
    rows = Rows([(700, 1), (3, 40), (511, 1), (90, 5), (64, 130)], 150)
    _check_attend(ctx, kv, 0, rows, 8, 2, 128, 5)


def test_sharp_and_flat_softmax():
    """Scores of several hundred (one key takes all) and scores of zero (the mean over the keys)."""
    cfg, ctx = context(8, 2, 64)
    kv = random_arena(cfg, 200, 4, -6, -6)
    rows = Rows([(1500, 1), (0, 70), (30, 3), (513, 1)], 200)
    assert _check_attend(ctx, kv, 0, rows, 8, 2, 64, 5, scale=1e-12) <= 1.0
    # large scores: the fp32 rounding of the score itself (|s| 2^-22 at most after 64 products) enters the exponent
    q = torch.zeros(rows.T, 8 * 64, dtype=torch.float16, device="cuda")
    out = torch.empty_like(q)
    cache = oracle_layer(kv, 0)
    K0 = [cache.rows(0, p, sum(s)) for p, s in zip(rows.pages, rows.segs)]
    for (p, n), at, K in zip(rows.segs, rows.start, K0):      # every row points at its own first key
        for h in range(8):
            q[at:at + n, h * 64:(h + 1) * 64] = torch.from_numpy(K[0, h // 4] * 20).half().cuda()
    ctx.kv8_attention(kv, 0, rows.dev, q, out)
    assert ctx.status_poll() == 0
    got = out.cpu().numpy().astype(np.float64)
    for (p, n), at, K, pages in zip(rows.segs, rows.start, K0, rows.pages):
        V = cache.rows(1, pages, p + n)
        qn = q[at:at + n].cpu().numpy().astype(np.float64).reshape(n, 8, 64)
        ref, mass = O.attend(qn, K, V, p, 0.125)
        s_max = np.abs(np.einsum("nhd,khd->nhk", qn, np.repeat(K, 4, axis=1)) * 0.125).max()
        assert s_max > 100
        err = np.abs(got[at:at + n].reshape(n, 8, 64) - ref)
        assert np.all(err <= attend_bound(mass, p + n, np.abs(V).max()) + mass * s_max * 2.0 ** -20 + np.abs(V).max() * s_max * 2.0 ** -22)


@pytest.mark.parametrize("scale", [1e-38, 1e-36, 2.0 ** -90])
def test_scales_that_leave_nothing_of_the_scores(scale):
    """The factor of the scores times a block's scale may be too small for fp32: every key counts the same, and none that a row
    must not see, in decode rows, splits and chunks."""
    cfg, ctx = context(8, 2, 128)
    kv = random_arena(cfg, 150, 4)
    kv.scales()[..., 0] = 2.0 ** -32
    rows = Rows([(700, 1), (3, 40), (511, 1), (90, 5), (64, 130), (0, 2)], 150)
    _check_attend(ctx, kv, 0, rows, 8, 2, 128, 5, scale=scale)


@pytest.mark.parametrize("scale", [0.0, 1.0, 2.0 ** 30, 2.0 ** 60])
def test_scores_beyond_a_million(scale):
    """Queries of 60000, keys of one dimension each with values on the codes of e4m3: scores of 2^20 to 2^90, whose largest takes all;
    neighbouring values differ by 2^-4 of themselves at least, and equal ones are equal in fp32 too (V's scales are one).  Positive
    and negative scores, decode rows, splits and chunks."""
    cfg, ctx = context(8, 2, 64)
    kv = random_arena(cfg, 150, 4, 0, 0)
    t, d = np.arange(16)[:, None], np.arange(64)[None, :]
    a = layer_bytes(kv, 0).copy()
    r = np.random.default_rng(3)
    a[..., :16 * 64] = 0
    a[..., O.k_byte(np.arange(16), 0)] = r.integers(0x40, 0x7F, (150, 2, 16)) | (np.arange(2)[None, :, None] << 7)   # head 1: negative keys
    kv.arena[:a.size] = torch.from_numpy(a.reshape(-1)).cuda()
    kv.scales()[..., 0] = 2.0 ** 8
    rows = Rows([(700, 1), (3, 40), (511, 1), (90, 5), (64, 130), (0, 2), (20, 1)], 150)
    q = torch.zeros(rows.T, 8, 64, dtype=torch.float16, device="cuda")
    q[:, :, 0] = 60000.0
    out = torch.empty(rows.T, 512, dtype=torch.float16, device="cuda")
    ctx.kv8_attention(kv, 0, rows.dev, q.view(rows.T, 512), out, scale=scale)
    assert ctx.status_poll() == 0
    cache, got, qn = oracle_layer(kv, 0), out.cpu().numpy().astype(np.float64), q.cpu().numpy().astype(np.float64)
    for (p, n), at, pages in zip(rows.segs, rows.start, rows.pages):
        K, V = (cache.rows(w, pages, p + n) for w in range(2))
        ref, mass = O.attend(qn[at:at + n], K, V, p, scale or 0.125)
        err = np.abs(got[at:at + n].reshape(n, 8, 64) - ref)
        assert np.all(err <= attend_bound(mass, p + n, np.abs(V).max())), ((p, n), np.max(err))


def test_scales_up_to_their_limit():
    """2^60 keeps every score finite (65504 * 448 * 2^24 * 128 * 2^60 log2(e) < 2^117): queries of zero still give the mean, and
    anything above is refused."""
    cfg, ctx = context(8, 2, 64)
    kv = random_arena(cfg, 100, 4)
    kv.scales()[..., 0] = 2.0 ** 24
    rows = Rows([(700, 1), (3, 40), (20, 1)], 100)
    _check_attend(ctx, kv, 0, rows, 8, 2, 64, 5, scale=2.0 ** 60, q_scale=0.0)
    q = torch.full((rows.T, 512), 65504.0, dtype=torch.float16, device="cuda")
    out = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, out, scale=2.0 ** 60)
    assert bool(torch.isfinite(out).all()) and ctx.status_poll() == 0
    for scale in (2.0 ** 60 * 1.001, 1e30, 3e38):
        with pytest.raises(B.HbError) as e:
            ctx.kv8_attention(kv, 0, rows.dev, q, out, scale=scale)
        assert e.value.code == -1


def test_stale_bytes_behind_the_last_key():
    """NaN codes in the unused slots of a request's last page, and in pages of nobody, do not reach any row."""
    cfg, ctx = context(8, 2, 128)
    kv = random_arena(cfg, 60, 4)
    rows = Rows([(4, 1), (17, 40), (0, 1), (250, 1), (33, 9)], 60, seed=3)
    used = {(int(pg), t) for (p, n), pages in zip(rows.segs, rows.pages) for i, pg in enumerate(pages) for t in range(16) if i * 16 + t < p + n}
    t, d = np.arange(16)[:, None], np.arange(128)[None, :]
    a = layer_bytes(kv, 0).copy()
    for pg in range(60):
        for tok in range(16):
            if (pg, tok) not in used:
                a[pg][:, O.k_byte(tok, d[0])] = 0x7F
                a[pg][:, 16 * 128 + O.v_byte(tok, d[0])] = 0xFF
    kv.arena[:a.size] = torch.from_numpy(a.reshape(-1)).cuda()
    assert np.isnan(oracle_layer(kv, 0).codes[1]).any()
    _check_attend(ctx, kv, 0, rows, 8, 2, 128, 6)


@pytest.mark.parametrize("dh", [64, 128])
def test_nan_in_tokens_that_come_later(dh):
    """A token whose key and value (or value alone, in one dimension) are NaN: rows before it are what they are without it,
    to the bit; rows that see it are NaN (in that dimension at least); in decode rows, small and large chunks."""
    cfg, ctx = context(8, 2, dh)
    segs = [(20, 4), (600, 2), (9, 40), (100, 200), (30, 1), (70, 130)]
    bad = [22, 601, 30, 250, 7, 70 + 129]               # position of the token in its request
    rows = Rows(segs, 120, seed=5)
    kv = random_arena(cfg, 120, 4)
    q = torch.randn(rows.T, 8 * dh, device="cuda").half()
    clean = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, clean)
    saved = kv.arena.clone()
    for whole in (True, False):
        a = layer_bytes(kv, 0).copy()
        for pages, b in zip(rows.pages, bad):
            dims = np.arange(dh) if whole else np.array([dh // 2 + 3])
            blk = a[pages[b // 16]]
            blk[:, 16 * dh + O.v_byte(b % 16, dims)] = 0x7F
            if whole:
                blk[:, O.k_byte(b % 16, dims)] = 0xFF
        kv.arena[:a.size] = torch.from_numpy(a.reshape(-1)).cuda()
        out = torch.empty_like(q)
        ctx.kv8_attention(kv, 0, rows.dev, q, out)
        assert ctx.status_poll() == 0
        for (p, n), at, b in zip(segs, rows.start, bad):
            sees = torch.arange(p, p + n, device="cuda") >= b
            got, ref = out[at:at + n].view(n, 8, dh), clean[at:at + n].view(n, 8, dh)
            assert torch.equal(got[~sees], ref[~sees]), (p, n)
            hit = got[sees] if whole else got[sees][..., dh // 2 + 3]
            assert bool(torch.isnan(hit).all()), (p, n)
        kv.arena.copy_(saved)


def test_a_requests_result_does_not_depend_on_its_batch():
    """Every segment alone gives the bits it gives in the batch."""
    cfg, ctx = context(32, 8, 128)
    kv = random_arena(cfg, 700, 4)
    segs = [(700, 1), (100, 4), (2000, 1), (40, 200), (511, 2), (1300, 77), (5, 1)]
    rows = Rows(segs, 700, seed=3)
    q = torch.randn(rows.T, 32 * 128, device="cuda").half()
    out = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, out)
    for i, (p, n) in enumerate(segs):
        one = Rows([(p, n)], 700)
        one.dev.page_ids.copy_(torch.from_numpy(rows.pages[i]).cuda())
        at = rows.start[i]
        alone = torch.empty(n, 32 * 128, dtype=torch.float16, device="cuda")
        ctx.kv8_attention(kv, 0, one.dev, q[at:at + n], alone)
        assert torch.equal(alone, out[at:at + n]), (p, n)
    assert ctx.status_poll() == 0


@pytest.mark.parametrize("dh", [64, 128])
def test_as_many_segments_as_there_may_be(dh):
    """8192 segments, most of them without rows: chunks and decode rows among them give the bits they give alone."""
    cfg, ctx = context(8, 2, dh)
    kv = random_arena(cfg, 300, 4)
    some = {0: (40, 70), 3000: (300, 1), 5001: (0, 33), 8191: (500, 300)}
    segs = [some.get(i, (0, 0)) for i in range(8192)]
    rows = Rows(segs, 300, seed=3)
    q = torch.randn(rows.T, 8 * dh, device="cuda").half()
    out = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, out)
    for i, (p, n) in some.items():
        one = Rows([(p, n)], 300)
        one.dev.page_ids.copy_(torch.from_numpy(rows.pages[i]).cuda())
        at = rows.start[i]
        alone = torch.empty(n, 8 * dh, dtype=torch.float16, device="cuda")
        ctx.kv8_attention(kv, 0, one.dev, q[at:at + n].contiguous(), alone)
        assert torch.equal(alone, out[at:at + n]), (p, n)
    assert ctx.status_poll() == 0


def test_long_contexts_and_offsets_beyond_32_bits():
    """An arena of more than 4 GiB, contexts of 40000 and 131072 keys whose pages lie at its far end (listed
    several times over), appended to and read."""
    cfg, ctx = context(8, 8, 128, layers=1)
    n_pages = 131000                                   # 131000 * 8 * 4128 bytes = 4.03 GiB
    kv = B.KvCache8(cfg, n_pages)
    assert kv.arena.numel() > 2 ** 32
    tail = 300
    small = random_arena(cfg, tail, 8)
    kv._blocks()[0, n_pages - tail:] = small._blocks()[0]
    segs = [(131071, 1), (39999, 1), (32768, 1)]
    rows = Rows(segs, 131072)                          # page lists replaced below
    r = np.random.default_rng(3)
    ids = [r.integers(n_pages - tail + 3, n_pages, len(p)).astype(np.int32) for p in rows.pages]
    for i, p in enumerate(ids):
        p[-1] = n_pages - tail + i                     # the page that is appended to is the request's own
    rows.pages = ids
    rows.dev.page_ids.copy_(torch.from_numpy(np.concatenate(ids)).cuda())
    x = torch.randn(3, 24 * 128, device="cuda").half()
    q = torch.empty(3, 8 * 128, dtype=torch.float16, device="cuda")
    ctx.kv8_append(kv, 0, rows.dev, x, q)
    out = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, out)
    assert ctx.status_poll() == 0
    a = kv._blocks()[0, n_pages - tail:].cpu().numpy()
    cache = O.read_layer(a, 128)
    got, qn = out.cpu().numpy().astype(np.float64), q.cpu().numpy().astype(np.float64)
    assert np.array_equal(qn, x[:, :8 * 128].cpu().numpy().astype(np.float64))
    for i, (p, n) in enumerate(segs):
        K, V = (cache.rows(w, ids[i] - (n_pages - tail), p + n) for w in range(2))
        new = x[i].cpu().numpy().astype(np.float64).reshape(24, 128)
        assert np.all(np.abs(K[-1] - new[8:16]) <= 2.0 ** -4 * np.abs(new[8:16]) + 2.0 ** -8)
        ref, mass = O.attend(qn[i].reshape(1, 8, 128), K, V, p, 128 ** -0.5)
        assert np.all(np.abs(got[i].reshape(1, 8, 128) - ref) <= attend_bound(mass, p + n, np.abs(V).max()))


# ---- the calls around them ---------------------------------------------------------------------------------------


def _small(seed=0, n_pages=64):
    cfg, ctx = context(8, 2, 64)
    kv = random_arena(cfg, n_pages, seed)
    rows = Rows([(30, 1), (700, 1), (0, 20)], n_pages, seed=seed)
    return ctx, kv, rows, torch.randn(rows.T, 8 * 64, device="cuda").half()


def test_bad_page_ids_and_segments_are_reported_and_skipped():
    """A page id outside the arena or an inconsistent segment: a status bit, the other segments' results, nothing
    written for the bad one."""
    ctx, kv, rows, q = _small()
    good = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, good)
    assert ctx.status_poll() == 0
    x = torch.randn(rows.T, 12 * 64, device="cuda").half()
    arena = kv.arena.clone()
    for field, value in ((None, None), (2, 21), (2, -1), (3, -5), (3, 2 ** 31 - 2), (4, -1), (4, 2 ** 31 - 2), (5, 43), (1, -1), (1, 2 ** 31 - 1)):
        seg, ids = rows.dev.segs.clone(), rows.dev.page_ids.clone()
        if field is None:
            ids[3] = 64                                # some page of segment 1 (pages 0 - 1 are segment 0's)
        else:
            seg[1, field] = value
        bad = B.SegRows(seg, ids, rows.dev.row_seg, rows.dev.struct.max_q_len, rows.dev.struct.max_keys)
        out = torch.full_like(q, -3.0)
        ctx.kv8_attention(kv, 0, bad, q, out)
        assert ctx.status_poll() == 2, (field, value)
        keep = [0] + list(range(2, rows.T))
        assert torch.equal(out[keep], good[keep]) and torch.all(out[1] == -3.0), (field, value)
        if field is not None:
            q_out = torch.full_like(q, -3.0)
            ctx.kv8_append(kv, 0, bad, x, q_out)
            assert ctx.status_poll() == 4 and torch.all(q_out[1] == -3.0), (field, value)
            kv.arena.copy_(arena)
    ids = rows.dev.page_ids.clone()
    ids[2 + 43] = -7                                   # the page row 1 writes (position 700, page 43 of segment 1)
    ctx.kv8_append(kv, 0, B.SegRows(rows.dev.segs, ids, rows.dev.row_seg, 20, 701), x, torch.empty_like(q))
    assert ctx.status_poll() == 4


@pytest.mark.parametrize("bad", [-1, -2, -3, -2 ** 31, 400, 2 ** 31 - 1])
def test_no_page_id_outside_the_arena_is_followed(bad):
    """Any id outside the arena, at the first, a middle and the last page of a decode row (one split and several, any of the
    four warps, behind a warp's first 32 pages), of a row with two column tiles and of a chunk, and at the page that an
    append writes: reported, the segment's rows left alone, the other segments right."""
    cfg, ctx = context(16, 2, 64)
    kv = random_arena(cfg, 400, 3)
    segs = [(200, 1), (3000, 1), (90, 2), (100, 20), (17, 1), (480, 1), (30, 1)]
    rows = Rows(segs, 400, seed=3)
    q = torch.randn(rows.T, 16 * 64, device="cuda").half()
    good = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, good)
    assert ctx.status_poll() == 0
    for i, (p, n) in enumerate(segs[:6]):
        first, count = rows.table[i, 4], (p + n + 15) // 16
        for at in sorted({0, 1, 2, 3, min(40, count - 1), count // 2, count - 1} & set(range(count))):
            ids = rows.dev.page_ids.clone()
            ids[int(first) + at] = bad
            out = torch.full_like(q, -3.0)
            ctx.kv8_attention(kv, 0, B.SegRows(rows.dev.segs, ids, rows.dev.row_seg, 20, 3001), q, out)
            assert ctx.status_poll() == 2, (i, at)
            gone = torch.zeros(rows.T, dtype=torch.bool, device="cuda")
            gone[rows.start[i]:rows.start[i] + n] = True
            assert torch.all(out[gone] == -3.0) and torch.equal(out[~gone], good[~gone]), (i, at)
    arena = kv.arena.clone()
    x = torch.randn(rows.T, 20 * 64, device="cuda").half()
    for i, (p, n) in enumerate(segs):
        ids = rows.dev.page_ids.clone()
        ids[int(rows.table[i, 4]) + p // 16] = bad
        before = kv.codes()[0, rows.pages[i][p // 16]].view(torch.uint8).clone()
        ctx.kv8_append(kv, 0, B.SegRows(rows.dev.segs, ids, rows.dev.row_seg, 20, 3001), x, torch.empty_like(q))
        assert ctx.status_poll() == 4, i
        assert torch.equal(kv.codes()[0, rows.pages[i][p // 16]].view(torch.uint8), before), i
        kv.arena.copy_(arena)


def test_many_chunks_with_bad_pages():
    """Short chunks, two out of three of them with a page id outside the arena, several of those in a row for every
    block: none of their rows is written, all others are right."""
    cfg, ctx = context(8, 2, 64)
    kv = random_arena(cfg, 1100, 5)
    segs = [(i % 23, 5 + i % 12) for i in range(500)]  # 20 to 64 columns, one or two pages
    rows = Rows(segs, 1100, seed=6)
    q = torch.randn(rows.T, 8 * 64, device="cuda").half()
    good = torch.empty_like(q)
    ctx.kv8_attention(kv, 0, rows.dev, q, good)
    assert ctx.status_poll() == 0
    ids = rows.dev.page_ids.clone()
    bad = [i for i in range(500) if i // 150 % 3 != 1 and i % 7 < 5]
    first = rows.table[:, 4]
    ids[torch.from_numpy(first[bad]).long().cuda()] = 1100
    out = torch.full_like(q, -3.0)
    ctx.kv8_attention(kv, 0, B.SegRows(rows.dev.segs, ids, rows.dev.row_seg, 16, 38), q, out)
    assert ctx.status_poll() == 2
    gone = np.zeros(rows.T, dtype=bool)
    for i in bad:
        gone[rows.start[i]:rows.start[i] + segs[i][1]] = True
    gone = torch.from_numpy(gone).cuda()
    assert torch.all(out[gone] == -3.0) and torch.equal(out[~gone], good[~gone])


def test_rows_of_one_step_for_two_models():
    """The same SegRows in contexts that differ in their query heads only: each call has the workspace it needs."""
    rows = Rows([(2000, 1), (2300, 1)], 300, seed=1)
    for hq in (2, 16):
        cfg, ctx = context(hq, 2, 64)
        kv = random_arena(cfg, 300, 2)
        q = torch.randn(rows.T, hq * 64, device="cuda").half()
        out, alone = torch.empty_like(q), torch.empty_like(q)
        ctx.kv8_attention(kv, 0, rows.dev, q, out)
        ctx.kv8_attention(kv, 0, Rows(rows.segs, 300, seed=1).dev, q, alone)
        assert torch.equal(out, alone) and ctx.status_poll() == 0


def test_arena_of_the_caller():
    cfg, _ = context(8, 2, 64)
    n = B.kv8_arena_bytes(cfg, 4)
    kv = B.KvCache8(cfg, 4, arena=torch.zeros(n + 5, dtype=torch.uint8, device="cuda"))
    assert kv.codes().shape == (2, 4, 2, 32 * 64) and kv.scales().shape == (2, 4, 2, 2)
    for bad in (torch.zeros(n - 1, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.int8, device="cuda"),
                torch.zeros(n, dtype=torch.uint8), torch.zeros(2, n, dtype=torch.uint8, device="cuda"),
                torch.zeros(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            B.KvCache8(cfg, 4, arena=bad)
    with pytest.raises(B.HbError):                     # not 256-byte aligned
        B.KvCache8(cfg, 4, arena=torch.zeros(n + 16, dtype=torch.uint8, device="cuda")[16:])


def test_append_beyond_the_rotary_table_is_reported():
    ctx, kv, rows, q = _small()
    x = torch.randn(rows.T, 12 * 64, device="cuda").half()
    out = torch.full_like(q, -3.0)
    ctx.kv8_append(kv, 0, rows.dev, x, out, rope=B.Rope.table(700, 64, 1e4))
    assert ctx.status_poll() == 4 and torch.all(out[1] == -3.0) and not torch.any(out[0] == -3.0)


def test_refusals():
    cfg, ctx = context(8, 2, 64)
    _, kv, rows, q = _small()
    lib, P = B.lib, C.c_void_p
    qp = q.data_ptr()
    need = C.c_size_t()
    assert lib.hb_kv8_attention_workspace(C.byref(cfg), C.byref(rows.dev.struct), C.byref(need)) == 0 and need.value > 0
    ws = torch.empty(need.value + 256, dtype=torch.uint8, device="cuda")

    def attend(layer=0, kvh=kv.handle, r=rows.dev.struct, qa=qp, qs=512, o=qp + 0, os_=512, scale=0.0, w=ws.data_ptr(), wb=need.value):
        return lib.hb_kv8_attention(ctx.handle, kvh, layer, C.byref(r), P(qa), qs, P(o), os_, scale, P(w), wb, None)
    assert attend(layer=2) == -1 and attend(layer=-1) == -1 and attend(kvh=None) == -1
    assert attend(qa=qp + 8) == -1 and attend(o=qp + 2) == -1 and attend(qs=511) == -1 and attend(qs=504) == -1 and attend(os_=516) == -1
    assert attend(scale=-1.0) == -1 and attend(scale=float("nan")) == -1 and attend(scale=float("inf")) == -1
    assert attend(w=0) == -1 and attend(wb=need.value - 1) == -1 and attend(w=ws.data_ptr() + 16) == -1
    assert attend(qa=0) == -1 and attend(o=0) == -1
    kv16 = B.KvCache(cfg, 4)
    assert attend(kvh=kv16.handle) == -1
    for k, v in (("n_segs", -1), ("n_rows", -1), ("max_keys", -1), ("max_q_len", -1), ("n_page_ids", -1), ("segs", None),
                 ("page_ids", None), ("row_seg", None), ("segs", rows.dev.segs.data_ptr() + 4)):
        r = B.RowsStruct.from_buffer_copy(rows.dev.struct)
        setattr(r, k, v)
        assert attend(r=r) == -1, k
    for k, v in (("n_segs", 8193), ("n_rows", (1 << 26) + 1), ("max_keys", (1 << 30) + 1)):
        r = B.RowsStruct.from_buffer_copy(rows.dev.struct)
        setattr(r, k, v)
        assert attend(r=r) == -5, k

    def append(**kw):
        a = B.AppendArgs(qkv=qp, q_out=qp, qkv_stride=768, q_stride=512, norm_eps=1e-6, rope_rows=0, rot_dim=0, rope_layout=0)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.hb_kv8_append(ctx.handle, kv.handle, 0, C.byref(rows.dev.struct), C.byref(a), None)
    assert append(qkv=qp + 8) == -1 and append(q_out=qp + 4) == -1 and append(qkv_stride=760) == -1 and append(qkv_stride=772) == -1
    assert append(q_stride=504) == -1 and append(rot_dim=8) == -1 and append(rot_dim=80) == -1 and append(rot_dim=-16) == -1
    assert append(rot_dim=64) == -1 and append(rope_layout=2) == -1 and append(qkv=None) == -1 and append(q_out=None) == -1
    assert append(rot_dim=64, rope_cos=qp, rope_sin=qp + 4, rope_rows=10) == -1
    assert append(rot_dim=64, rope_cos=qp, rope_sin=qp, rope_rows=0) == -1
    assert append(q_gain=qp, norm_eps=-1.0) == -1 and append(k_gain=qp + 2) == -1 and append(k_gain=qp, norm_eps=float("nan")) == -1
    with pytest.raises(TypeError):
        ctx.kv8_attention(kv16, 0, rows.dev, q, torch.empty_like(q))
    with pytest.raises(ValueError):
        ctx.kv8_attention(kv, 0, rows.dev, q.float(), torch.empty_like(q))
    with pytest.raises(ValueError):
        ctx.kv8_attention(kv, 0, rows.dev, q[:-1], torch.empty_like(q))
    with pytest.raises(ValueError):
        ctx.kv8_attention(kv, 0, rows.dev, q.cpu(), torch.empty_like(q))
    with pytest.raises(ValueError):
        ctx.kv8_append(kv, 0, rows.dev, q, torch.empty_like(q))
    # the step refuses an 8-bit cache of another model
    assert ctx.status_poll() == 0


def test_rows_beyond_a_bound_of_zero_are_reported():
    """A segment with rows where the call says that there are none, or keys where it says that there are none."""
    ctx, kv, rows, q = _small()
    for max_q_len, max_keys in ((0, 701), (20, 0), (0, 0)):
        out = torch.full_like(q, -3.0)
        ctx.kv8_attention(kv, 0, B.SegRows(rows.dev.segs, rows.dev.page_ids, rows.dev.row_seg, max_q_len, max_keys), q, out)
        assert ctx.status_poll() == 2 and torch.all(out == -3.0), (max_q_len, max_keys)


def test_nothing_to_do():
    cfg, ctx = context(8, 2, 64)
    kv = random_arena(cfg, 4, 0)
    empty = Rows([], 4)
    z = torch.empty(0, 512, dtype=torch.float16, device="cuda")
    ctx.kv8_append(kv, 0, empty.dev, torch.empty(0, 768, dtype=torch.float16, device="cuda"), z)
    ctx.kv8_attention(kv, 0, empty.dev, z, z)
    rows = Rows([(5, 0), (0, 0)], 4, gap=2)            # segments without rows, rows of nobody
    q = torch.full((4, 512), 2.0, dtype=torch.float16, device="cuda")
    before = kv.arena.clone()
    ctx.kv8_append(kv, 0, rows.dev, torch.ones(4, 768, dtype=torch.float16, device="cuda"), q)
    ctx.kv8_attention(kv, 0, rows.dev, q, q)
    assert torch.all(q == 2.0) and torch.equal(kv.arena, before) and ctx.status_poll() == 0


def test_two_calls_at_once_on_two_streams():
    """The same context, two streams, no order between them: each call has its own workspace."""
    cfg, ctx = context(32, 8, 128)
    kv = random_arena(cfg, 1200, 4)
    sets = []
    for seed in range(2):
        rows = Rows([(3000 - 40 * seed, 1), (1500, 1), (900 + seed, 3), (2200, 1)], 1200, seed=seed)
        q = torch.randn(rows.T, 4096, device="cuda").half()
        want = torch.empty_like(q)
        ctx.kv8_attention(kv, 0, rows.dev, q, want)
        sets.append((rows, q, want))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(s[1]) for s in sets] for _ in range(20)]
    for o in outs:
        for st, (rows, q, _), out in zip(streams, sets, o):
            ctx.kv8_attention(kv, 0, rows.dev, q, out, stream=st)
    torch.cuda.synchronize()
    for o in outs:
        for (_, _, want), out in zip(sets, o):
            assert torch.equal(out, want)
    assert ctx.status_poll() == 0


def test_captured_step_follows_the_arrays():
    """Append and attention of a decode batch captured once and replayed while the segments advance by one token a
    step: bit for bit what eager calls give, over page and split borders."""
    cfg, ctx = context(8, 2, 128)
    starts = [5, 15, 500, 508, 1020]
    n_pages = 400
    rows = Rows([(p + 40, 1) for p in starts], n_pages, max_keys=1100)
    rope = B.Rope.table(1100, 128, 1e4)
    first = rows.dev.segs.clone()
    first[:, 3] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    x = torch.randn(12, 5, 12 * 128, device="cuda").half()
    results = []
    for captured in (False, True):
        kv = random_arena(cfg, n_pages, 4)
        rows.dev.segs.copy_(first)
        xin = torch.empty_like(x[0])
        q, out = torch.empty(5, 1024, dtype=torch.float16, device="cuda"), torch.empty(5, 1024, dtype=torch.float16, device="cuda")

        def step():
            ctx.kv8_append(kv, 1, rows.dev, xin, q, rope=rope)
            ctx.kv8_attention(kv, 1, rows.dev, q, out)
        graph = None
        if captured:
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
            torch.cuda.synchronize()
        got = []
        for t in range(12):
            xin.copy_(x[t])
            graph.replay() if captured else step()
            got.append(out.clone())
            rows.dev.segs[:, 3] += 1
        results.append((got, kv.arena.clone()))
    assert all(torch.equal(a, b) for a, b in zip(results[0][0], results[1][0]))
    assert torch.equal(results[0][1], results[1][1]) and ctx.status_poll() == 0


def test_two_captured_graphs_share_nothing():
    """Two graphs captured from the same pool and replayed one after the other, twice."""
    ctx, kv, rows, q = _small(1, 96)
    rows2 = Rows([(650, 1), (600, 2)], 96, seed=7)
    q2 = torch.randn(rows2.T, 512, device="cuda").half()
    want, want2, out, out2 = torch.empty_like(q), torch.empty_like(q2), torch.empty_like(q), torch.empty_like(q2)
    ctx.kv8_attention(kv, 0, rows.dev, q, want)
    ctx.kv8_attention(kv, 0, rows2.dev, q2, want2)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        ctx.kv8_attention(kv, 0, rows.dev, q, out)
    with torch.cuda.graph(g2, pool=g1.pool()):
        ctx.kv8_attention(kv, 0, rows2.dev, q2, out2)
    for _ in range(2):
        out.zero_(); out2.zero_()
        g1.replay(); g2.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want2)


def test_prompt_in_chunks_then_decode():
    """A run as a program makes it: two prompts appended and attended to in chunks, then decode steps, over two layers.
    Against the plain statement on full-precision keys and values the error is the cache's: every key and value is
    off by at most 2^-4 of itself (plus half the smallest step of its block)."""
    hq, hkv, dh, eps = 8, 2, 128, 1e-6
    cfg, ctx = context(hq, hkv, dh)
    kv = B.KvCache8(cfg, 64, fill=0xFF)
    rope = B.Rope.table(256, dh, 1e4, B.ROPE_HALVES)
    cos, sin = B.rope_table(256, dh, 1e4)
    lens = [70, 37]
    pages = [kv.alloc(8), kv.alloc(6)]
    r = np.random.default_rng(2)
    x16 = [[r.standard_normal((n + 8, (hq + 2 * hkv) * dh)).astype(np.float16) for n in lens] for _ in range(2)]
    gain = (1 + 0.1 * torch.randn(dh, generator=torch.Generator().manual_seed(3))).bfloat16()
    done = [0, 0]
    plan = [(32, 16), (32, 21), (6, 1)] + [(1, 1)] * 7     # the second request decodes while the first still prefills
    while any(plan):
        take, plan = plan[0], plan[1:]
        table, row_seg, at, ids = [], [], 0, []
        for i, n in enumerate(take):
            table.append([0, at, n, done[i], len(ids), len(pages[i]), -1, 0, 0, -1, -1, 0])
            row_seg += [i] * n
            ids += pages[i]
            at += n
        up = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        rows = B.SegRows(up(table), up(ids), up(row_seg), max(take), max(d + n for d, n in zip(done, take)))
        for layer in range(2):
            x = np.concatenate([x16[layer][i][done[i]:done[i] + n] for i, n in enumerate(take)])
            q, out = (torch.empty(at, hq * dh, dtype=torch.float16, device="cuda") for _ in range(2))
            ctx.kv8_append(kv, layer, rows, torch.from_numpy(x).cuda(), q, rope=rope, q_norm=gain.cuda(), k_norm=gain.cuda(), norm_eps=eps)
            ctx.kv8_attention(kv, layer, rows, q, out)
            got, row = out.cpu().numpy().astype(np.float64), 0
            for i, n in enumerate(take):
                y = x16[layer][i][:done[i] + n].astype(np.float64).reshape(-1, hq + 2 * hkv, dh)
                y[:, :hq + hkv] = O.rmsnorm_head(y[:, :hq + hkv], gain.double().numpy(), eps)
                for j in range(len(y)):
                    y[j, :hq + hkv] = O.rotate(y[j, :hq + hkv], cos[j], sin[j], True)
                ref, mass = O.attend(y[done[i]:, :hq], y[:, hq:hq + hkv], y[:, hq + hkv:], done[i], dh ** -0.5)
                # |dk| <= 2^-4 |k|: a score moves by at most 2^-4 sum |q||k| / sqrt(dh), a weight by twice that, a value by 2^-4
                ds = 2.0 ** -4 * np.abs(y[done[i]:, :hq]).reshape(n, hkv, hq // hkv, dh)
                ds = np.einsum("nhgd,khd->nhgk", ds, np.abs(y[:, hq:hq + hkv])).max(axis=3).reshape(n, hq, 1) * dh ** -0.5
                err = np.abs(got[row:row + n].reshape(n, hq, dh) - ref)
                assert np.all(err <= (np.expm1(2 * ds) + 2.0 ** -4 + 2.0 ** -9) * mass * 1.1 + 1e-2), (layer, done, np.max(err))
                assert np.sqrt(np.mean(err ** 2)) <= 0.06 * np.sqrt(np.mean(mass ** 2))
                row += n
        done = [d + n for d, n in zip(done, take)]
    assert ctx.status_poll() == 0
