"""Products with bias, activation and residual, dense and grouped, through the C-ABI against float64."""
import math

import pytest
import torch

from paper_2609_25405_b200 import binding as B
from tests.dense_util import ACTS, E4M3, check, ctx, gen, linear64, operand, status, strided

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _case(m, n, k, ab, c_t, seed=0, groups=1, act="none", gated=False, bias=False, residual=None, scales=None, std=0.05):
    g = gen(seed + m * 31 + n * 7 + k)
    a, w = operand(g, m, k, ab), operand(g, groups * n, k, ab, 1.0 if ab == E4M3 else std)
    scales = ab == E4M3 if scales is None else scales
    cols = n // 2 if gated else n
    unit = 0.01 if ab == E4M3 else 1.0
    return dict(a=a, w=w.unflatten(0, (groups, n)), a_scale=unit * (0.5 + torch.rand(m, generator=g, device="cuda")) if scales else None,
                w_scale=unit * (std if ab == E4M3 else 1.0) * (0.5 + torch.rand(groups, n, generator=g, device="cuda")) if scales else None,
                bias=torch.randn(groups, n, generator=g, device="cuda") if bias else None, act=act, gated=gated,
                residual=None if residual is None else (2 * torch.randn(m, cols, generator=g, device="cuda")).to(residual), c_t=c_t, cols=cols)


def _one(v):
    return None if v is None else v[0]


def _run(c, out):
    ctx().linear(c["a"], c["w"][0], out, a_scale=c["a_scale"], w_scale=_one(c["w_scale"]), bias=_one(c["bias"]), act=ACTS[c["act"]],
                 gated=c["gated"], residual=c["residual"])
    return out


def _want(c, rows=slice(None), e=0):
    pick = lambda v: None if v is None else v[rows]   # noqa: E731
    of = lambda v: None if v is None else v[e]        # noqa: E731
    return linear64(c["a"][rows], c["w"][e], pick(c["a_scale"]), of(c["w_scale"]), of(c["bias"]), c["act"], c["gated"], pick(c["residual"]),
                    c["c_t"])


SIZES = [(1, 1, 1), (1, 8, 16), (1, 130, 4096), (2, 128, 64), (3, 5, 7), (15, 129, 127), (16, 256, 128), (17, 33, 129), (31, 1000, 255),
         (33, 300, 1000), (48, 128, 640), (63, 640, 65), (64, 128, 256), (65, 500, 500), (100, 1030, 300), (127, 127, 128), (128, 384, 96), (129, 256, 2049),
         (200, 2100, 80), (255, 257, 300), (256, 512, 1024), (257, 1026, 130), (513, 770, 384), (1000, 4100, 200), (2048, 1100, 128),
         (1, 28674, 64), (5, 96, 14336), (700, 64, 4096), (4100, 40, 40)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("ab,c_t", [(E4M3, F16), (E4M3, F32), (F16, F16), (F16, F32), (BF16, BF16)])
def test_products_of_every_size(m, n, k, ab, c_t):
    c = _case(m, n, k, ab, c_t)
    out = _run(c, torch.full((m, n), 9.0, device="cuda", dtype=c_t))
    check(out, *_want(c))
    assert status() == 0


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("bias,residual", [(False, None), (True, F32), (True, F16), (False, BF16)])
@pytest.mark.parametrize("m", [3, 70, 600])
def test_epilogues(m, act, gated, bias, residual):
    for ab, c_t, n in ((E4M3, F16, 520), (F16, F32, 264), (BF16, BF16, 1034), (E4M3, F32, 130), (F16, F16, 26)):
        c = _case(m, n, 200, ab, c_t, act=act, gated=gated, bias=bias, residual=residual, std=0.3)
        check(_run(c, torch.full((m, c["cols"]), 9.0, device="cuda", dtype=c_t)), *_want(c))
    assert status() == 0


@pytest.mark.parametrize("ab", [F16, BF16])
def test_scales_of_16_bit_operands(ab):
    c = _case(37, 200, 100, ab, F32, scales=True)
    check(_run(c, torch.empty(37, 200, device="cuda")), *_want(c))


@pytest.mark.parametrize("m", [1, 40, 130, 520])
@pytest.mark.parametrize("c_t", [F16, F32, BF16])
def test_outputs_in_wider_matrices(m, c_t):
    """Output and residual at every alignment, in place too; nothing beside the columns is written."""
    for n, pitch, off in ((96, 128, 0), (96, 100, 4), (96, 99, 1), (95, 97, 2), (130, 131, 1)):
        for gated in (False, True):
            if gated and n % 2:
                continue
            c = _case(m, n, 72, F16, c_t, gated=gated, act="silu" if gated else "none", residual=c_t)
            want = _want(c)
            out, whole = strided(m, c["cols"], c_t, pitch, off, fill=5.0)
            out.copy_(c["residual"])
            c["residual"] = out
            check(_run(c, out), *want)
            out[:] = 5.0
            assert bool((whole == 5.0).all())


def test_operands_in_wider_matrices():
    """Rows with a pitch, columns from an offset of 16 bytes; what lies beside them is NaN."""
    g = gen(1)
    for ab, off, pitch in ((E4M3, 16, 400), (F16, 8, 240), (BF16, 24, 248)):
        a, _ = strided(90, 200, ab, pitch, off)
        w, _ = strided(70, 200, ab, pitch, off)
        for t in (a, w):
            t.copy_(torch.randn(*t.shape, generator=g, device="cuda").to(ab))
        out = torch.empty(90, 70, device="cuda")
        ctx().linear(a, w, out)
        check(out, *linear64(a, w))


def test_nan_and_infinity_stay_in_their_rows_and_columns():
    for m in (20, 300):
        c = _case(m, 300, 256, F16, F32)
        c["a"][3, 5] = math.nan
        c["a"][7, 255] = math.inf
        c["w"][0, 11, 0] = math.nan
        out = _run(c, torch.empty(m, 300, device="cuda"))
        y, bound = _want(c)
        assert bool(torch.isnan(out[3]).all()) and bool(torch.isnan(out[:, 11]).all())
        keep = torch.ones(m, 300, dtype=torch.bool, device="cuda")
        keep[3] = keep[7] = False
        keep[:, 11] = False
        check(out[keep], y[keep], bound[keep])
        assert not torch.isfinite(out[7]).any()


def test_fp16_outputs_saturate():
    a, w = torch.full((2, 64), 100.0, device="cuda").half(), torch.full((16, 64), 100.0, device="cuda").half()
    w[1] = -100
    out = torch.empty(2, 16, device="cuda", dtype=F16)
    ctx().linear(a, w, out)
    assert float(out[0, 0]) == 65504 and float(out[1, 1]) == -65504
    wide = torch.empty(2, 16, device="cuda", dtype=BF16)
    ctx().linear(a, w, wide)
    assert float(wide[0, 0]) == 638976.0


def test_activations_far_out():
    """z of +-200 and beyond: no NaN from an exponential that overflows."""
    a = torch.zeros(8, 16, device="cuda", dtype=F16)
    a[:, 0] = torch.tensor([-60000.0, -200.0, -89.0, -20.0, 20.0, 89.0, 200.0, 60000.0], device="cuda")
    w = torch.zeros(8, 16, device="cuda", dtype=F16)
    w[:, 0] = 1
    for act in ACTS:
        out = torch.empty(8, 8, device="cuda")
        ctx().linear(a, w, out, act=ACTS[act])
        check(out, *linear64(a, w, act=act))


def test_equal_calls_give_equal_bits():
    for m, n, k, ab in ((5, 700, 4096, E4M3), (90, 600, 3000, F16), (700, 900, 1000, E4M3)):
        c = _case(m, n, k, ab, F32)
        first = _run(c, torch.empty(m, n, device="cuda"))
        for _ in range(5):
            assert torch.equal(_run(c, torch.empty(m, n, device="cuda")), first)


def test_captured_replayed_and_on_two_streams():
    cs = [_case(m, 800, 2048, ab, F16) for m, ab in ((4, E4M3), (300, F16))]
    want = [_want(c) for c in cs]
    outs = [torch.empty(c["a"].shape[0], 800, device="cuda", dtype=F16) for c in cs]
    graph = torch.cuda.CUDAGraph()
    for c, o in zip(cs, outs):
        _run(c, o)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for c, o in zip(cs, outs):
            _run(c, o)
    for o in outs:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        check(o, *w)
    streams = [torch.cuda.Stream() for _ in range(2)]
    more = [[torch.empty_like(o) for _ in range(10)] for o in outs]
    torch.cuda.synchronize()
    for i in range(10):
        for c, o, s in zip(cs, more, streams):
            ctx().linear(c["a"], c["w"][0], o[i], a_scale=c["a_scale"], w_scale=_one(c["w_scale"]), stream=s)
    torch.cuda.synchronize()
    for o, w in zip(more, want):
        for x in o:
            check(x, *w)
    assert status() == 0


# ---- grouped -----------------------------------------------------------------------------------------------------


def _run_grouped(c, start, out):
    ctx().linear_grouped(c["a"], c["w"], torch.tensor(start, dtype=torch.int32, device="cuda"), out, a_scale=c["a_scale"], w_scale=c["w_scale"],
                         bias=c["bias"], act=ACTS[c["act"]], gated=c["gated"], residual=c["residual"])
    return out


def _check_grouped(c, start, out, fill=9.0):
    done = torch.zeros(out.shape[0], dtype=torch.bool, device="cuda")
    for e in range(len(start) - 1):
        lo, hi = start[e], start[e + 1]
        if max([0] + start[:e]) <= lo < hi <= out.shape[0]:
            check(out[lo:hi], *_want(c, slice(lo, hi), e))
            done[lo:hi] = True
    assert bool((out[~done].float() == fill).all())


STARTS = [[0, 5], [0, 0, 3, 3, 40], [2, 2, 7, 30, 31, 60], [0, 129, 130, 386, 500], [0] * 9 + [70] * 3, [1, 1, 1], [0, 16, 32, 48, 64, 80], [0, 700, 1400],
          [10, 300, 301, 302, 700, 1000]]


@pytest.mark.parametrize("start", STARTS)
@pytest.mark.parametrize("ab,c_t", [(E4M3, F16), (F16, F32), (BF16, BF16)])
def test_groups_of_every_size(start, ab, c_t):
    """Empty groups, groups that end inside a tile, rows before the first and behind the last group."""
    m = start[-1] + 7
    for n, k in ((130, 100), (520, 64), (64, 1000)):
        c = _case(m, n, k, ab, c_t, groups=len(start) - 1, bias=True, act="silu", residual=c_t)
        _check_grouped(c, start, _run_grouped(c, start, torch.full((m, n), 9.0, device="cuda", dtype=c_t)))
    assert status() == 0


@pytest.mark.parametrize("groups", [1, 33, 200, 512])
def test_many_groups(groups):
    g = torch.Generator().manual_seed(groups)
    counts = torch.randint(0, 9, (groups,), generator=g)
    start = [0] + torch.cumsum(counts, 0).tolist()
    c = _case(start[-1] + 1, 48, 80, E4M3, F16, groups=groups, gated=True, act="gelu")
    _check_grouped(c, start, _run_grouped(c, start, torch.full((start[-1] + 1, 24), 9.0, device="cuda", dtype=F16)))
    assert status() == 0


# (rows, n, k, operands, groups): between them they take every kernel: few rows, tiles of 32 to 128 tokens alone and shared by four and
# eight CTAs, pairs; long sums onto fp32, short products
KERNELS = [(9, 3333, 586, F16, 0), (18, 2691, 539, F16, 0), (2, 2415, 526, F16, 3), (18, 2480, 72, F16, 0), (16, 6144, 2048, E4M3, 0), (5, 40, 4000, E4M3, 3), (1253, 16, 885, F16, 20), (18, 6240, 9444, E4M3, 0), (169, 2325, 3993, F16, 0), (863, 155, 3069, F16, 23),
           (2485, 151, 4260, F16, 0), (2032, 144, 4935, F16, 22), (66, 16, 1459, F16, 0), (133, 21, 1670, F16, 1), (313, 36, 1797, F16, 1),
           (1666, 1286, 799, F16, 0), (336, 956, 1610, F16, 18), (4100, 4100, 700, F16, 0), (520, 5000, 3000, E4M3, 0), (1300, 2570, 1030, BF16, 0)]


@pytest.mark.parametrize("m,n,k,ab,groups", KERNELS)
@pytest.mark.parametrize("c_t,gated,residual", [(F32, False, F32), (F16, True, None), (F32, True, F16)])
def test_every_kernel(m, n, k, ab, groups, c_t, gated, residual):
    n += n % 2 if gated else 0
    c = _case(m, n, k, ab, c_t, groups=max(groups, 1), act="silu" if gated else "none", gated=gated, bias=True, residual=residual)
    out = torch.full((m, c["cols"]), 9.0, device="cuda", dtype=c_t)
    if not groups:
        check(_run(c, out), *_want(c))
    else:
        cuts = torch.randint(0, m + 1, (groups - 1,), generator=torch.Generator().manual_seed(m)).sort()[0].tolist()
        start = [0] + cuts + [m]
        _check_grouped(c, start, _run_grouped(c, start, out))
    assert status() == 0


def test_one_group_is_the_plain_product():
    for m, ab in ((5, E4M3), (300, F16)):
        c = _case(m, 520, 300, ab, F32)
        check(_run_grouped(c, [0, m], torch.empty(m, 520, device="cuda")), *_want(c))


def test_weights_with_space_between_groups():
    c = _case(50, 40, 64, F16, F32, groups=3)
    wide = torch.full((3, 48, 80), math.nan, device="cuda", dtype=F16)
    wide[:, :40, :64] = c["w"]
    c["w"] = wide[:, :40, :64]
    start = [0, 20, 30, 50]
    _check_grouped(c, start, _run_grouped(c, start, torch.empty(50, 40, device="cuda")))


@pytest.mark.parametrize("start", [[0, 10, 5, 20], [-1, 5, 10, 20], [0, 10, 21, 30], [0, 2 ** 31 - 1, 5, 20], [3, -2 ** 31, 4, 9]])
def test_bad_bounds_are_reported_and_skipped(start):
    c = _case(20, 64, 64, F16, F32, groups=3)
    out = _run_grouped(c, start, torch.full((20, 64), 9.0, device="cuda"))
    assert status() == 1024
    _check_grouped(c, start, out)


def test_bounds_are_read_when_the_graph_runs():
    c = _case(400, 200, 128, E4M3, F16, groups=4)
    start = torch.tensor([0, 100, 200, 300, 400], dtype=torch.int32, device="cuda")
    out = torch.full((400, 200), 9.0, device="cuda", dtype=F16)
    call = lambda: ctx().linear_grouped(c["a"], c["w"], start, out, a_scale=c["a_scale"], w_scale=c["w_scale"])   # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for bounds in ([0, 0, 0, 0, 400], [7, 390, 391, 391, 399], [0, 1, 2, 3, 4]):
        start.copy_(torch.tensor(bounds, dtype=torch.int32))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        _check_grouped(c, bounds, out)


# ---- together ----------------------------------------------------------------------------------------------------


def test_feed_forward_of_experts_in_8_bits():
    """norm -> gather by expert -> gate/up -> 8 bits -> down, each stage against the definition on the stage's own inputs."""
    T, d, F, E = 37, 256, 512, 4
    g = gen(12)
    x, r = torch.randn(T, d, generator=g, device="cuda").half(), torch.randn(T, d, generator=g, device="cuda")
    y = torch.empty(T, d, device="cuda", dtype=F16)
    ctx().norm(x, torch.ones(d, device="cuda").bfloat16(), y, residual=r, sum_out=r)
    expert = torch.randint(E, (T,), generator=g, device="cuda")
    order = torch.argsort(expert, stable=True).to(torch.int32)
    start = torch.searchsorted(expert[order.long()], torch.arange(E + 1, device="cuda")).to(torch.int32)
    codes, scale = torch.empty(T, d, device="cuda", dtype=E4M3), torch.empty(T, device="cuda")
    ctx().quant_rows(y, codes, scale, index=order)
    up = _case(T, 2 * F, d, E4M3, F16, groups=E, gated=True, act="silu")
    up.update(a=codes, a_scale=scale)
    inner = torch.empty(T, F, device="cuda", dtype=F16)
    ctx().linear_grouped(codes, up["w"], start, inner, a_scale=scale, w_scale=up["w_scale"], act=B.ACT_SILU, gated=True)
    _check_grouped(up, start.tolist(), inner)
    c2, s2 = torch.empty(T, F, device="cuda", dtype=E4M3), torch.empty(T, device="cuda")
    ctx().quant_rows(inner, c2, s2)
    down = _case(T, d, F, E4M3, F32, groups=E)
    down.update(a=c2, a_scale=s2, residual=r[order.long()])
    out = torch.empty(T, d, device="cuda")
    ctx().linear_grouped(c2, down["w"], start, out, a_scale=s2, w_scale=down["w_scale"], residual=down["residual"])
    _check_grouped(down, start.tolist(), out)
    assert status() == 0


def test_refusals():
    a, w = torch.zeros(4, 64, device="cuda", dtype=F16), torch.zeros(8, 64, device="cuda", dtype=F16)
    o = torch.zeros(4, 8, device="cuda")
    s4 = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    bad = [lambda: ctx().linear(a, w.bfloat16(), o), lambda: ctx().linear(a.float(), w.float(), o), lambda: ctx().linear(a[:, :56], w, o),
           lambda: ctx().linear(a, w, o[:3]), lambda: ctx().linear(a, w, o[:, :7]), lambda: ctx().linear(a, w, o, gated=True),
           lambda: ctx().linear(a, w[:7], o[:, :3], gated=True), lambda: ctx().linear(a, w, o.to(E4M3)),
           lambda: ctx().linear(a, w, o, residual=o[:, :4]), lambda: ctx().linear(a, w, o, residual=w[:4, :8].to(E4M3)),
           lambda: ctx().linear(a, w, o, a_scale=torch.zeros(3, device="cuda")), lambda: ctx().linear(a, w, o, bias=torch.zeros(8, device="cuda").half()),
           lambda: ctx().linear(a, w, o, act=5), lambda: ctx().linear(a, w, o, act=-1), lambda: ctx().linear(a.cpu(), w, o),
           lambda: ctx().linear(a[:, 1:], w[:, 1:], o),                        # rows off 16-byte boundaries
           lambda: ctx().linear(torch.zeros(4, 65, device="cuda", dtype=F16)[:, :64], w, o),
           lambda: ctx().linear(a, w[:1].expand(8, 64), o), lambda: ctx().linear(a, w, o[:1].expand(4, 8)),
           lambda: ctx().linear_grouped(a, w, s4, o), lambda: ctx().linear_grouped(a, w[None], None, o),
           lambda: ctx().linear_grouped(a, w[None], s4[:1], o), lambda: ctx().linear_grouped(a, w[None].expand(2, 8, 64), torch.zeros(3, dtype=torch.int32, device="cuda"), o),
           lambda: ctx().linear_grouped(a, w[None], s4.long(), o), lambda: ctx().linear_grouped(a, w[None], s4, o, bias=torch.zeros(9, device="cuda")),
           lambda: ctx().linear_grouped(a, torch.zeros(513, 8, 64, device="cuda", dtype=F16), torch.zeros(514, dtype=torch.int32, device="cuda"), o)]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, B.HbError)):
            f()
            raise AssertionError(i)
    ctx().linear(a[:0], w, o[:0])
    ctx().linear_grouped(a[:0], w[None], torch.zeros(2, dtype=torch.int32, device="cuda"), o[:0])
    assert status() == 0
