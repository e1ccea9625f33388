"""Norm with residual addition and rows to 8 bits through the C-ABI against float64."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2609_25405_b200 import binding as B
from tests.dense_util import E4M3, ctx, e4m3_64, gen, status, strided

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _norm64(x, residual, gain, eps):
    s = x.double() + (0 if residual is None else residual.double())
    y = s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt()
    return s, y if gain is None else y * gain.double()


def _check_rows(y, y64, scale=None):
    """fp32 inside: the mean of d squares is off by at most (log2 d + 4) 2^-24 in trees and chains of 32, half of that under the
    root, rsqrt 2^-22, two products 2^-24 each, s itself 2^-24: 2^-20 of |y| together; then the output's half step."""
    inner = y64.abs() * 2.0 ** -20 + 1e-37
    if scale is None:
        half = torch.finfo(y.dtype).eps / 2
        tol = inner + y64.abs() * half * (1 + 2.0 ** -20) + (2.0 ** -25 if y.dtype == F16 else 0.0)
        assert bool(((y.double() - y64).abs() <= tol).all())
        return
    top = y64.abs().amax(dim=1).clamp(min=2.0 ** -100)
    assert bool(((scale.double() - top / 448).abs() <= top / 448 * 2.0 ** -19).all())
    # a code is off by half an e4m3 step of the value over the scale: 2^-4 of the value, at least 2^-10 of the scale's unit
    v, unit = y.double() * scale.double()[:, None], scale.double()[:, None]
    tol = (y64.abs() * 2.0 ** -4).maximum(unit * 2.0 ** -10) * (1 + 2.0 ** -18) + y64.abs() * 2.0 ** -19
    assert bool(((v - y64).abs() <= tol).all())
    # and is the nearest one wherever the value over the scale is not within 2^-18 of a border
    u = (y64 / unit).cpu().numpy()
    lo, hi = e4m3_64(np.clip(u * (1 - 2.0 ** -18), -448, 448)), e4m3_64(np.clip(u * (1 + 2.0 ** -18), -448, 448))
    c = y.double().cpu().numpy()
    assert np.all((c == lo) | (c == hi))


SIZES = [(1, 1), (3, 7), (9, 8), (5, 64), (1, 255), (17, 256), (8, 257), (2, 1000), (3, 1024), (70, 1032), (4, 2048), (2, 2049), (5, 2056),
         (3, 4096), (1, 4104), (2, 8191), (3, 8192), (2, 8200), (2, 14336), (1, 16384), (2, 16392), (1, 20001), (1, 32767), (2, 32768)]


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("x_t,r_t,y_t", [(F16, F32, E4M3), (F32, None, E4M3), (BF16, BF16, BF16), (F32, F16, F32), (F16, F16, F16),
                                         (BF16, None, F16), (F16, None, E4M3), (F32, F32, BF16)])
def test_norm_rows_of_every_size(rows, d, x_t, r_t, y_t):
    g = gen(rows * 100003 + d)
    x = (torch.randn(rows, d, generator=g, device="cuda") * 3).to(x_t)
    r = None if r_t is None else torch.randn(rows, d, generator=g, device="cuda").to(r_t)
    gain = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).bfloat16() if d % 3 else None
    y = torch.empty(rows, d, device="cuda", dtype=y_t)
    scale = torch.full((rows,), 99.0, device="cuda") if y_t == E4M3 else None
    s = None if r is None else torch.empty_like(r)
    ctx().norm(x, gain, y, residual=r, sum_out=s, y_scale=scale, eps=1e-5)
    s64, y64 = _norm64(x, r, gain, 1e-5)
    _check_rows(y, y64, scale)
    if r is not None:
        assert torch.equal(s, (x.float() + r.float()).to(r_t))   # one fp32 addition, rounded once
    assert status() == 0


@pytest.mark.parametrize("y_t", [E4M3, F16, F32])
def test_norm_views_in_wider_matrices(y_t):
    """Strides and offsets on and off 16-byte boundaries give the same values; nothing beside the rows is written."""
    g = gen(5)
    rows, d = 6, 1000
    base = torch.randn(rows, d, generator=g, device="cuda").half()
    res = torch.randn(rows, d, generator=g, device="cuda")
    gain = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16()
    ref = None
    for pitch, off in ((1000, 0), (1024, 8), (1024, 16), (1001, 1), (1013, 3), (1040, 32)):
        x, _ = strided(rows, d, F16, pitch, off)
        r, r_all = strided(rows, d, F32, pitch, off, fill=7.0)
        y, y_all = strided(rows, d, y_t, pitch, off, fill=7.0)
        x.copy_(base)
        r.copy_(res)
        scale = torch.empty(rows, device="cuda") if y_t == E4M3 else None
        ctx().norm(x, gain, y, residual=r, sum_out=r, y_scale=scale, eps=1e-5)   # the sum in place
        _check_rows(y, _norm64(base, res, gain, 1e-5)[1], scale)
        got = (y.float().clone(), r.clone())
        y[:] = 7.0
        r[:] = 7.0
        assert bool((y_all.float() == 7.0).all()) and bool((r_all == 7.0).all())
        ref = got if ref is None else ref
        if off % 8 == 0 and pitch % 8 == 0:
            assert torch.equal(got[0], ref[0])
        assert torch.equal(got[1], ref[1])


@pytest.mark.parametrize("d", [3, 200, 2000, 8000, 8001, 20000])
@pytest.mark.parametrize("x_t,r_t,y_t", [(F16, F32, E4M3), (F32, BF16, F16), (BF16, None, F32)])
def test_norm_of_arrays_aligned_differently(d, x_t, r_t, y_t):
    """Every array at an offset and stride of its own: no access of several elements fits them all."""
    g = gen(d)
    x, _ = strided(5, d, x_t, d + 3, 1)
    x.copy_(torch.randn(5, d, generator=g, device="cuda"))
    r = r_all = None
    if r_t is not None:
        r, r_all = strided(5, d, r_t, d + 6, 2, fill=7.0)
        r.copy_(torch.randn(5, d, generator=g, device="cuda"))
    y, y_all = strided(5, d, y_t, d + 8, 5, fill=7.0)
    gain = (1 + 0.1 * torch.randn(d + 1, generator=g, device="cuda")).bfloat16()[1:]
    scale = torch.empty(5, device="cuda") if y_t == E4M3 else None
    _, want = _norm64(x, r, gain, 1e-5)
    ctx().norm(x, gain, y, residual=r, sum_out=r, y_scale=scale, eps=1e-5)
    _check_rows(y, want, scale)
    y.copy_(torch.full((5, d), 7.0, device="cuda").to(y_t))
    assert bool((y_all.float() == 7.0).all())
    if r is not None:
        r.fill_(7.0)
        assert bool((r_all == 7.0).all())


def test_norm_in_place():
    g = gen(8)
    x = torch.randn(33, 2048, generator=g, device="cuda").bfloat16()
    want = torch.empty_like(x)
    ctx().norm(x, None, want)
    ctx().norm(x, None, x)
    assert torch.equal(x, want)


@pytest.mark.parametrize("d", [64, 1000, 4096, 9001])
def test_norm_of_odd_values(d):
    """Zeros, an infinity, a NaN, values whose squares overflow, values near the smallest."""
    x = torch.ones(6, d, device="cuda")
    x[0] = 0
    x[1, d // 2] = math.inf
    x[2, d - 1] = math.nan
    x[3] = 1e30
    x[4] = 1e-42
    y, scale = torch.empty(6, d, device="cuda", dtype=E4M3), torch.empty(6, device="cuda")
    ctx().norm(x, None, y, y_scale=scale, eps=0.0 if d == 64 else 1e-5)
    v = y.float() * scale[:, None]
    if d != 64:
        assert bool((v[0] == 0).all()) and float(scale[0]) == np.float32(2.0 ** -100) / np.float32(448)
    for r in (1, 2):
        assert math.isnan(scale[r]) and bool(torch.isnan(y[r].float()).all())
    assert bool((v[3] == 0).all())         # the mean square is infinite, as in fp32 by hand
    assert bool(torch.isfinite(v[5]).all())
    assert float((v[5] - 1).abs().max()) < 1e-4
    y16 = torch.empty(6, d, device="cuda", dtype=F16)
    x[5] = 1e-3
    x[5, 0] = 60000.0
    ctx().norm(x, torch.full((d,), 3e4, device="cuda").bfloat16(), y16, eps=1e-5)
    assert float(y16[5, 0]) == 65504.0 and bool(torch.isnan(y16[2]).all())
    assert status() == 0


@pytest.mark.parametrize("x_t", [F32, F16, BF16])
@pytest.mark.parametrize("rows,d", [(1, 1), (5, 8), (7, 100), (40, 1024), (33, 1500), (64, 4096), (9, 5001), (3, 14336), (2, 32768)])
def test_quant_rows(rows, d, x_t):
    g = gen(rows * 7 + d)
    x = (torch.randn(rows, d, generator=g, device="cuda") * torch.logspace(-3, 3, rows, device="cuda")[:, None]).to(x_t)
    codes, scale = torch.empty(rows, d, device="cuda", dtype=E4M3), torch.empty(rows, device="cuda")
    ctx().quant_rows(x, codes, scale)
    _check_rows(codes, x.double(), scale)
    index = torch.randint(rows, (2 * rows + 1,), generator=g, device="cuda", dtype=torch.int32)   # the same row twice
    c2, s2 = torch.empty(2 * rows + 1, d, device="cuda", dtype=E4M3), torch.empty(2 * rows + 1, device="cuda")
    ctx().quant_rows(x, c2, s2, index=index)
    assert torch.equal(c2.float(), codes[index.long()].float()) and torch.equal(s2, scale[index.long()])


@pytest.mark.parametrize("x_t", [F32, F16])
@pytest.mark.parametrize("d", [5, 61, 1000, 1001, 4095, 14335, 32760, 32765, 32767])
def test_quant_of_rows_off_every_boundary(d, x_t):
    """Source rows and codes at offsets and strides that have nothing in common; nothing beside the rows is written."""
    g = gen(d)
    for x_pitch, x_off, c_pitch, c_off in ((d + 3, 1, d + 5, 2), (d + 8, 0, d + 1, 1), (d + 1, 1, d + 16, 3)):
        x, _ = strided(7, d, x_t, x_pitch, x_off)
        x.copy_(torch.randn(7, d, generator=g, device="cuda"))
        c, whole = strided(5, d, E4M3, c_pitch, c_off, fill=3.0)
        index = torch.tensor([6, 0, 3, 3, 1], dtype=torch.int32, device="cuda")
        scale = torch.empty(5, device="cuda")
        ctx().quant_rows(x, c, scale, index=index)
        _check_rows(c, x.double()[index.long()], scale)
        c.copy_(torch.full((5, d), 3.0, device="cuda").to(E4M3))
        assert bool((whole.float() == 3.0).all())


@pytest.mark.parametrize("d", [96, 2048, 6001])
def test_quant_index_that_names_no_row(d):
    """Negative: the row stays; beyond the source: the row stays and the call is reported."""
    x = torch.randn(4, d, device="cuda")
    codes, scale = torch.full((5, d), 2.0, device="cuda").to(E4M3), torch.full((5,), -3.0, device="cuda")
    ctx().quant_rows(x, codes, scale, index=torch.tensor([3, -1, 0, -5, 2], dtype=torch.int32, device="cuda"))
    assert status() == 0
    assert scale[1] == -3.0 and scale[3] == -3.0 and bool((codes[[1, 3]].float() == 2.0).all())
    ctx().quant_rows(x, codes, scale, index=torch.tensor([4, -1, 2 ** 31 - 1, 1, 2], dtype=torch.int32, device="cuda"))
    assert status() == 512
    assert scale[1] == -3.0 and bool((codes[1].float() == 2.0).all())
    _check_rows(codes[3:], x[[1, 2]].double(), scale[3:])


def test_quant_of_odd_values():
    x = torch.ones(5, 300, device="cuda", dtype=F16)
    x[0] = 0
    x[1, 7] = math.inf
    x[2, 299] = math.nan
    x[3] = 2.0 ** -24
    x[4, ::2] = -65504.0
    codes, scale = torch.empty(5, 300, device="cuda", dtype=E4M3), torch.empty(5, device="cuda")
    ctx().quant_rows(x, codes, scale)
    v = codes.float() * scale[:, None]
    assert bool((v[0] == 0).all()) and bool(torch.isnan(v[1]).all()) and bool(torch.isnan(v[2]).all())
    assert float((v[3] / 2.0 ** -24 - 1).abs().max()) < 1e-6 and float((v[4, ::2] / -65504 - 1).abs().max()) < 1e-6
    tiny = torch.full((2, 64), 1e-38, device="cuda")     # below the smallest scale: few bits, but finite and not larger
    c2, s2 = torch.empty(2, 64, device="cuda", dtype=E4M3), torch.empty(2, device="cuda")
    ctx().quant_rows(tiny, c2, s2)
    assert bool((c2.float() == 0).all()) and bool((s2 > 0).all())


def test_norm_captured_and_replayed_on_another_stream():
    g = gen(3)
    x = torch.randn(20, 4096, generator=g, device="cuda").half()
    y, scale = torch.empty(20, 4096, device="cuda", dtype=E4M3), torch.empty(20, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx().norm(x, None, y, y_scale=scale, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx().norm(x, None, y, y_scale=scale)
    x.copy_(torch.randn(20, 4096, generator=g, device="cuda").half() * 5)
    graph.replay()
    torch.cuda.synchronize()
    _check_rows(y, _norm64(x, None, None, ctx().cfg.rms_eps)[1], scale)


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    y, s = torch.zeros(4, 64, device="cuda", dtype=E4M3), torch.zeros(4, device="cuda")
    h = torch.zeros(4, 64, device="cuda", dtype=F16)
    bad = [lambda: ctx().norm(x, None, y),                                     # codes without scales
           lambda: ctx().norm(x, None, h, y_scale=s),                          # scales without codes
           lambda: ctx().norm(x, None, y, y_scale=s, sum_out=x),               # a sum without a residual
           lambda: ctx().norm(x, None, y[:3], y_scale=s),
           lambda: ctx().norm(x, None, h, residual=x[:, :32]),
           lambda: ctx().norm(x, None, h, residual=x, sum_out=h),              # of another type
           lambda: ctx().norm(x, torch.ones(64, device="cuda"), h),            # fp32 gain
           lambda: ctx().norm(x.cpu(), None, h),
           lambda: ctx().norm(y, None, h),
           lambda: ctx().norm(x, None, h, eps=-1.0),
           lambda: ctx().norm(x, None, h, eps=math.nan),
           lambda: ctx().norm(x.T, None, h.T),
           lambda: ctx().norm(x[:1].expand(4, 64), None, h),                   # rows on top of each other
           lambda: ctx().quant_rows(x, h, s),
           lambda: ctx().quant_rows(x, y[:3], s),
           lambda: ctx().quant_rows(x, y, s[:3]),
           lambda: ctx().quant_rows(x, y, s, index=torch.zeros(4, dtype=torch.int64, device="cuda")),
           lambda: ctx().quant_rows(torch.zeros(1, 32776, device="cuda"), torch.zeros(1, 32776, device="cuda", dtype=E4M3), s[:1])]
    for f in bad:
        with pytest.raises((ValueError, B.HbError)):
            f()
    ctx().norm(x[:0], None, h[:0])
    ctx().quant_rows(x[:0], y[:0], s[:0])
    assert status() == 0
    assert C.sizeof(B.NormArgs) == 104
