"""Codes of hb_quant_rows: the nearest to the quotient by the scale that is handed out, and rows turned to codes in place."""
import numpy as np
import pytest
import torch

from tests.dense_util import E4M3, ctx, gen, status, strided

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _codes(x, scale):
    """The fp32 quotient, rounded once to e4m3."""
    return (x.float() / scale[:, None]).to(E4M3).view(torch.uint8)


@pytest.mark.gpu
@pytest.mark.parametrize("x_t", [F32, F16, BF16])
@pytest.mark.parametrize("rows,d,pitch,off", [(4000, 64, 64, 0), (900, 1024, 1024, 0), (300, 2048, 2048, 0), (64, 4096, 4096, 0), (700, 8192, 8192, 0),
                                              (300, 14336, 14336, 0), (20, 14336, 14336, 0), (9, 32768, 32768, 0), (400, 3001, 3003, 1), (7, 32767, 32769, 1)])
def test_codes_are_the_quotients(rows, d, pitch, off, x_t):
    """Equal codes, bit by bit: values of few bits whose ratios fall on borders between codes often, rows of magnitudes from the smallest
    to the largest that the type has, zeros of both signs."""
    g = gen(rows + d)
    x, _ = strided(rows, d, x_t, pitch, off)
    v = torch.randn(rows, d, generator=g, device="cuda")
    if x_t != F16:      # (fp16 keeps its own range; its products with 2^-100 would all be zero)
        v = v * torch.exp2(torch.linspace(-100, 120, rows, device="cuda"))[:, None]
    else:
        v = v * torch.exp2(torch.linspace(-12, 12, rows, device="cuda"))[:, None]
    v[:, ::7] = (v[:, ::7].bfloat16().float() if x_t == F32 else v[:, ::7])
    v[0::5, 0] = -0.0
    x.copy_(v)
    codes, scale = torch.empty(rows, d, device="cuda", dtype=E4M3), torch.empty(rows, device="cuda")
    ctx().quant_rows(x, codes, scale)
    assert torch.equal(codes.view(torch.uint8), _codes(x, scale))
    top = x.float().abs().amax(dim=1).clamp(min=2.0 ** -100)
    assert torch.equal(scale, top / 448)
    index = torch.randint(rows, (rows + 3,), generator=g, device="cuda", dtype=torch.int32)
    c2, s2 = torch.empty(rows + 3, d, device="cuda", dtype=E4M3), torch.empty(rows + 3, device="cuda")
    ctx().quant_rows(x, c2, s2, index=index)
    assert torch.equal(c2.view(torch.uint8), codes.view(torch.uint8)[index.long()]) and torch.equal(s2, scale[index.long()])
    assert status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("x_t", [F16, F32])
@pytest.mark.parametrize("rows,d", [(5, 64), (33, 1024), (400, 1536), (40, 8192), (400, 14336), (3, 32768), (50, 1001)])
def test_codes_in_place(rows, d, x_t):
    """Codes at the start of their own rows' bytes, as the step with 8-bit weights lays them."""
    x = torch.randn(rows, d, generator=gen(d), device="cuda").to(x_t)
    was = x.clone()
    codes, scale = x.view(E4M3)[:, :d], torch.empty(rows, device="cuda")
    ctx().quant_rows(x, codes, scale)
    assert torch.equal(codes.contiguous().view(torch.uint8), _codes(was, scale))
    rest = d * x.element_size()
    assert torch.equal(x.view(torch.uint8)[:, d:rest], was.view(torch.uint8)[:, d:rest])


def test_corrected_quotient_has_the_quotients_code():
    """The kernel's quotient, q0 - (q0 u - x) / u with q0 = x / u by the rounded reciprocal, in fp32 with single roundings: before the last one it is
    within 2^-46 of x / u, so it rounds as x / u does but next to the middle of two floats, and only a middle beside a border
    of codes matters.  Every 24-bit u with a 24-bit x within 2^-42 of such a middle is tried, for a border of each mantissa."""
    f32 = np.float32
    cases = differ = 0
    for mantissa in range(16, 32):
        for half in (1, -1):
            # border b = mantissa / 16; the middle is b + 2^-24, or b - 2^-24 (b - 2^-25 below a power of two), in units of 2^-25
            mid = mantissa * 2 ** 21 + (2 if half == 1 else -2 if mantissa > 16 else -1)
            u = np.arange(2 ** 23, 2 ** 24, dtype=np.int64)
            p = u * mid                                          # x 2^25
            step = np.where(p >= 2 ** 49, 2 ** 26, np.where(p >= 2 ** 48, 2 ** 25, 2 ** 24))   # of floats of x's size, times 2^25
            off = p % step
            near = np.minimum(off, step - off) <= 64
            u, p, step = u[near], p[near], step[near]
            for k in (-1, 0, 1):
                x = ((p + step // 2) // step + k) * step         # times 2^25
                xf, uf = (x / 2.0 ** 25).astype(f32), u.astype(f32)
                recip = (1.0 / uf.astype(np.float64)).astype(f32)          # (no 24-bit reciprocal lies within 2^-50 of a middle)
                q0 = xf * recip
                # q0 u - x exactly: integers of at most 48 bits over a common power of two
                e = 2.0 ** 24
                r = (q0.astype(np.float64) * e).astype(np.int64) * u - (x.astype(object) // 2).astype(np.int64)   # times 2^24
                rf = r.astype(f32)
                # q0 - r recip, rounded once: in units of 2^-24 2^-72, as Python integers
                got = np.array([_round24(int(a * e) << 72, -int(b) * int(c * 2.0 ** 72)) for a, b, c in
                                zip(q0.astype(np.float64), rf.astype(np.float64), recip.astype(np.float64))])
                want = (xf.astype(np.float64) / uf.astype(np.float64)).astype(f32)   # (53 bits hold it 2^-48 from any middle)
                cases += len(u)
                differ += int(np.sum(got != want.astype(np.float64)))
    assert cases > 1000 and differ == 0


def _round24(a, b):
    """a + b in units of 2^-96 to 24 bits, ties to even."""
    v = a + b
    s = v.bit_length() - 24
    k, rest = v >> s, v & ((1 << s) - 1)
    k += rest > (1 << (s - 1)) or (rest == (1 << (s - 1)) and k & 1)
    return float(k) * 2.0 ** (s - 96)
