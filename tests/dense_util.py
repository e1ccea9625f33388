"""Inputs, definitions in 64 bits and error bounds for the tests of the dense operators."""
import math

import numpy as np
import torch

from paper_2609_25405_b200 import binding as B
from tests.kv8_util import context

E4M3 = torch.float8_e4m3fn
ACTS = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU, "gelu_tanh": B.ACT_GELU_TANH}
LARGEST = {torch.float16: 65504.0, torch.float32: math.inf, torch.bfloat16: math.inf}


def ctx():
    return context(2, 1, 64)[1]


def status():
    return ctx().status_poll()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def strided(rows, cols, dtype, pitch, offset=0, fill=float("nan")):
    """[rows, cols] inside a wider matrix whose other elements hold `fill`; (view, whole)."""
    whole = torch.empty(rows, pitch, device="cuda", dtype=torch.float32).fill_(fill).to(dtype)
    return whole[:, offset:offset + cols], whole


def operand(g, rows, cols, dtype, std=1.0, pitch=None):
    """A matrix of 16-byte aligned rows, NaN behind each row's end."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    v, _ = strided(rows, cols, dtype, pitch or (cols + per - 1) // per * per + per)
    x = torch.randn(rows, cols, generator=g, device="cuda") * std
    v.copy_((x * 100).clamp(-448, 448).to(E4M3) if dtype == E4M3 else x.to(dtype))
    return v


def act64(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.where(z != z, z, 0.0))
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if kind == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def linear64(a, w, a_scale=None, w_scale=None, bias=None, act="none", gated=False, residual=None, c_dtype=torch.float32):
    """(result in 64 bits, bound on the error of a result of c_dtype).

    The products of two 16- or 8-bit values are exact in fp32.  A tensor core instruction adds 16 (32) of them to the
    running sum and may cut what does not fit: one step of 2^-23 of the largest partial sum, which `mass`, the sum of
    the magnitudes, bounds; 16 of them once more for sums that are split and joined.  Scales and bias: 2^-24 each of
    what they touch.  The activations' slopes stay below 1.13; 2^-20 of |z| for exp, erf and the division.  Residual:
    2^-24 of the sum.  Last the output's own half step (and 2^-25 among fp16's subnormals)."""
    a, w = a.double(), w.double()
    f = torch.ones(a.shape[0], 1, device="cuda", dtype=torch.float64)
    if a_scale is not None:
        f = f * a_scale.double()[:, None]
    if w_scale is not None:
        f = f * w_scale.double()
    steps = math.ceil(a.shape[1] / 16) + 16
    z, e = (a @ w.T) * f, (a.abs() @ w.abs().T) * f.abs() * steps * 2.0 ** -23
    if bias is not None:
        z = z + bias.double()
    e = e + z.abs() * 2.0 ** -22 + (0 if bias is None else bias.double().abs() * 2.0 ** -22)
    if gated:
        g, u, eg, eu = z[:, 0::2], z[:, 1::2], e[:, 0::2], e[:, 1::2]
        y = act64(g, act) * u
        e = (1.13 * eg + g.abs() * 2.0 ** -20) * (u.abs() + eu) + act64(g, act).abs() * eu + y.abs() * 2.0 ** -23
    else:
        y = act64(z, act)
        e = 1.13 * e + z.abs() * 2.0 ** -20
    if residual is not None:
        y = y + residual.double()
        e = e + y.abs() * 2.0 ** -23
    big = LARGEST[c_dtype]
    y = y.clamp(-big, big) if math.isfinite(big) else y
    return y, e + (y.abs() + e) * torch.finfo(c_dtype).eps / 2 + (2.0 ** -25 if c_dtype == torch.float16 else 0.0)


def check(got, want, bound):
    got, want = got.double(), want
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    off = (got - want).abs()
    bad = (off > bound) & ~nan
    assert not bad.any(), (int(bad.sum()), float((off / bound)[bad].max()), bad.nonzero()[:4].tolist())


def e4m3_64(x):
    """Nearest e4m3 value, ties to even, |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    _, p = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(p, -5) - 4)
    return np.round(x / step) * step
