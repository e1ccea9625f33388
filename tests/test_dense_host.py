"""The dense operators on the host: refusals of the C calls before anything is launched, argument structs, the definition's own
pins.  No GPU: the context is an address that a refused call never follows."""
import ctypes as C
import math
import struct

import numpy as np
import pytest
import torch

from paper_2609_25405_b200 import binding as B
from tests.dense_util import act64, e4m3_64

CTX, P = C.c_void_p(1 << 20), 1 << 21     # stored, never touched
BAD, LARGE, CUDA = -1, -5, -2


def _norm(**kw):
    a = B.NormArgs(x=P, y=P, x_stride=64, y_stride=64, x_dtype=B.DTYPE_F16, y_dtype=B.DTYPE_F16, n_rows=4, d=64, eps=1e-5)
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lib.hb_norm(CTX, C.byref(a), None)


def _linear(**kw):
    a = B.LinearArgs(a=P, w=P, c=P, a_stride=64, w_stride=64, c_stride=32, m=4, n=32, k=64, ab_dtype=B.DTYPE_F16, c_dtype=B.DTYPE_F32)
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lib.hb_linear(CTX, C.byref(a), None)


def _grouped(groups=2, stride=2048, start=P, **kw):
    a = B.LinearArgs(a=P, w=P, c=P, a_stride=64, w_stride=64, c_stride=32, m=4, n=32, k=64, ab_dtype=B.DTYPE_F16, c_dtype=B.DTYPE_F32)
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lib.hb_linear_grouped(CTX, C.byref(a), start, groups, stride, None)


def _quant(x=P, dtype=B.DTYPE_F16, x_stride=64, n_src=4, index=None, n_rows=4, d=64, codes=P, codes_stride=64, scale=P):
    return B.lib.hb_quant_rows(CTX, x, dtype, x_stride, n_src, index, n_rows, d, codes, codes_stride, scale, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(y=None), BAD), (dict(n_rows=-1), BAD), (dict(d=0), BAD), (dict(d=B.NORM_MAX_D + 1, x_stride=1 << 20, y_stride=1 << 20), LARGE),
    (dict(x_stride=63), BAD), (dict(y_stride=63), BAD), (dict(x_dtype=B.DTYPE_E4M3), BAD), (dict(x_dtype=4), BAD), (dict(y_dtype=-1), BAD),
    (dict(y_dtype=B.DTYPE_E4M3), BAD), (dict(y_scale=P), BAD), (dict(sum_out=P, sum_stride=64), BAD), (dict(eps=-1e-6), BAD), (dict(eps=math.nan), BAD),
    (dict(residual=P, residual_stride=60), BAD), (dict(residual=P, residual_stride=64, residual_dtype=B.DTYPE_E4M3), BAD),
    (dict(residual=P, residual_stride=64, sum_out=P, sum_stride=32), BAD), (dict(x=P + 1), BAD), (dict(gain=P + 1), BAD),
    (dict(residual=P + 2, residual_stride=64, residual_dtype=B.DTYPE_F32), BAD), (dict(y_dtype=B.DTYPE_E4M3, y_scale=P + 2), BAD)])
def test_norm_refusals(kw, code):
    assert _norm(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(codes=None), BAD), (dict(scale=None), BAD), (dict(n_rows=-1), BAD), (dict(n_src=-1), BAD), (dict(n_src=3), BAD),
    (dict(d=0), BAD), (dict(d=B.NORM_MAX_D + 1, x_stride=1 << 20, codes_stride=1 << 20), LARGE), (dict(x_stride=63), BAD), (dict(codes_stride=63), BAD),
    (dict(dtype=B.DTYPE_E4M3), BAD), (dict(x=P + 1), BAD), (dict(scale=P + 2), BAD), (dict(index=P + 2), BAD)])
def test_quant_refusals(kw, code):
    assert _quant(**kw) == code


LINEAR_BAD = [
    (dict(a=None), BAD), (dict(w=None), BAD), (dict(c=None), BAD), (dict(m=-1), BAD), (dict(n=0), BAD), (dict(k=0), BAD), (dict(a_stride=56), BAD),
    (dict(w_stride=56), BAD), (dict(c_stride=31), BAD), (dict(a_stride=65), BAD), (dict(w_stride=68), BAD), (dict(a=P + 8), BAD), (dict(w=P + 2), BAD),
    (dict(c=P + 2), BAD), (dict(ab_dtype=B.DTYPE_F32), BAD), (dict(ab_dtype=4), BAD), (dict(c_dtype=B.DTYPE_E4M3), BAD), (dict(act=5), BAD),
    (dict(act=-1), BAD), (dict(gated=2), BAD), (dict(gated=1, n=31), BAD), (dict(residual=P, residual_stride=16), BAD),
    (dict(residual=P, residual_stride=32, residual_dtype=B.DTYPE_E4M3), BAD), (dict(residual=P + 2, residual_stride=32), BAD), (dict(a_scale=P + 1), BAD),
    (dict(w_scale=P + 2), BAD), (dict(bias=P + 3), BAD), (dict(m=(1 << 26) + 1), LARGE), (dict(n=(1 << 26) + 1, c_stride=1 << 27), LARGE),
    (dict(a_stride=(1 << 36) + 8), LARGE), (dict(c_stride=(1 << 36) + 8), LARGE)]


@pytest.mark.parametrize("kw,code", LINEAR_BAD)
def test_linear_refusals(kw, code):
    assert _linear(**kw) == code
    assert _grouped(**kw) == code


@pytest.mark.parametrize("kw,code", [(dict(groups=0), BAD), (dict(groups=513), LARGE), (dict(stride=2047), BAD), (dict(stride=2052), BAD), (dict(start=None), BAD),
                                     (dict(start=P + 2), BAD), (dict(stride=(1 << 36) + 8), LARGE)])
def test_grouped_refusals(kw, code):
    assert _grouped(**kw) == code


def test_calls_without_a_context_or_arguments():
    assert B.lib.hb_norm(None, C.byref(B.NormArgs()), None) == BAD and B.lib.hb_norm(CTX, None, None) == BAD
    assert B.lib.hb_linear(None, C.byref(B.LinearArgs()), None) == BAD and B.lib.hb_linear(CTX, None, None) == BAD
    assert B.lib.hb_linear_grouped(CTX, None, None, 1, 64, None) == BAD
    assert B.lib.hb_quant_rows(None, P, 1, 64, 4, None, 4, 64, P, 64, P, None) == BAD
    assert B.lib.hb_mixed_step8(None, None, None, None, None, None, None, None) == BAD


def test_no_rows_is_no_work():
    """Nothing is launched, and arrays may be missing."""
    assert _norm(n_rows=0, x=None, y=None) == 0 and _norm(n_rows=0, y_dtype=B.DTYPE_E4M3) == 0
    assert _quant(n_rows=0, n_src=0, x=None, codes=None, scale=None) == 0
    assert _linear(m=0, a=None, c=None) == 0 and _grouped(m=0, a=None, c=None) == 0


def test_structs_are_their_packed_forms():
    """The binding passes packed bytes: field by field the C struct's."""
    v = list(range(1, 7)) + [10, 11, 12, 13] + [1, 2, 3, 4, 5] + [0.5]
    a = B.NormArgs.from_buffer_copy(B._pack_norm(*v))
    assert [getattr(a, n) for n, _ in B.NormArgs._fields_] == v and C.sizeof(a) == struct.calcsize("6Q4q5if")
    v = list(range(1, 8)) + [10, 11, 12, 13] + list(range(20, 28))
    a = B.LinearArgs.from_buffer_copy(B._pack_linear(*v))
    assert [getattr(a, n) for n, _ in B.LinearArgs._fields_] == v


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(2, 64)
    for f in (lambda: B._matrix(x, 0, "x"), lambda: B._packed(x, torch.float32, (2, 64), 0, "x")):
        with pytest.raises(ValueError):
            f()
    assert B._packed(None, torch.float32, (2,), 0, "x") == 0


def test_the_definitions_activations_are_torchs():
    z = torch.linspace(-12, 12, 4001, dtype=torch.float64)
    f = torch.nn.functional
    for kind, want in (("relu", f.relu(z)), ("silu", f.silu(z)), ("gelu", f.gelu(z)), ("gelu_tanh", f.gelu(z, approximate="tanh")), ("none", z)):
        assert float((act64(z, kind) - want).abs().max()) <= 1e-12


def test_the_approximation_of_erfc():
    """Abramowitz and Stegun 7.1.26, as the GELU uses it, in 64 bits: at most 1.5e-7 off, so x Phi(x) at most 2^-23 |x|."""
    x = np.linspace(-30, 30, 200001)
    u = np.abs(x) / math.sqrt(2)
    t = 1 / (1 + 0.3275911 * u)
    p = ((((1.061405429 * t - 1.453152027) * t + 1.421413741) * t - 0.284496736) * t + 0.254829592) * t * np.exp(-u * u)
    erfc = np.array([math.erfc(v) for v in u])
    assert np.max(np.abs(p - erfc)) <= 1.5e-7
    phi = np.where(x < 0, 0.5 * p, 1 - 0.5 * p)
    exact = np.where(x < 0, 0.5 * erfc, 1 - 0.5 * erfc)
    assert np.all(np.abs(x * phi - x * exact) <= 2.0 ** -23 * np.abs(x))


def test_e4m3_of_the_definition_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 5001), 2.0 ** np.linspace(-12, 8, 3001)]).astype(np.float32)
    assert np.array_equal(e4m3_64(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
