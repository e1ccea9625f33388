"""Every kernel of hb_linear and hb_linear_grouped, dense and with groups, plain, gated, with a residual, in place and off 16-byte boundaries;
which kernel a case takes is asked on the host and held to what is written beside it."""
import pytest
import torch

from tests.dense_util import ACTS, E4M3, check, ctx, linear64, status, strided
from tests.test_gpu_linear import _case
from tests.test_linear_variant import B, variant

F32, F16 = torch.float32, torch.float16
CODE = {F32: B.DTYPE_F32, F16: B.DTYPE_F16, E4M3: B.DTYPE_E4M3}
PLAIN, LONG, SHORT = 0, 1, 2
TILES = {(t, s, PLAIN) for t in (8, 16) for s in (1, 2)} | {(t, s, PLAIN) for t in (32, 64, 128) for s in (4, 8)} | \
        {(t, 1, m) for t in (32, 64, 128, 256) for m in (PLAIN, LONG)} | {(t, 1, SHORT) for t in (128, 256)}

# (kernel, m, n, k, operands, groups)
CASES = [
    ((8, 1, PLAIN), 4, 140, 1069, F16, 0), ((8, 1, PLAIN), 11, 150, 1073, F16, 2), ((8, 2, PLAIN), 53, 1298, 537, F16, 0),
    ((8, 2, PLAIN), 45, 1304, 608, F16, 2), ((16, 1, PLAIN), 5, 142, 40, F16, 0), ((16, 1, PLAIN), 5, 142, 41, F16, 2),
    ((16, 2, PLAIN), 50, 1244, 70, F16, 0), ((16, 2, PLAIN), 179, 420, 68, F16, 3),
    ((32, 1, PLAIN), 66, 142, 41, F16, 0), ((32, 1, PLAIN), 135, 146, 41, E4M3, 2), ((32, 1, LONG), 67, 146, 663, F16, 0),
    ((32, 1, LONG), 138, 142, 724, F16, 2), ((32, 4, PLAIN), 31, 4950, 2892, F16, 0), ((32, 4, PLAIN), 218, 410, 2903, F16, 8),
    ((32, 8, PLAIN), 68, 142, 1448, F16, 0), ((32, 8, PLAIN), 144, 144, 1429, F16, 2),
    ((64, 1, PLAIN), 134, 142, 41, F16, 0), ((64, 1, PLAIN), 275, 142, 47, F16, 2), ((64, 1, LONG), 162, 146, 666, F16, 0),
    ((64, 1, LONG), 329, 142, 736, F16, 2), ((64, 4, PLAIN), 141, 2378, 3599, F16, 0), ((64, 4, PLAIN), 1987, 198, 3868, F16, 8),
    ((64, 8, PLAIN), 141, 152, 1673, F16, 0), ((64, 8, PLAIN), 337, 158, 1688, F16, 2),
    ((128, 1, PLAIN), 280, 142, 539, F16, 0), ((128, 1, PLAIN), 553, 144, 529, F16, 2), ((128, 1, LONG), 284, 144, 684, F16, 0),
    ((128, 1, LONG), 560, 158, 824, F16, 2), ((128, 1, SHORT), 272, 148, 40, F16, 0), ((128, 1, SHORT), 577, 146, 42, E4M3, 2),
    ((128, 4, PLAIN), 2403, 142, 4369, F16, 0), ((128, 4, PLAIN), 2435, 142, 4214, F16, 2), ((128, 8, PLAIN), 265, 142, 1906, F16, 0),
    ((128, 8, PLAIN), 615, 148, 1851, F16, 2),
    ((256, 1, PLAIN), 4986, 446, 819, F16, 0), ((256, 1, PLAIN), 4762, 398, 794, F16, 5), ((256, 1, LONG), 3837, 542, 799, F16, 0),
    ((256, 1, LONG), 1128, 1982, 813, F16, 2), ((256, 1, SHORT), 3961, 530, 1200, E4M3, 0), ((256, 1, SHORT), 4707, 448, 1238, E4M3, 3)]


def _outputs(kernel):
    """Output types with which the case takes that kernel: segments are for fp32, whole tiles in one accumulator for 16 bits."""
    if kernel[0] >= 32 and kernel[1] == 1 and kernel[2] != SHORT:
        short_k = kernel[0] < 128          # (their cases have fewer k-blocks than a segment)
        return (F32,) if kernel[2] == LONG else (F16, F32) if short_k else (F16,)
    return (F16, F32)


def test_the_cases_take_every_kernel():
    assert {c[0] for c in CASES if c[5] == 0} == TILES and {c[0] for c in CASES if c[5] > 0} == TILES
    for kernel, m, n, k, ab, groups in CASES:
        for c_t in _outputs(kernel):
            assert variant(m, n, k, CODE[ab], CODE[c_t], groups) == kernel, (m, n, k, ab, c_t, groups)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,m,n,k,ab,groups", CASES)
def test_every_kernel_with_every_end(kernel, m, n, k, ab, groups):
    outputs = _outputs(kernel)
    # (activation, gated, residual, offset of C and the residual in wider rows)
    for i, (act, gated, residual, off) in enumerate([("none", False, F32, 0), ("silu", True, None, 0), ("gelu", True, F16, 0), ("relu", False, F16, 3),
                                                     ("silu", True, F32, 1), ("none", False, "c", 0)]):
        c_t = outputs[i % len(outputs)]
        in_place, residual = residual == "c", c_t if residual == "c" else residual      # (the residual is C itself)
        c = _case(m, n, k, ab, c_t, seed=i, groups=max(groups, 1), act=act, gated=gated, bias=i % 2 == 0, residual=residual)
        out, whole = strided(m, c["cols"], c_t, c["cols"] + 2 * off + (16 - c["cols"] % 16 if off == 0 else 0), off, fill=9.0)
        if residual is not None and off:
            r, _ = strided(m, c["cols"], residual, c["cols"] + off, off)
            c["residual"] = r.copy_(c["residual"])
        if in_place:
            out.copy_(c["residual"])
        pick = lambda v, rows: None if v is None else v[rows]   # noqa: E731
        args = dict(a_scale=c["a_scale"], act=ACTS[act], gated=gated, residual=out if in_place else c["residual"])
        if not groups:
            ctx().linear(c["a"], c["w"][0], out, w_scale=pick(c["w_scale"], 0), bias=pick(c["bias"], 0), **args)
            start = [0, m]
        else:
            # uneven groups, the last row of all left out
            cuts = sorted(int(m * (e * 0.77 + 0.1 * i) / groups) for e in range(1, groups))
            start = [0] + cuts + [m - 1]
            ctx().linear_grouped(c["a"], c["w"], torch.tensor(start, dtype=torch.int32, device="cuda"), out, w_scale=c["w_scale"], bias=c["bias"], **args)
        for e in range(len(start) - 1):
            rows = slice(start[e], start[e + 1])
            if start[e + 1] > start[e]:
                check(out[rows], *linear64(c["a"][rows], c["w"][e], pick(c["a_scale"], rows), pick(c["w_scale"], e), pick(c["bias"], e), act, gated,
                                           pick(c["residual"], rows), c_t))
        if in_place and groups:
            assert torch.equal(out[m - 1], c["residual"][m - 1])
        out[:m if in_place else start[-1]] = 9.0
        assert bool((whole.float() == 9.0).all())
        assert status() == 0
