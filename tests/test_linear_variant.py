"""Which kernel hb_linear and hb_linear_grouped take, asked on the host (hb_linear_variant): no GPU."""
import ctypes as C

import pytest

from paper_2609_25405_b200 import binding as B

E4M3, F16, F32 = B.DTYPE_E4M3, B.DTYPE_F16, B.DTYPE_F32


def variant(m, n, k, ab, c_t=F16, groups=0, sms=148, gated=0, act=0):
    """(rows of a tile, share, mode)."""
    a, out = B.LinearArgs(m=m, n=n, k=k, ab_dtype=ab, c_dtype=c_t, gated=gated, act=act), (C.c_int32 * 3)()
    assert B.lib.hb_linear_variant(C.byref(a), groups, sms, out) == 0
    return tuple(out)


@pytest.mark.parametrize("m,n,k,ab,want", [
    # the weights bound all of these: the smallest tile that holds the rows, not the pairs that the bound hides
    (1, 28672, 4096, E4M3, (32, 1)), (8, 28672, 4096, E4M3, (32, 1)), (32, 28672, 4096, E4M3, (32, 1)), (64, 28672, 4096, E4M3, (64, 1)),
    (128, 28672, 4096, E4M3, (128, 1)), (40, 18500, 12076, E4M3, (64, 1)), (105, 18599, 8805, F16, (128, 1)),
    # what the comment at the rule says of both sides
    (8, 2048, 2048, F16, (8, 1)), (64, 1024, 8192, F16, (32, 8)), (300, 4096, 4096, F16, (128, 1)), (2000, 4096, 4096, F16, (256, 1))])
def test_the_rule(m, n, k, ab, want):
    assert variant(m, n, k, ab)[:2] == want


def test_more_weights_do_not_move_the_choice_back():
    """From the feature count on at which the weights bound a product of few rows, a wider one never takes the pairs."""
    for m in (8, 64):
        took = [variant(m, n, 4096, E4M3)[0] for n in range(20480, 40961, 512)]
        assert 256 not in took


def test_chains_of_additions_are_bounded():
    """fp32 outputs: at most 64 k-blocks (128 bytes of K) in one accumulator, or sums that leave in segments; 16 bits out: 256."""
    for ab, size in ((F16, 2), (E4M3, 1)):
        for c_t, most in ((F32, 64), (F16, 256)):
            for m in (1, 8, 16, 33, 64, 100, 200, 500, 3000):
                for n in (16, 150, 1024, 5000):
                    for k in (64, 5000, 14336, 32768, 65537, 1 << 18, 1 << 22):
                        for groups in (0, 4):
                            tokens, share, mode = variant(m, n, k, ab, c_t, groups)
                            blocks = (k * size + 127) // 128
                            blocks = -(-blocks // 8) if tokens <= 16 else 10 if mode == 1 else -(-blocks // share)
                            assert blocks <= most, (m, n, k, ab, c_t, groups)


def test_refusals():
    out = (C.c_int32 * 3)()
    good = dict(m=4, n=32, k=64, ab_dtype=F16, c_dtype=F32)
    for kw in (dict(m=0), dict(n=0), dict(k=0)):
        assert B.lib.hb_linear_variant(C.byref(B.LinearArgs(**dict(good, **kw))), 0, 148, out) == -1
    for kw in (dict(m=(1 << 26) + 1), dict(n=2 ** 31 - 1), dict(k=2 ** 31 - 1)):
        assert B.lib.hb_linear_variant(C.byref(B.LinearArgs(**dict(good, **kw))), 0, 148, out) == -5
    a = B.LinearArgs(**good)
    assert B.lib.hb_linear_variant(C.byref(a), B.LINEAR_MAX_GROUPS + 1, 148, out) == -5
    assert B.lib.hb_linear_variant(None, 0, 148, out) == -1 and B.lib.hb_linear_variant(C.byref(a), 0, 148, None) == -1
    assert B.lib.hb_linear_variant(C.byref(a), -1, 148, out) == -1 and B.lib.hb_linear_variant(C.byref(a), 0, 0, out) == -1
    assert B.lib.hb_linear_variant(C.byref(a), 0, 148, out) == 0
