"""Builds step rows, caches and inputs for the tests of the 8-bit cache operators."""
import numpy as np
import torch

from oracle import kv8 as O
from paper_2609_25405_b200 import binding as B
from paper_2609_25405_b200 import synth

_CTX = {}


def context(hq, hkv, dh, layers=2, max_pos=4096):
    """(cfg, Context) of a geometry, one per session."""
    key = (hq, hkv, dh, layers, max_pos)
    if key not in _CTX:
        cfg = B.model_cfg(synth.ModelShape("ops", layers, 64, hq, hkv, dh, 64, 64), max_pos)
        _CTX[key] = (cfg, B.Context(cfg, 1, 1, 1))
    return _CTX[key]


class Rows:
    """Segments [(pos_start, q_len)] laid out one after the other, `gaps` padding rows after each, page lists drawn
    without replacement out of n_pages."""

    def __init__(self, segs, n_pages, seed=0, gap=0, max_q_len=None, max_keys=None):
        r = np.random.default_rng(seed)
        need = [(p + q + 15) // 16 for p, q in segs]
        assert sum(need) <= n_pages
        ids = r.permutation(n_pages)[:sum(need)].astype(np.int32)
        self.pages, table, row_seg, at, pt = [], [], [], 0, 0
        for i, ((p, q), n) in enumerate(zip(segs, need)):
            self.pages.append(ids[pt:pt + n])
            table.append([0, at, q, p, pt, n, -1, 0, 1, -1, -1, 0])
            row_seg += [i] * q + [-1] * gap
            at += q + gap
            pt += n
        self.segs, self.table, self.T = segs, np.array(table, dtype=np.int32).reshape(-1, 12), at
        self.start = self.table[:, 1]
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.dev = B.SegRows(up(self.table), up(ids), up(np.array(row_seg, dtype=np.int32)),
                             max((q for _, q in segs), default=0) if max_q_len is None else max_q_len,
                             max((p + q for p, q in segs), default=0) if max_keys is None else max_keys)


def random_arena(cfg, n_pages, seed, scale_lo=-9, scale_hi=-4):
    """Every code finite and e4m3-normal-distributed, scales 2^scale_lo .. 2^scale_hi per block."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kv = B.KvCache8(cfg, n_pages)
    kv.arena.zero_()
    shape = tuple(kv.codes().shape)
    kv.codes().copy_((torch.randn(shape, generator=g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn))
    e = torch.randint(scale_lo, scale_hi + 1, tuple(kv.scales().shape), generator=g, device="cuda")
    kv.scales().copy_(torch.exp2(e.float()))
    return kv


def layer_bytes(kv, layer):
    c = kv.cfg
    return kv.arena.cpu().numpy().reshape(c.n_layers, kv.n_pages, c.n_kv_heads, 32 * c.head_dim + 32)[layer]


def oracle_layer(kv, layer):
    return O.read_layer(layer_bytes(kv, layer), kv.cfg.head_dim)


# Bound on an element of the attention's output: the output's own rounding to fp16 (2^-11 of the value, which
# the mass bounds), the rounding of every probability to fp16 (2^-11 of each term), and 2^-13 for fp32 scores of
# some tens (2^-24 * |s| * sums of 128 products) and the exponential (2^-22); absolute: fp16 subnormals of the output
# (2^-25), and of the probabilities (2^-25 where the largest is at least 2^6, times codes of up to twice the largest |v|: 2^-30 per key).
def attend_bound(mass, n_keys, vmax):
    return (2.0 ** -11 + 2.0 ** -11 + 2.0 ** -13) * mass + 2.0 ** -25 + vmax * n_keys * 2.0 ** -30
