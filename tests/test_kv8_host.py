"""The 8-bit KV cache on the host: sizes, refusals, page bookkeeping, rotary tables, the oracle's pins.  No GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from oracle import kv8 as O
from paper_2609_25405_b200 import binding as B
from paper_2609_25405_b200 import synth

TINY = synth.SHAPES["tiny"]
CFG = B.model_cfg(TINY, 256)


def test_e4m3_rounding_of_the_oracle_is_torchs():
    """Every code, every midpoint between neighbours and its two fp32 neighbours, and random values."""
    vals = np.unique(O.code_value(np.arange(127)))
    mid = (vals[1:] + vals[:-1]) / 2
    x = np.concatenate([vals, mid, np.nextafter(mid.astype(np.float32), np.float32(1e9)),
                        np.nextafter(mid.astype(np.float32), np.float32(0)), np.random.default_rng(0).uniform(0, 448, 4000)])
    x = np.concatenate([x, -x]).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(O.e4m3(x), ref)
    assert np.all(np.abs(O.e4m3(x) - x) <= O.e4m3_half_step(x))


def test_code_values_are_torchs():
    b = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(b).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(O.code_value(b), ref, equal_nan=True)


@pytest.mark.parametrize("dh", [64, 128])
def test_byte_orders_are_permutations(dh):
    t, d = np.arange(16)[:, None], np.arange(dh)[None, :]
    for f in (O.k_byte, O.v_byte):
        assert sorted(f(t, d).ravel()) == list(range(16 * dh))


def test_scale_exponent_of_the_oracle():
    for a, e in ((448.0, 0), (np.nextafter(448.0, 1e9), 1), (224.0, -1), (1.75, -8), (1.76, -7), (0.0, -32), (65504.0, 8),
                 (np.inf, 24), (2.0 ** -60, -32)):
        assert O.exponent(a) == e, a


def test_arena_bytes_and_create_refusals():
    n = C.c_size_t()
    assert B.lib.hb_kv8_arena_bytes(C.byref(CFG), 10, C.byref(n)) == 0
    assert n.value == TINY.L * 10 * TINY.Hkv * (32 * TINY.Dh + 32)
    bad = B.model_cfg(TINY, 256); bad.head_dim = 96
    assert B.lib.hb_kv8_arena_bytes(C.byref(bad), 10, C.byref(n)) == -1
    assert B.lib.hb_kv8_arena_bytes(C.byref(CFG), 0, C.byref(n)) == -1
    h = C.c_void_p()
    fake = 1 << 20                       # an aligned address that is only stored, never touched
    size = B.kv8_arena_bytes(CFG, 10)
    assert B.lib.hb_kv8_create(C.byref(CFG), C.c_void_p(fake), size - 1, 10, C.byref(h)) == -1
    assert B.lib.hb_kv8_create(C.byref(CFG), C.c_void_p(fake + 128), size, 10, C.byref(h)) == -1
    assert B.lib.hb_kv8_create(C.byref(CFG), C.c_void_p(fake), size, 10, None) == -1
    assert B.lib.hb_kv8_create(C.byref(CFG), C.c_void_p(fake), size, 10, C.byref(h)) == 0
    assert B.lib.hb_kv_destroy(h) == 0


def test_pages_of_an_8_bit_cache():
    kv = B.KvCache8(CFG, 4, device=None)
    assert kv.alloc(3) == [0, 1, 2]
    kv.free([1])
    assert kv.alloc(2) == [1, 3] and kv.free_count() == 0
    with pytest.raises(B.HbError):
        kv.alloc(1)


def test_workspace_grows_with_the_splits():
    n = C.c_size_t()
    size = lambda rows, segs, keys: (B.lib.hb_kv8_attention_workspace(C.byref(CFG), C.byref(B.RowsStruct(  # noqa: E731
        n_rows=rows, n_segs=segs, max_keys=keys)), C.byref(n)), n.value)
    assert size(4, 4, 0) == (0, 0) and size(4, 4, 511) == (0, 0)
    rec = TINY.Dh * 4 + 8
    assert size(4, 4, 1024) == (0, 4 * TINY.Hq * 3 * rec)              # every row's heads ...
    assert size(1000, 4, 1024) == (0, 4 * TINY.Hkv * 16 * 3 * rec)     # ... or 16 columns per segment and KV head
    assert size(4, 4, 1 << 20) == (0, 4 * TINY.Hq * 64 * rec)          # never more than 64 splits
    assert size(-1, 1, 10)[0] == -1 and size(1, -1, 10)[0] == -1 and size(1, 1, -1)[0] == -1 and size(1, 8193, 10)[0] == -5
    assert size((1 << 26) + 1, 1, 10)[0] == -5 and size(1, 1, (1 << 30) + 1)[0] == -5


def test_calls_without_a_context_or_cache_are_refused():
    rows, args = B.RowsStruct(), B.AppendArgs()
    assert B.lib.hb_kv8_append(None, None, 0, C.byref(rows), C.byref(args), None) == -1
    assert B.lib.hb_kv8_attention(None, None, 0, C.byref(rows), None, 64, None, 64, 0.0, None, 0, None) == -1


def test_rows_on_the_host_are_refused():
    z = torch.zeros(1, 12, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.SegRows(z, torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 1)
    with pytest.raises(ValueError):
        B.Rope(torch.zeros(4, 8), torch.zeros(4, 8))


def _angles(n, rot, theta):
    f = theta ** (-2.0 * np.arange(rot // 2) / rot)
    return f, np.arange(n)[:, None] * f


def test_rope_table_plain_and_linear():
    cos, sin = B.rope_table(70, 32, 1e4)
    _, a = _angles(70, 32, 1e4)
    # stored as float: half a unit in the last place
    assert np.all(np.abs(cos - np.cos(a)) <= 2.0 ** -24) and np.all(np.abs(sin - np.sin(a)) <= 2.0 ** -24)
    cos, sin = B.rope_table(70, 32, 1e4, B.RopeScaling(B.ROPE_LINEAR, 4.0, 0, 0, 0, 1.0))
    assert np.all(np.abs(cos - np.cos(a / 4)) <= 2.0 ** -24) and np.all(np.abs(sin - np.sin(a / 4)) <= 2.0 ** -24)


def test_rope_table_far_positions_keep_their_angle():
    cos, _ = B.rope_table(131072, 16, 1e4)
    f, _ = _angles(1, 16, 1e4)
    assert np.all(np.abs(cos[131071] - np.cos(131071 * f)) <= 2.0 ** -24)


def test_rope_table_by_parts():
    sc = B.RopeScaling(B.ROPE_BY_PARTS, 8.0, 4096.0, 1.0, 32.0, 1.25)
    cos, sin = B.rope_table(50, 128, 1e4, sc)
    f, _ = _angles(1, 128, 1e4)
    turns = 4096.0 * f / (2 * np.pi)
    g = np.clip((turns - 1.0) / 31.0, 0, 1)
    assert g.max() == 1.0 and g.min() == 0.0 and ((g > 0) & (g < 1)).any()
    a = np.arange(50)[:, None] * (f * (g + (1 - g) / 8.0))
    assert np.all(np.abs(cos - 1.25 * np.cos(a)) <= 1.25 * 2.0 ** -24 + 1e-15)
    assert np.all(np.abs(sin - 1.25 * np.sin(a)) <= 1.25 * 2.0 ** -24 + 1e-15)


@pytest.mark.parametrize("args", [(0, 32, 1e4, None), (4, 31, 1e4, None), (4, 0, 1e4, None), (4, 32, 0.0, None),
                                  (4, 32, 1e4, (3, 2.0, 10.0, 1.0, 2.0, 1.0)), (4, 32, 1e4, (1, 0.5, 10.0, 1.0, 2.0, 1.0)),
                                  (4, 32, 1e4, (2, 2.0, 0.0, 1.0, 2.0, 1.0)), (4, 32, 1e4, (2, 2.0, 10.0, 2.0, 2.0, 1.0)),
                                  (4, 32, 1e4, (1, 2.0, 10.0, 1.0, 2.0, 0.0)), (4, 32, float("nan"), None)])
def test_rope_table_refusals(args):
    n, rot, theta, sc = args
    with pytest.raises(B.HbError) as e:
        B.rope_table(n, rot, theta, B.RopeScaling(*sc) if sc else None)
    assert e.value.code == -1


def test_oracle_attention_is_softmax_attention():
    """Against torch's own on a small case: grouped heads, causal with earlier tokens."""
    r = np.random.default_rng(1)
    q, k, v = r.standard_normal((5, 4, 64)), r.standard_normal((12, 2, 64)), r.standard_normal((12, 2, 64))
    out, _ = O.attend(q, k, v, 7, 0.125)
    mask = torch.ones(5, 12, dtype=torch.bool).tril(7)
    to = lambda a, rep: torch.from_numpy(a).transpose(0, 1).repeat_interleave(rep, 0)  # noqa: E731
    ref = torch.nn.functional.scaled_dot_product_attention(to(q, 1), to(k, 2), to(v, 2), attn_mask=mask, scale=0.125)
    assert np.max(np.abs(out - ref.transpose(0, 1).numpy())) < 1e-13


def _kernels():
    """(name, body) of every kernel of the library's sources."""
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    for f in sorted(os.listdir(csrc)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, f)).read())
        for m in re.finditer(r"__global__ void (?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)|__maxnreg__\(\d+\))?\s*(\w+)\(", text):
            at = start = text.index("{", m.end())
            depth = 0
            while True:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
                if depth == 0:
                    break
            yield m.group(1), text[start + 1:at - 1]


def _before_wait(body):
    """The part of a kernel before its own wait for the launch in front of it (one that every path takes), or None."""
    for m in re.finditer(r"grid_dep_wait\(\)", body):
        head = body[:m.start()]
        if head.count("{") == head.count("}"):
            return head
    return None


def test_kernels_read_nothing_before_they_wait():
    """A kernel that may be resident while the launch before it drains sees what came before only behind griddepcontrol.wait,
    whatever that launch has waited for itself: no segment, row, page id or query is read ahead of it."""
    reads = re.compile(r"__ldg|load_seg|build_prefix|find_item|tc_item|locate\(|load_ids|bulk_load")
    heads = {name: _before_wait(body) for name, body in _kernels() if "grid_dep_" in body}
    assert {"kv8_append_small_kernel", "kv8_append_kernel", "kv8_attend_kernel", "kv8_chunk_kernel", "kv8_join_kernel",
            "attn_varlen_kernel", "norm_kernel"} <= set(heads)
    for name, head in heads.items():
        assert head is not None, name
        assert not reads.search(head), (name, reads.search(head).group())
    for f in ("kv8_append.cu", "kv8_attention.cu", "attention.cu", "elementwise.cu"):   # every launch that may overlap names such a kernel
        text = open(os.path.join(os.path.dirname(B.__file__), "csrc", f)).read()
        for m in re.finditer(r"hb_launch_kernel\((\w+)", text):
            assert m.group(1) in heads or m.group(1) in ("kern", "tc"), m.group(1)
