"""ctypes binding of libhb.so: argument marshalling only.

Every step of the path runs inside the library's CUDA kernels; torch is used
here for device memory and streams.  Importing this module loads the library
and raises if it has not been built -- there is no fallback of any kind.
"""
import ctypes as C
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhb.so")

HB_OK = 0
ERRORS = {0: "HB_OK", -1: "HB_ERR_BAD_ARG", -2: "HB_ERR_CUDA", -3: "HB_ERR_OOM_PAGES",
          -4: "HB_ERR_OOM_SLOTS", -5: "HB_ERR_TOO_LARGE", -6: "HB_ERR_BAD_DESC",
          -7: "HB_ERR_DEVICE_STATUS", -8: "HB_ERR_UNSUPPORTED"}
from .consts import (KIND_DECODE, KIND_PREFILL_CHUNK, KIND_EMBED_CHUNK, POOL_NONE, POOL_MEAN,  # noqa: F401,E402
                     POOL_LAST, POOL_CLS, POOL_WMEAN, POOL_MAX, EPI_F16, EPI_F32, EPI_RESID_F32, EPI_SWIGLU, CLASSES,
                     ROPE_PAIRS, ROPE_HALVES, ROPE_LINEAR, ROPE_BY_PARTS, LOGPROBS_MAX_K, DTYPE_F32, DTYPE_F16, DTYPE_BF16, DTYPE_E4M3,
                     ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH, NORM_MAX_D, LINEAR_MAX_GROUPS)


class HbError(RuntimeError):
    def __init__(self, code, what):
        super().__init__(f"{what}: {ERRORS.get(code, code)}")
        self.code = code


class ModelCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ffn", C.c_int32),
                ("vocab", C.c_int32), ("page_size", C.c_int32), ("max_pos", C.c_int32),
                ("rope_theta", C.c_float), ("rms_eps", C.c_float)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down")]


class Weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("layers", C.POINTER(LayerWeights)),
                ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class LayerWeights8(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "ffn_norm", "wqkv", "wo", "w_gate_up", "w_down", "wqkv_scale", "wo_scale",
                                          "gate_up_scale", "down_scale")]


class Weights8(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("layers", C.POINTER(LayerWeights8)), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class LoraLayer(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("a_qkv", "b_qkv", "a_o", "b_o", "a_gu", "b_gu", "a_d", "b_d")]


class Lora(C.Structure):
    _fields_ = [("rank", C.c_int32), ("scale", C.c_float), ("layers", C.POINTER(LoraLayer))]


class Seg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "q_start", "q_len", "pos_start", "pt_start", "pt_len",
                                         "pool_slot", "pool_mode", "is_final", "logits_row", "emb_row",
                                         "reserved")]


class BatchDesc(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("n_segs", C.c_int32), ("n_page_ids", C.c_int32),
                ("n_logit_rows", C.c_int32), ("n_emb_rows", C.c_int32),
                ("token_ids", C.POINTER(C.c_int32)), ("segs", C.POINTER(Seg)),
                ("page_ids", C.POINTER(C.c_int32))]


class RowsStruct(C.Structure):
    _fields_ = [("segs", C.c_void_p), ("page_ids", C.c_void_p), ("row_seg", C.c_void_p), ("n_segs", C.c_int32),
                ("n_page_ids", C.c_int32), ("n_rows", C.c_int32), ("max_q_len", C.c_int32), ("max_keys", C.c_int32)]


class AppendArgs(C.Structure):
    _fields_ = [("qkv", C.c_void_p), ("q_out", C.c_void_p), ("qkv_stride", C.c_int64), ("q_stride", C.c_int64),
                ("q_gain", C.c_void_p), ("k_gain", C.c_void_p), ("norm_eps", C.c_float), ("rope_cos", C.c_void_p),
                ("rope_sin", C.c_void_p), ("rope_rows", C.c_int32), ("rot_dim", C.c_int32), ("rope_layout", C.c_int32)]


class RopeScaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("factor", C.c_double), ("orig_len", C.c_double), ("lo", C.c_double),
                ("hi", C.c_double), ("attn_factor", C.c_double)]


class NormArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("x", "residual", "sum_out", "gain", "y", "y_scale")] + \
               [(n, C.c_int64) for n in ("x_stride", "residual_stride", "sum_stride", "y_stride")] + \
               [(n, C.c_int32) for n in ("x_dtype", "residual_dtype", "y_dtype", "n_rows", "d")] + [("eps", C.c_float)]


class LinearArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("a", "w", "a_scale", "w_scale", "bias", "residual", "c")] + \
               [(n, C.c_int64) for n in ("a_stride", "w_stride", "residual_stride", "c_stride")] + \
               [(n, C.c_int32) for n in ("m", "n", "k", "ab_dtype", "c_dtype", "residual_dtype", "act", "gated")]


SEG_DTYPE = np.dtype([(n, np.int32) for n, _ in Seg._fields_])

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_25405_b200.build` "
                      "(there is no CPU fallback)")
lib = C.CDLL(LIB_PATH)

_P = C.c_void_p
_sig = {
    "hb_workspace_bytes": [C.POINTER(ModelCfg), C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)],
    "hb_create": [C.POINTER(ModelCfg), C.c_int32, C.c_int32, C.c_int32, _P, C.c_size_t, C.POINTER(_P)],
    "hb_destroy": [_P],
    "hb_kv_arena_bytes": [C.POINTER(ModelCfg), C.c_int32, C.POINTER(C.c_size_t)],
    "hb_kv_create": [C.POINTER(ModelCfg), _P, C.c_size_t, C.c_int32, C.POINTER(_P)],
    "hb_kv_destroy": [_P],
    "hb_kv_alloc_pages": [_P, C.c_int32, C.POINTER(C.c_int32)],
    "hb_kv_free_pages": [_P, C.c_int32, C.POINTER(C.c_int32)],
    "hb_kv_free_count": [_P, C.POINTER(C.c_int32)],
    "hb_kv8_arena_bytes": [C.POINTER(ModelCfg), C.c_int32, C.POINTER(C.c_size_t)],
    "hb_kv8_create": [C.POINTER(ModelCfg), _P, C.c_size_t, C.c_int32, C.POINTER(_P)],
    "hb_kv8_append": [_P, _P, C.c_int32, C.POINTER(RowsStruct), C.POINTER(AppendArgs), _P],
    "hb_kv8_attention_workspace": [C.POINTER(ModelCfg), C.POINTER(RowsStruct), C.POINTER(C.c_size_t)],
    "hb_kv8_attention": [_P, _P, C.c_int32, C.POINTER(RowsStruct), _P, C.c_int64, _P, C.c_int64, C.c_float, _P,
                         C.c_size_t, _P],
    "hb_logprobs": [_P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_int64, _P, C.c_int32, _P, _P, _P, _P, _P],
    "hb_norm": [_P, C.POINTER(NormArgs), _P],
    "hb_quant_rows": [_P, _P, C.c_int32, C.c_int64, C.c_int32, _P, C.c_int32, C.c_int32, _P, C.c_int64, _P, _P],
    "hb_linear": [_P, C.POINTER(LinearArgs), _P],
    "hb_linear_grouped": [_P, C.POINTER(LinearArgs), _P, C.c_int32, C.c_int64, _P],
    "hb_linear_variant": [C.POINTER(LinearArgs), C.c_int32, C.c_int32, C.POINTER(C.c_int32)],
    "hb_rope_table": [C.c_int32, C.c_int32, C.c_double, C.POINTER(RopeScaling), _P, _P],
    "hb_pool_arena_bytes": [C.POINTER(ModelCfg), C.c_int32, C.POINTER(C.c_size_t)],
    "hb_pool_create": [C.POINTER(ModelCfg), _P, C.c_size_t, C.c_int32, C.POINTER(_P)],
    "hb_pool_destroy": [_P],
    "hb_pool_alloc_slot": [_P, C.POINTER(C.c_int32)],
    "hb_pool_free_slot": [_P, C.c_int32],
    "hb_pool_row_buffer_bytes": [_P, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)],
    "hb_pool_attach_row_buffer": [_P, _P, C.c_size_t, C.c_int32],
    "hb_validate_desc": [C.POINTER(ModelCfg), C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                         C.POINTER(BatchDesc)],
    "hb_mixed_step": [_P, C.POINTER(BatchDesc), C.POINTER(Weights), _P, _P, _P, _P, _P],
    "hb_mixed_step_lora": [_P, C.POINTER(BatchDesc), C.POINTER(Weights), C.POINTER(Lora), _P, _P, _P, _P, _P],
    "hb_mixed_step8": [_P, C.POINTER(BatchDesc), C.POINTER(Weights8), _P, _P, _P, _P, _P],
    "hb_weights_pack_f16": [_P, _P, C.c_size_t, _P],
    "hb_argmax": [_P, _P, C.c_int32, _P, _P],
    "hb_pool_chunk": [_P, _P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P, _P],
    "hb_pool_chunk_noalloc": [_P, _P, C.c_int32, C.c_int32, C.c_float, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P,
                              _P],
    "hb_gemm_pair": [_P, _P, _P, _P, _P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P],
    "hb_status_poll": [_P, _P, C.POINTER(C.c_uint32)],
    "hb_last_launch_count": [_P, C.POINTER(C.c_int32)],
    "hb_selftest_wait_expiry": [_P, C.c_uint32, _P],
    "hb_profile_enable": [_P, C.c_int],
    "hb_profile_read": [_P, C.POINTER(C.c_float), C.POINTER(C.c_int32)],
    "hb_gemm": [_P, _P, _P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P],
    "hb_gemm_set_walk": [C.c_int32, C.c_int32],
    "hb_gemm_set_cta_limit": [C.c_int32],
    "hb_attn_set_block_limit": [C.c_int32],
    "hb_attn_set_split_keys": [C.c_int32],
}
for _name, _args in _sig.items():
    _f = getattr(lib, _name)
    _f.argtypes = _args
    _f.restype = C.c_int
EXPORTS = tuple(_sig)


def check(code, what):
    if code != HB_OK:
        raise HbError(code, what)


def model_cfg(shape, max_pos):
    """hb_model_cfg from a synth.ModelShape-like object."""
    return ModelCfg(shape.L, shape.d, shape.Hq, shape.Hkv, shape.Dh, shape.F, shape.V,
                    shape.page_size, int(max_pos), float(shape.rope_theta), float(shape.rms_eps))


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _stream_of(stream, device_index):
    """Raw handle of `stream`, or of the device's current stream: without building a Stream object, which
    costs as much as a small kernel's launch."""
    return torch._C._cuda_getCurrentRawStream(device_index) if stream is None else stream.cuda_stream


def bf16_from_f32(a, device="cuda"):
    """numpy float32 (bf16-exact values) -> torch bf16 tensor on `device`, bit-exact."""
    bits = (np.ascontiguousarray(a, dtype=np.float32).view(np.uint32) >> np.uint32(16)).astype(np.uint16)
    return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)


def rope_pair_order(Dh):
    """Stored position j of a q/k head holds rotary element rope_pair_order(Dh)[j]:
    (0, Dh/2, 1, Dh/2 + 1, ...)."""
    half = Dh // 2
    order = np.empty(Dh, dtype=np.int64)
    order[0::2] = np.arange(half)
    order[1::2] = np.arange(half) + half
    return order


def rope_interleave_rows(w, Dh):
    """Reorder the rows of a q or k projection [H*Dh, d] into the library's pair-interleaved
    head layout (a layout change only: input marshalling)."""
    H = w.shape[0] // Dh
    idx = (np.arange(H)[:, None] * Dh + rope_pair_order(Dh)[None, :]).ravel()
    return w[idx]


def pack_f16_(t, stream=None):
    """Repack a bf16 tensor to fp16 in place (library kernel); returns the fp16 view."""
    assert t.dtype == torch.bfloat16 and t.is_contiguous()
    check(lib.hb_weights_pack_f16(C.c_void_p(t.data_ptr()), C.c_void_p(t.data_ptr()), t.numel(),
                                  _stream_ptr(stream)), "hb_weights_pack_f16")
    return t.view(torch.float16)


class DeviceWeights:
    """Weights resident in HBM in the library's layout (projection matrices repacked to fp16 in
    place, gains and token embedding bf16), plus the hb_weights struct."""

    def __init__(self, n_layers):
        self.tensors = []          # keep-alive
        self.layers = (LayerWeights * n_layers)()
        self.struct = Weights()
        self.struct.layers = C.cast(self.layers, C.POINTER(LayerWeights))

    def _keep(self, t):
        self.tensors.append(t)
        return t.data_ptr()

    @classmethod
    def from_synth(cls, W, device="cuda"):
        """Upload synth.Weights: q/k/v rows are concatenated, gate/up rows interleaved."""
        s = W.shape
        self = cls(s.L)
        up = lambda a: self._keep(bf16_from_f32(a, device))
        upw = lambda a: self._keep(pack_f16_(bf16_from_f32(a, device)))
        self.struct.tok_emb = up(W.tok_emb)
        self.struct.lm_head = upw(W.lm_head)
        self.struct.final_norm = up(W.final_norm)
        for l in range(s.L):
            w = W.layer(l)
            lw = self.layers[l]
            lw.attn_norm = up(w["attn_norm"])
            lw.ffn_norm = up(w["ffn_norm"])
            lw.wqkv = upw(np.concatenate([rope_interleave_rows(w["wq"], s.Dh), rope_interleave_rows(w["wk"], s.Dh),
                                          w["wv"]], axis=0))
            lw.wo = upw(w["wo"])
            gu = np.empty((2 * s.F, s.d), dtype=np.float32)
            gu[0::2] = w["wg"]
            gu[1::2] = w["wu"]
            lw.w_gate_up = upw(gu)
            lw.w_down = upw(w["wd"])
        return self

    @classmethod
    def random_on_device(cls, shape, seed=0, std=0.02, device="cuda"):
        """N(0, std^2) bf16 weights drawn on the device (benchmarks; not bit-matched to the
        host generator)."""
        self = cls(shape.L)
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def rnd(r, c, pack=True):
            t = torch.empty((r, c), dtype=torch.bfloat16, device=device)
            t.normal_(0.0, std, generator=g)
            return self._keep(pack_f16_(t) if pack else t)

        ones = lambda: self._keep(torch.ones(shape.d, dtype=torch.bfloat16, device=device))
        self.struct.tok_emb = rnd(shape.V, shape.d, pack=False)
        self.struct.lm_head = rnd(shape.V, shape.d)
        self.struct.final_norm = ones()
        for l in range(shape.L):
            lw = self.layers[l]
            lw.attn_norm = ones()
            lw.ffn_norm = ones()
            lw.wqkv = rnd(shape.n_qkv, shape.d)
            lw.wo = rnd(shape.d, shape.Hq * shape.Dh)
            lw.w_gate_up = rnd(2 * shape.F, shape.d)
            lw.w_down = rnd(shape.d, shape.F)
        return self


class DeviceWeights8:
    """Weights with the projections in 8 bits (e4m3 codes and a scale per row), plus the hb_weights8 struct; token embedding, gains
    and LM head as in DeviceWeights.  About half the memory of DeviceWeights; for an Engine with kv_dtype="e4m3"."""

    def __init__(self, n_layers, device="cuda"):
        self.tensors = []          # keep-alive
        self.layers = (LayerWeights8 * n_layers)()
        self.struct = Weights8()
        self.struct.layers = C.cast(self.layers, C.POINTER(LayerWeights8))
        self.codes = [{} for _ in range(n_layers)]   # per layer: name -> (codes, scale)
        self._device = device
        with torch.cuda.device(device):
            self._ctx = Context(ModelCfg(1, 64, 1, 1, 64, 64, 64, 16, 64, 1e4, 1e-5), 1, 1, 1)   # quantises the rows, on that device

    def _keep(self, t):
        self.tensors.append(t)
        return t.data_ptr()

    def _set(self, layer, name, scale_name, w):
        """Quantises the rows of w [out, in] (bf16, fp16 or fp32 on the device)."""
        codes = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=w.device)
        scale = torch.empty(w.shape[0], dtype=torch.float32, device=w.device)
        with torch.cuda.device(self._device):
            self._ctx.quant_rows(w, codes, scale)
        self.codes[layer][name] = (codes, scale)
        setattr(self.layers[layer], name, self._keep(codes))
        setattr(self.layers[layer], scale_name, self._keep(scale))

    def _packed_head(self, lm_head):
        with torch.cuda.device(self._device):
            return pack_f16_(lm_head)

    def _rest(self, tok_emb, final_norm, lm_head):
        self.struct.tok_emb, self.struct.final_norm, self.struct.lm_head = (self._keep(t) for t in (tok_emb, final_norm, lm_head))
        torch.cuda.synchronize(self._device)      # the rows' sources go when the caller's do
        self._ctx.close()
        return self

    @classmethod
    def from_synth(cls, W, device="cuda"):
        """Upload synth.Weights: rows in DeviceWeights' order, quantised by the library."""
        s = W.shape
        self = cls(s.L, device)
        up = lambda a: bf16_from_f32(a, device)   # noqa: E731
        for l in range(s.L):
            w = W.layer(l)
            self.layers[l].attn_norm, self.layers[l].ffn_norm = self._keep(up(w["attn_norm"])), self._keep(up(w["ffn_norm"]))
            gu = np.empty((2 * s.F, s.d), dtype=np.float32)
            gu[0::2], gu[1::2] = w["wg"], w["wu"]
            qkv = np.concatenate([rope_interleave_rows(w["wq"], s.Dh), rope_interleave_rows(w["wk"], s.Dh), w["wv"]], axis=0)
            for name, scale, a in (("wqkv", "wqkv_scale", qkv), ("wo", "wo_scale", w["wo"]), ("w_gate_up", "gate_up_scale", gu),
                                   ("w_down", "down_scale", w["wd"])):
                self._set(l, name, scale, up(a))
        return self._rest(up(W.tok_emb), up(W.final_norm), self._packed_head(up(W.lm_head)))

    @classmethod
    def random_on_device(cls, shape, seed=0, std=0.02, device="cuda"):
        """N(0, std^2) weights drawn on the device (benchmarks)."""
        self = cls(shape.L, device)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        rnd = lambda r, c: torch.empty((r, c), dtype=torch.bfloat16, device=device).normal_(0.0, std, generator=g)   # noqa: E731
        ones = lambda: torch.ones(shape.d, dtype=torch.bfloat16, device=device)   # noqa: E731
        for l in range(shape.L):
            self.layers[l].attn_norm, self.layers[l].ffn_norm = self._keep(ones()), self._keep(ones())
            for name, scale, r, c in (("wqkv", "wqkv_scale", shape.n_qkv, shape.d), ("wo", "wo_scale", shape.d, shape.Hq * shape.Dh),
                                      ("w_gate_up", "gate_up_scale", 2 * shape.F, shape.d), ("w_down", "down_scale", shape.d, shape.F)):
                self._set(l, name, scale, rnd(r, c))
        return self._rest(rnd(shape.V, shape.d), ones(), self._packed_head(rnd(shape.V, shape.d)))


def _pad64(n):
    return (n + 63) // 64 * 64


class DeviceLora:
    """Adapter factors resident in HBM in the library's packed layout (fp16), plus the hb_lora
    struct.  Packing is layout only: factors are stacked / placed in column blocks next to the fused
    weights they pair with; the bf16 -> fp16 repack runs in the library."""

    def __init__(self, n_layers, rank, scale):
        self.tensors = []
        self.layers = (LoraLayer * n_layers)()
        self.struct = Lora(int(rank), float(scale), C.cast(self.layers, C.POINTER(LoraLayer)))
        self.rank = int(rank)

    def _keep(self, t):
        self.tensors.append(t)
        return t.data_ptr()

    @staticmethod
    def _stack_down(factors, R):
        """A factors [r, in] stacked by rows into [R, in], zero padded."""
        out = np.zeros((R, factors[0].shape[1]), dtype=np.float32)
        at = 0
        for a in factors:
            out[at:at + a.shape[0]] = a
            at += a.shape[0]
        return out

    @classmethod
    def from_synth(cls, ad, device="cuda"):
        """Upload synth.LoraAdapters."""
        s, r = ad.shape, ad.rank
        self = cls(s.L, r, ad.scale)
        upw = lambda a: self._keep(pack_f16_(bf16_from_f32(a, device)))
        R1, R2, R3 = 64, _pad64(2 * r), _pad64(3 * r)
        for l in range(s.L):
            f = {n: ad.factors(l, n) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd")}
            ll = self.layers[l]
            ll.a_qkv = upw(self._stack_down([f["wq"][0], f["wk"][0], f["wv"][0]], R3))
            nq, nk = s.Hq * s.Dh, s.Hkv * s.Dh
            b = np.zeros((nq + 2 * nk, R3), dtype=np.float32)
            b[:nq, 0:r] = rope_interleave_rows(f["wq"][1], s.Dh)
            b[nq:nq + nk, r:2 * r] = rope_interleave_rows(f["wk"][1], s.Dh)
            b[nq + nk:, 2 * r:3 * r] = f["wv"][1]
            ll.b_qkv = upw(b)
            ll.a_o = upw(self._stack_down([f["wo"][0]], R1))
            b = np.zeros((s.d, R1), dtype=np.float32)
            b[:, :r] = f["wo"][1]
            ll.b_o = upw(b)
            ll.a_gu = upw(self._stack_down([f["wg"][0], f["wu"][0]], R2))
            b = np.zeros((2 * s.F, R2), dtype=np.float32)
            b[0::2, 0:r] = f["wg"][1]
            b[1::2, r:2 * r] = f["wu"][1]
            ll.b_gu = upw(b)
            ll.a_d = upw(self._stack_down([f["wd"][0]], R1))
            b = np.zeros((s.d, R1), dtype=np.float32)
            b[:, :r] = f["wd"][1]
            ll.b_d = upw(b)
        return self

    @classmethod
    def random_on_device(cls, shape, rank, seed=7, std=0.02, scale=2.0, device="cuda"):
        """Random factors drawn on the device in the packed layout (benchmarks): the blocks that the
        layout keeps at zero are zeroed after the draw."""
        self = cls(shape.L, rank, scale)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        r = rank
        R1, R2, R3 = 64, _pad64(2 * r), _pad64(3 * r)
        nq, nk = shape.Hq * shape.Dh, shape.Hkv * shape.Dh

        def rnd(rows, cols):
            t = torch.empty((rows, cols), dtype=torch.bfloat16, device=device)
            t.normal_(0.0, std, generator=g)
            return t

        fin = lambda t: self._keep(pack_f16_(t.contiguous()))
        for l in range(shape.L):
            ll = self.layers[l]
            a = rnd(R3, shape.d); a[3 * r:] = 0
            ll.a_qkv = fin(a)
            b = rnd(nq + 2 * nk, R3)
            keep = torch.zeros_like(b, dtype=torch.bool)
            keep[:nq, 0:r] = True; keep[nq:nq + nk, r:2 * r] = True; keep[nq + nk:, 2 * r:3 * r] = True
            ll.b_qkv = fin(torch.where(keep, b, torch.zeros_like(b)))
            a = rnd(R1, nq); a[r:] = 0
            ll.a_o = fin(a)
            b = rnd(shape.d, R1); b[:, r:] = 0
            ll.b_o = fin(b)
            a = rnd(R2, shape.d); a[2 * r:] = 0
            ll.a_gu = fin(a)
            b = rnd(2 * shape.F, R2)
            keep = torch.zeros_like(b, dtype=torch.bool)
            keep[0::2, 0:r] = True; keep[1::2, r:2 * r] = True
            ll.b_gu = fin(torch.where(keep, b, torch.zeros_like(b)))
            a = rnd(R1, shape.F); a[r:] = 0
            ll.a_d = fin(a)
            b = rnd(shape.d, R1); b[:, r:] = 0
            ll.b_d = fin(b)
        return self


def kv_arena_bytes(cfg, n_pages):
    nbytes = C.c_size_t()
    check(lib.hb_kv_arena_bytes(C.byref(cfg), n_pages, C.byref(nbytes)), "hb_kv_arena_bytes")
    return nbytes.value


class KvCache:
    """Caller-owned KV arena (torch) + the library's page free list.  `arena`: an int16 tensor to
    use instead of allocating one (it must hold n_pages; several caches may be laid over one
    buffer one after the other)."""

    def __init__(self, cfg, n_pages, device="cuda", fill=None, arena=None):
        self.cfg = cfg
        self.n_pages = n_pages
        nbytes = C.c_size_t(kv_arena_bytes(cfg, n_pages))
        self.handle = C.c_void_p()
        if device is None:      # bookkeeping only (host tests): no arena
            self.arena = None
            check(lib.hb_kv_create(C.byref(cfg), None, 0, n_pages, C.byref(self.handle)), "hb_kv_create")
            return
        if arena is not None:
            if arena.dtype != torch.int16 or arena.numel() * 2 < nbytes.value:
                raise ValueError("arena too small for n_pages")
            self.arena = arena[: nbytes.value // 2]
        else:
            self.arena = torch.empty(nbytes.value // 2, dtype=torch.int16, device=device)
        if fill is not None:
            self.arena.fill_(fill)
        check(lib.hb_kv_create(C.byref(cfg), C.c_void_p(self.arena.data_ptr()), nbytes.value, n_pages,
                               C.byref(self.handle)), "hb_kv_create")

    def view(self):
        """fp16 view [L, page, Hkv, 2 (slot group), 2 (K|V), Dh/64, 8, 64] (the arena's own layout)."""
        c = self.cfg
        return self.arena.view(torch.float16).view(c.n_layers, self.n_pages, c.n_kv_heads, 2, 2, c.head_dim // 64,
                                                   8, 64)

    def rows(self, layer, pages, slots, is_v):
        """K (is_v = 0) or V (1) rows of `layer` at (pages[i], slots[i]) as [n, Hkv, Dh] fp16, in the
        stored head-dimension order."""
        v = self.view()[layer][:, :, :, is_v]                   # [page, Hkv, group, H2, 8, 64]
        r = v[pages, :, slots // 8, :, slots % 8, :]            # [n, Hkv, H2, 64]
        return r.reshape(r.shape[0], r.shape[1], -1)

    def alloc(self, n):
        ids = (C.c_int32 * max(n, 1))()
        check(lib.hb_kv_alloc_pages(self.handle, n, ids), "hb_kv_alloc_pages")
        return list(ids[:n])

    def free(self, ids):
        arr = (C.c_int32 * max(len(ids), 1))(*ids)
        check(lib.hb_kv_free_pages(self.handle, len(ids), arr), "hb_kv_free_pages")

    def free_count(self):
        n = C.c_int32()
        check(lib.hb_kv_free_count(self.handle, C.byref(n)), "hb_kv_free_count")
        return n.value

    def close(self):
        if self.handle:
            lib.hb_kv_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def kv8_arena_bytes(cfg, n_pages):
    nbytes = C.c_size_t()
    check(lib.hb_kv8_arena_bytes(C.byref(cfg), n_pages, C.byref(nbytes)), "hb_kv8_arena_bytes")
    return nbytes.value


class KvCache8(KvCache):
    """8-bit KV arena (e4m3 codes, one power-of-two scale per page and KV head for K and for V) + the
    library's page free list.  `arena`: a uint8 tensor to use instead of allocating one."""

    def __init__(self, cfg, n_pages, device="cuda", fill=None, arena=None):
        self.cfg = cfg
        self.n_pages = n_pages
        nbytes = kv8_arena_bytes(cfg, n_pages)
        self.handle = C.c_void_p()
        self.arena = None
        if device is not None:
            if arena is not None:
                if arena.dtype != torch.uint8 or arena.dim() != 1 or not arena.is_contiguous() or arena.numel() < nbytes or not arena.is_cuda:
                    raise ValueError("arena: a contiguous uint8 vector on the GPU that holds n_pages")
                self.arena = arena[:nbytes]
            else:
                self.arena = torch.empty(nbytes, dtype=torch.uint8, device=device)
            if fill is not None:
                self.arena.fill_(fill)
        self.index = self.arena.get_device() if self.arena is not None else -1
        ptr = C.c_void_p(self.arena.data_ptr()) if self.arena is not None else None
        check(lib.hb_kv8_create(C.byref(cfg), ptr, nbytes, n_pages, C.byref(self.handle)), "hb_kv8_create")

    def _blocks(self):
        c = self.cfg
        return self.arena.view(c.n_layers, self.n_pages, c.n_kv_heads, 32 * c.head_dim + 32)

    def codes(self):
        """[L, page, Hkv, 32 * Dh] float8_e4m3fn view: K codes, then V codes, in the arena's own order."""
        return self._blocks()[..., :32 * self.cfg.head_dim].view(torch.float8_e4m3fn)

    def scales(self):
        """[L, page, Hkv, 2] fp32 view: scale of K, scale of V."""
        d = 32 * self.cfg.head_dim
        return self._blocks()[..., d:d + 8].view(torch.float32)

    def view(self):
        raise TypeError("an 8-bit arena has no 16-bit view: use codes() and scales(), or rows()")

    def rows(self, layer, pages, slots, is_v):
        """K (is_v = 0) or V (1) rows of `layer` at (pages[i], slots[i]) as [n, Hkv, Dh] fp32 (code * scale)."""
        dh = self.cfg.head_dim
        d = torch.arange(dh, device=self.arena.device)
        t = torch.as_tensor(slots, device=self.arena.device).view(-1, 1)
        if is_v:
            at = 16 * dh + d // 32 * 512 + (d % 8 * 4 + t % 8 // 2) * 16 + d % 32 // 8 * 4 + t // 8 * 2 + t % 2
        else:
            at = d // 64 * 1024 + t * 64 + d % 64
        pages = torch.as_tensor(pages, device=self.arena.device)
        bytes_ = self._blocks()[layer][pages].gather(2, at[:, None].expand(-1, self.cfg.n_kv_heads, -1))
        return bytes_.view(torch.float8_e4m3fn).float() * self.scales()[layer][pages][..., is_v, None]


class SegRows:
    """The rows of a step in device memory, as the operators over the 8-bit cache read them: segs int32
    [R, 12] (SEG_DTYPE), page_ids int32, row_seg int32 [T] (segment of each row, -1 = padding).
    max_q_len / max_keys bound every segment's q_len and pos_start + q_len."""

    def __init__(self, segs, page_ids, row_seg, max_q_len, max_keys):
        for t, n in ((segs, "segs"), (page_ids, "page_ids"), (row_seg, "row_seg")):
            if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous() or t.device != segs.device:
                raise ValueError(f"{n}: a contiguous int32 tensor on the GPU")
        if segs.dim() != 2 or segs.shape[1] != 12 or page_ids.dim() != 1 or row_seg.dim() != 1:
            raise ValueError("segs [R, 12], page_ids [n], row_seg [T]")
        self.segs, self.page_ids, self.row_seg = segs, page_ids, row_seg
        self.index = segs.get_device()
        self._need = {}            # workspace bytes by (n_heads, n_kv_heads, head_dim)
        self.struct = RowsStruct(segs.data_ptr(), page_ids.data_ptr(), row_seg.data_ptr(), segs.shape[0],
                                 page_ids.shape[0], row_seg.shape[0], int(max_q_len), int(max_keys))

    def workspace_bytes(self, cfg):
        """hb_kv8_attention_workspace of these rows."""
        key = (cfg.n_heads, cfg.n_kv_heads, cfg.head_dim)
        if key not in self._need:
            need = C.c_size_t()
            check(lib.hb_kv8_attention_workspace(C.byref(cfg), C.byref(self.struct), C.byref(need)), "hb_kv8_attention_workspace")
            self._need[key] = need.value
        return self._need[key]

    @classmethod
    def from_batch(cls, batch, device="cuda"):
        """Upload a Batch's segments and page lists."""
        segs = batch.segs
        row_seg = np.repeat(np.arange(len(segs), dtype=np.int32), segs["q_len"])
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
        return cls(up(segs.view(np.int32).reshape(len(segs), 12)), up(batch.page_ids), up(row_seg),
                   int(segs["q_len"].max(initial=0)), int((segs["pos_start"] + segs["q_len"]).max(initial=0)))


class Rope:
    """Rotary tables on the device: cos / sin fp32 [positions, rot_dim / 2], and which dimensions pair up."""

    def __init__(self, cos, sin, layout=ROPE_PAIRS):
        for t in (cos, sin):
            if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape != cos.shape or \
                    t.device != cos.device:
                raise ValueError("cos / sin: contiguous fp32 tensors [positions, rot_dim / 2] on the GPU")
        self.cos, self.sin, self.layout = cos, sin, layout
        self.index = cos.get_device()
        self.fields = (cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], layout)

    @classmethod
    def table(cls, n_pos, rot_dim, theta, layout=ROPE_PAIRS, scaling=None, device="cuda"):
        """Tables from hb_rope_table; `scaling`: RopeScaling or None."""
        cos, sin = rope_table(n_pos, rot_dim, theta, scaling)
        return cls(torch.from_numpy(cos).to(device), torch.from_numpy(sin).to(device), layout)


def rope_table(n_pos, rot_dim, theta, scaling=None):
    """(cos, sin) numpy fp32 [n_pos, rot_dim / 2] (host only)."""
    cos = np.empty((max(int(n_pos), 0), max(int(rot_dim), 0) // 2), dtype=np.float32)
    sin = np.empty_like(cos)
    check(lib.hb_rope_table(n_pos, rot_dim, float(theta), C.byref(scaling) if scaling is not None else None,
                            cos.ctypes.data_as(_P), sin.ctypes.data_as(_P)), "hb_rope_table")
    return cos, sin


def _rows_f16(t, rows, cols, device_index, name):
    """A [>= rows, cols] fp16 matrix with unit column stride: (pointer, row stride)."""
    if t.dtype is torch.float16 and t.get_device() == device_index and t.dim() == 2:
        have, c = t.shape
        stride, unit = t.stride()
        if c == cols and have >= rows and (unit == 1 or rows == 0):
            return t.data_ptr(), (stride if rows > 1 or stride >= cols else cols)
    raise ValueError(f"{name}: an fp16 tensor [{rows}, {cols}] with unit column stride on cuda:{device_index}")


_DTYPES = {torch.float32: DTYPE_F32, torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16, torch.float8_e4m3fn: DTYPE_E4M3}
# The argument structs of the dense operators as bytes, and the calls that take them so: building a ctypes structure costs
# more than a small kernel runs.
_pack_norm = struct.Struct("6Q4q5if").pack
_pack_linear = struct.Struct("7Q4q8i").pack
_dense = C.CDLL(LIB_PATH)
_dense.hb_norm.argtypes = [_P, C.c_char_p, _P]
_dense.hb_linear.argtypes = [_P, C.c_char_p, _P]
_dense.hb_linear_grouped.argtypes = [_P, C.c_char_p, _P, C.c_int32, C.c_int64, _P]


def _matrix(t, device_index, name):
    """A matrix with unit column stride: (pointer, rows, columns, row stride, HB_DTYPE_*)."""
    shape = t.shape
    if len(shape) == 2 and t.get_device() == device_index and t.dtype in _DTYPES:
        rows, cols = shape
        stride, unit = t.stride()
        if rows > 0x7fffffff or cols > 0x7fffffff:
            raise ValueError(f"{name}: at most 2^31 - 1 rows and columns")
        if unit == 1 or cols == 1 or rows == 0 or cols == 0:
            return t.data_ptr(), rows, cols, (stride if rows > 1 else (cols + 15) // 16 * 16), _DTYPES[t.dtype]   # (one row: any stride)
    raise ValueError(f"{name}: an fp32, fp16, bf16 or e4m3 matrix with unit column stride on cuda:{device_index}")


def _packed(t, dtype, shape, device_index, name):
    """Pointer of a contiguous tensor of that shape, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device_index or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor {list(shape)} on cuda:{device_index}")
    return t.data_ptr()


class Pool:
    """Caller-owned pooling arena (torch) + the library's slot free list."""

    def __init__(self, cfg, n_slots, device="cuda", fill=None):
        self.cfg = cfg
        self.n_slots = n_slots
        nbytes = C.c_size_t()
        check(lib.hb_pool_arena_bytes(C.byref(cfg), n_slots, C.byref(nbytes)), "hb_pool_arena_bytes")
        self.handle = C.c_void_p()
        if device is None:      # bookkeeping only (host tests): no arena
            self.arena = None
            check(lib.hb_pool_create(C.byref(cfg), None, 0, n_slots, C.byref(self.handle)), "hb_pool_create")
            return
        self.arena = torch.empty((nbytes.value + 3) // 4, dtype=torch.int32, device=device)
        if fill is not None:
            self.arena.fill_(fill)
        check(lib.hb_pool_create(C.byref(cfg), C.c_void_p(self.arena.data_ptr()), nbytes.value, n_slots,
                                 C.byref(self.handle)), "hb_pool_create")

    def attach_row_buffer(self, max_rows, fill=None):
        """Row buffer for buffered heads (POOL_MAX): [n_slots, max_rows, d] fp32, caller-owned."""
        nbytes = C.c_size_t()
        check(lib.hb_pool_row_buffer_bytes(C.byref(self.cfg), self.n_slots, max_rows, C.byref(nbytes)),
              "hb_pool_row_buffer_bytes")
        self.rows = torch.empty((self.n_slots, max_rows, self.cfg.d_model), dtype=torch.float32,
                                device=self.arena.device)
        if fill is not None:
            self.rows.fill_(fill)
        check(lib.hb_pool_attach_row_buffer(self.handle, C.c_void_p(self.rows.data_ptr()), nbytes.value, max_rows),
              "hb_pool_attach_row_buffer")
        return self.rows

    def sums(self):
        d = self.cfg.d_model
        return self.arena[: self.n_slots * d].view(torch.float32).view(self.n_slots, d)

    def meta(self):
        d = self.cfg.d_model
        return self.arena[self.n_slots * d: self.n_slots * d + self.n_slots * 4].view(self.n_slots, 4)

    def alloc(self):
        s = C.c_int32()
        check(lib.hb_pool_alloc_slot(self.handle, C.byref(s)), "hb_pool_alloc_slot")
        return s.value

    def free(self, slot):
        check(lib.hb_pool_free_slot(self.handle, slot), "hb_pool_free_slot")

    def close(self):
        if self.handle:
            lib.hb_pool_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Batch:
    """Host descriptor arrays (numpy, kept alive) and the hb_batch_desc over them."""

    def __init__(self, token_ids, segs, page_ids, n_logit_rows, n_emb_rows):
        self.token_ids = np.ascontiguousarray(token_ids, dtype=np.int32)
        self.segs = np.ascontiguousarray(segs, dtype=SEG_DTYPE)
        self.page_ids = np.ascontiguousarray(page_ids, dtype=np.int32)
        self.desc = BatchDesc(len(self.token_ids), len(self.segs), len(self.page_ids), n_logit_rows,
                              n_emb_rows,
                              self.token_ids.ctypes.data_as(C.POINTER(C.c_int32)),
                              self.segs.ctypes.data_as(C.POINTER(Seg)),
                              self.page_ids.ctypes.data_as(C.POINTER(C.c_int32)))

    @property
    def n_tokens(self):
        return len(self.token_ids)

    def host_bytes(self):
        return self.token_ids.nbytes + self.segs.nbytes + self.page_ids.nbytes


class Context:
    def __init__(self, cfg, max_tokens, max_segs, max_page_ids):
        if not torch.cuda.is_available():
            raise RuntimeError("libhb needs a CUDA device (B200); there is no CPU path")
        self.cfg = cfg
        self.handle = C.c_void_p()
        self.index = torch.cuda.current_device()
        self.device = torch.device("cuda", self.index)
        check(lib.hb_create(C.byref(cfg), max_tokens, max_segs, max_page_ids, None, 0, C.byref(self.handle)),
              "hb_create")

    def mixed_step(self, batch, weights, kv, pool, out_logits, out_emb, stream=None, lora=None):
        tail = (kv.handle, pool.handle if pool is not None else None,
                C.c_void_p(out_logits.data_ptr()) if out_logits is not None else None,
                C.c_void_p(out_emb.data_ptr()) if out_emb is not None else None, _stream_ptr(stream))
        if isinstance(weights, DeviceWeights8):
            if lora is not None or not isinstance(kv, KvCache8):
                raise ValueError("8-bit weights: with an 8-bit cache (KvCache8) and without adapters")
            check(lib.hb_mixed_step8(self.handle, C.byref(batch.desc), C.byref(weights.struct), *tail), "hb_mixed_step8")
        elif lora is None:
            check(lib.hb_mixed_step(self.handle, C.byref(batch.desc), C.byref(weights.struct), *tail), "hb_mixed_step")
        else:
            check(lib.hb_mixed_step_lora(self.handle, C.byref(batch.desc), C.byref(weights.struct),
                                         C.byref(lora.struct), *tail), "hb_mixed_step_lora")

    def argmax(self, logits, n_rows, out_tokens, stream=None):
        check(lib.hb_argmax(self.handle, C.c_void_p(logits.data_ptr()), n_rows,
                            C.c_void_p(out_tokens.data_ptr()), _stream_ptr(stream)), "hb_argmax")

    def logprobs(self, logits, tokens, out_logprob, out_entropy=None, out_top_ids=None, out_top_logprobs=None, stream=None):
        """hb_logprobs: logits fp32 or fp16 [n, vocab] (rows may be strided), tokens int32 [n] (negative = none),
        out_logprob fp32 [n] (tokens and out_logprob both or neither None), out_entropy fp32 [n], and the
        k = out_top_ids.shape[1] best alternatives: out_top_ids int32 [n, k], out_top_logprobs fp32 [n, k]."""
        dev, dt = self.index, logits.dtype
        if logits.dim() != 2 or (dt is not torch.float32 and dt is not torch.float16) or logits.get_device() != dev or \
                (logits.stride(1) != 1 and logits.numel()):
            raise ValueError(f"logits: fp32 or fp16 [n, vocab] with unit column stride on {self.device}")
        n, vocab = logits.shape
        k = 0 if out_top_ids is None else out_top_ids.size(-1)
        tp = self._vector(tokens, torch.int32, n, 1, "tokens")
        lp = self._vector(out_logprob, torch.float32, n, 1, "out_logprob")
        ep = self._vector(out_entropy, torch.float32, n, 1, "out_entropy")
        ip = self._vector(out_top_ids, torch.int32, n, k, "out_top_ids")
        vp = self._vector(out_top_logprobs, torch.float32, n, k, "out_top_logprobs")
        stride = logits.stride(0)
        if n <= 1 and stride < vocab:
            stride = vocab
        rc = lib.hb_logprobs(self.handle, logits.data_ptr(), DTYPE_F32 if dt is torch.float32 else DTYPE_F16, n, vocab, stride, tp,
                             k, lp, ep, ip, vp, _stream_of(stream, dev))
        if rc != HB_OK:
            raise HbError(rc, "hb_logprobs")

    def _vector(self, t, dtype, n, k, name):
        """Pointer of a contiguous [n] (k = 1) or [n, k] tensor, or None."""
        if t is None:
            return None
        if t.dtype is not dtype or t.get_device() != self.index or t.dim() > 2 or t.size(0) != n or t.numel() != n * k or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous {dtype} tensor of {n} x {k} on {self.device}")
        return t.data_ptr()

    def norm(self, x, gain, y, residual=None, sum_out=None, y_scale=None, eps=None, stream=None):
        """hb_norm: y = rmsnorm(x + residual) * gain over rows [n, d] (fp32, fp16 or bf16; y also float8_e4m3fn with
        y_scale fp32 [n]).  gain bf16 [d] or None; sum_out takes x + residual in the residual's type (it may be the residual);
        eps: None = the model's."""
        dev = self.index
        xp, n, d, xs, xt = _matrix(x, dev, "x")
        yp, yn, yd, ys, yt = _matrix(y, dev, "y")
        if yn != n or yd != d:
            raise ValueError(f"y: {n} x {d}, as x")
        rp = sp = rs = ss = rt = 0
        if residual is not None:
            rp, rn, rd, rs, rt = _matrix(residual, dev, "residual")
            if rn != n or rd != d:
                raise ValueError(f"residual: {n} x {d}, as x")
        if sum_out is not None:
            if sum_out is residual:
                sp, ss = rp, rs
            else:
                sp, sn, sd, ss, st = _matrix(sum_out, dev, "sum_out")
                if residual is None or sn != n or sd != d or st != rt:
                    raise ValueError(f"sum_out: {n} x {d} of the residual's type, with a residual")
        args = _pack_norm(xp, rp, sp, _packed(gain, torch.bfloat16, (d,), dev, "gain"), yp,
                          _packed(y_scale, torch.float32, (n,), dev, "y_scale"), xs, rs, ss, ys, xt, rt, yt, n, d,
                          self.cfg.rms_eps if eps is None else eps)
        rc = _dense.hb_norm(self.handle, args, _stream_of(stream, dev))
        if rc:
            raise HbError(rc, "hb_norm")

    def quant_rows(self, x, codes, scale, index=None, stream=None):
        """hb_quant_rows: codes float8_e4m3fn [n, d] and scale fp32 [n] of the rows of x (fp32, fp16 or bf16), in order or row
        index[r] (int32 [n]; negative leaves row r as it is)."""
        dev = self.index
        xp, n_src, d, xs, xt = _matrix(x, dev, "x")
        cp, n, cd, cs, ct = _matrix(codes, dev, "codes")
        if cd != d or ct != DTYPE_E4M3 or (index is None and n != n_src):
            raise ValueError(f"codes: float8_e4m3fn, {d} columns and a row for each row of x or entry of index")
        rc = lib.hb_quant_rows(self.handle, xp, xt, xs, n_src, _packed(index, torch.int32, (n,), dev, "index"), n, d, cp, cs,
                               _packed(scale, torch.float32, (n,), dev, "scale"), _stream_of(stream, dev))
        if rc:
            raise HbError(rc, "hb_quant_rows")

    def _linear_args(self, a, wp, n, k, ws, wt, per_column, out, a_scale, w_scale, bias, act, gated, residual):
        dev = self.index
        ap, m, ka, as_, at = _matrix(a, dev, "a")
        cp, cm, cn, cs, ct = _matrix(out, dev, "out")
        if ka != k or at != wt:
            raise ValueError(f"a: {k} columns of the weight's type")
        if cm != m or cn != (n // 2 if gated else n):
            raise ValueError(f"out: {m} x {n // 2 if gated else n}")
        rp = rs = rt = 0
        if residual is not None:
            rp, rm, rn, rs, rt = _matrix(residual, dev, "residual")
            if rm != cm or rn != cn:
                raise ValueError(f"residual: {cm} x {cn}, as out")
        return _pack_linear(ap, wp, _packed(a_scale, torch.float32, (m,), dev, "a_scale"),
                            _packed(w_scale, torch.float32, per_column, dev, "w_scale"),
                            _packed(bias, torch.float32, per_column, dev, "bias"), rp, cp, as_, ws, rs, cs, m, n, k, wt, ct, rt, act,
                            1 if gated else 0)

    def linear(self, a, w, out, a_scale=None, w_scale=None, bias=None, act=ACT_NONE, gated=False, residual=None, stream=None):
        """hb_linear: out = act(a_scale w_scale a w^T + bias) + residual.  a [m, k] and w [n, k] of one type (fp16, bf16 or
        float8_e4m3fn, rows on 16-byte boundaries), out and residual fp32, fp16 or bf16 [m, n], or [m, n / 2] where `gated`
        joins pairs of columns; a_scale fp32 [m], w_scale and bias fp32 [n]."""
        wp, n, k, ws, wt = _matrix(w, self.index, "w")
        args = self._linear_args(a, wp, n, k, ws, wt, (n,), out, a_scale, w_scale, bias, act, gated, residual)
        rc = _dense.hb_linear(self.handle, args, _stream_of(stream, self.index))
        if rc:
            raise HbError(rc, "hb_linear")

    def linear_grouped(self, a, w, group_start, out, a_scale=None, w_scale=None, bias=None, act=ACT_NONE, gated=False,
                       residual=None, stream=None):
        """hb_linear_grouped: linear() where rows group_start[g] .. group_start[g + 1] - 1 take w[g]: w [groups, n, k],
        group_start int32 [groups + 1] on the device, w_scale and bias fp32 [groups, n]."""
        shape, dev = w.shape, self.index
        if len(shape) != 3 or shape[0] < 1 or w.dtype not in _DTYPES or w.get_device() != dev:
            raise ValueError(f"w: fp16, bf16 or e4m3 [groups, n, k] on cuda:{dev}")
        groups, n, k = shape
        step, ws, unit = w.stride()
        if max(shape) > 0x7fffffff:
            raise ValueError("w: at most 2^31 - 1 groups, rows and columns")
        if unit != 1 and k > 1:
            raise ValueError("w: unit stride along k")
        if n == 1:
            ws = (k + 15) // 16 * 16
        if group_start is None:
            raise ValueError("group_start: int32 [groups + 1]")
        args = self._linear_args(a, w.data_ptr(), n, k, ws, _DTYPES[w.dtype], (groups, n), out, a_scale, w_scale, bias, act, gated, residual)
        rc = _dense.hb_linear_grouped(self.handle, args, _packed(group_start, torch.int32, (groups + 1,), dev, "group_start"),
                                      groups, step if groups > 1 else n * ws, _stream_of(stream, dev))
        if rc:
            raise HbError(rc, "hb_linear_grouped")

    def gemm_pair(self, A, B, A2, B2, Cout, M, N, K, K2, epilogue, stream=None):
        check(lib.hb_gemm_pair(self.handle, C.c_void_p(A.data_ptr()), C.c_void_p(B.data_ptr()),
                               C.c_void_p(A2.data_ptr()), C.c_void_p(B2.data_ptr()), C.c_void_p(Cout.data_ptr()),
                               M, N, K, K2, epilogue, _stream_ptr(stream)), "hb_gemm_pair")

    def gemm(self, A, B, Cout, M, N, K, epilogue, stream=None):
        check(lib.hb_gemm(self.handle, C.c_void_p(A.data_ptr()), C.c_void_p(B.data_ptr()),
                          C.c_void_p(Cout.data_ptr()), M, N, K, epilogue, _stream_ptr(stream)), "hb_gemm")

    def pool_chunk(self, x, gain, n_rows, mode, first_chunk, is_final, slot_sum, slot_meta, out_emb, stream=None):
        check(lib.hb_pool_chunk(self.handle, C.c_void_p(x.data_ptr()), C.c_void_p(gain.data_ptr()), n_rows, mode,
                                1 if first_chunk else 0, 1 if is_final else 0, C.c_void_p(slot_sum.data_ptr()),
                                C.c_void_p(slot_meta.data_ptr()),
                                C.c_void_p(out_emb.data_ptr()) if out_emb is not None else None,
                                _stream_ptr(stream)), "hb_pool_chunk")

    def _same_device(self, rows, kv):
        if not isinstance(kv, KvCache8):
            raise TypeError("an 8-bit cache (KvCache8)")
        if rows.index != self.index or kv.index != self.index:
            raise ValueError(f"rows and cache on the context's device, {self.device}")
        return self.index

    def _head_gain(self, gain, name):
        if gain is None:
            return None
        if gain.dtype is not torch.bfloat16 or gain.get_device() != self.index or gain.shape != (self.cfg.head_dim,) or \
                not gain.is_contiguous():
            raise ValueError(f"{name}: a contiguous bf16 tensor [{self.cfg.head_dim}] on {self.device}")
        return gain.data_ptr()

    def kv8_append(self, kv, layer, rows, qkv, q_out, rope=None, q_norm=None, k_norm=None, norm_eps=1e-6, stream=None):
        """hb_kv8_append: head norms (bf16 gains [Dh] or None), rotation (Rope or None), K / V of every row of
        `rows` (SegRows) appended to layer `layer` of a KvCache8; qkv fp16 [T, (Hq + 2 Hkv) Dh], q_out
        fp16 [T, Hq Dh] (rows may be strided views)."""
        c = self.cfg
        T, dev = rows.struct.n_rows, self._same_device(rows, kv)
        xp, xs = _rows_f16(qkv, T, (c.n_heads + 2 * c.n_kv_heads) * c.head_dim, dev, "qkv")
        qp, qs = _rows_f16(q_out, T, c.n_heads * c.head_dim, dev, "q_out")
        cos = sin = None
        n_pos = rot = layout = 0
        if rope is not None:
            if rope.index != dev:
                raise ValueError(f"rope: tables on cuda:{dev}")
            cos, sin, n_pos, rot, layout = rope.fields
        a = AppendArgs(xp, qp, xs, qs, self._head_gain(q_norm, "q_norm"), self._head_gain(k_norm, "k_norm"), norm_eps, cos, sin,
                       n_pos, rot, layout)
        rc = lib.hb_kv8_append(self.handle, kv.handle, layer, C.byref(rows.struct), C.byref(a), _stream_of(stream, dev))
        if rc != HB_OK:
            raise HbError(rc, "hb_kv8_append")

    def kv8_attention(self, kv, layer, rows, q, out, scale=0.0, stream=None):
        """hb_kv8_attention: causal attention of every row of `rows` over its request's pages of layer `layer` of a
        KvCache8; q and out fp16 [T, Hq Dh] (rows may be strided views); scale 0 = 1 / sqrt(Dh), at most 2^60.  The
        workspace of the call comes from torch's allocator, on the stream of the call."""
        c = self.cfg
        T, dev = rows.struct.n_rows, self._same_device(rows, kv)
        qp, qs = _rows_f16(q, T, c.n_heads * c.head_dim, dev, "q")
        op, os_ = _rows_f16(out, T, c.n_heads * c.head_dim, dev, "out")
        need, ws, wp = rows.workspace_bytes(c), None, None
        if need:   # allocated on the stream of the call, whose order then protects its reuse
            if stream is None:
                ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            else:
                with torch.cuda.stream(stream):
                    ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            wp = ws.data_ptr()
        rc = lib.hb_kv8_attention(self.handle, kv.handle, layer, C.byref(rows.struct), qp, qs, op, os_, scale, wp, need,
                                  _stream_of(stream, dev))
        if rc != HB_OK:
            raise HbError(rc, "hb_kv8_attention")

    def status_poll(self, stream=None):
        """Synchronises the stream; returns the device status code (0 = clean)."""
        code = C.c_uint32()
        rc = lib.hb_status_poll(self.handle, _stream_ptr(stream), C.byref(code))
        if rc not in (HB_OK, -7):
            raise HbError(rc, "hb_status_poll")
        return code.value

    def profile_enable(self, on):
        check(lib.hb_profile_enable(self.handle, 1 if on else 0), "hb_profile_enable")

    def profile_read(self):
        """{class name: (milliseconds, launches)} accumulated since the last read."""
        ms = (C.c_float * len(CLASSES))()
        n = (C.c_int32 * len(CLASSES))()
        check(lib.hb_profile_read(self.handle, ms, n), "hb_profile_read")
        return {CLASSES[i]: (float(ms[i]), int(n[i])) for i in range(len(CLASSES))}

    def selftest_wait_expiry(self, limit_ms=20, stream=None):
        check(lib.hb_selftest_wait_expiry(self.handle, limit_ms, _stream_ptr(stream)), "hb_selftest_wait_expiry")

    def last_launch_count(self):
        n = C.c_int32()
        check(lib.hb_last_launch_count(self.handle, C.byref(n)), "hb_last_launch_count")
        return n.value

    def close(self):
        if self.handle:
            lib.hb_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


NOALLOC_MAX_ROWS, NOALLOC_MAX_DMODEL = 2048, 4096


def pool_chunk_noalloc(x, gain, n_rows, d_model, rms_eps, mode, first_chunk, is_final, slot_sum, slot_meta,
                       out_emb, stream=None):
    """hb_pool_chunk_noalloc: the pooler for callers that may not allocate device memory (no
    context; scratch is a fixed array inside the library).  Returns the status code; sizes beyond
    NOALLOC_MAX_ROWS x NOALLOC_MAX_DMODEL give HB_ERR_TOO_LARGE (-5).  Calls that may overlap on
    the GPU must be serialised by the caller."""
    return lib.hb_pool_chunk_noalloc(C.c_void_p(x.data_ptr()), C.c_void_p(gain.data_ptr()), n_rows, d_model,
                                     float(rms_eps), mode, 1 if first_chunk else 0, 1 if is_final else 0,
                                     C.c_void_p(slot_sum.data_ptr()), C.c_void_p(slot_meta.data_ptr()),
                                     C.c_void_p(out_emb.data_ptr()) if out_emb is not None else None,
                                     _stream_ptr(stream))


def gemm_set_walk(band=-1, hints=-1):
    """Force the projection GEMM's tile walk (tests / tuning); -1 = automatic."""
    check(lib.hb_gemm_set_walk(band, hints), "hb_gemm_set_walk")


def gemm_set_cta_limit(max_ctas=0):
    """Cap the CTAs of every projection GEMM launch (tuning); 0 = one per SM."""
    check(lib.hb_gemm_set_cta_limit(max_ctas), "hb_gemm_set_cta_limit")


def attn_set_block_limit(max_blocks=0):
    """Cap the resident blocks of every attention launch (tests); 0 = two per SM."""
    check(lib.hb_attn_set_block_limit(max_blocks), "hb_attn_set_block_limit")


def attn_set_split_keys(keys=0):
    """Keys per decode attention item for contexts created from now on; 0 = the default (2048)."""
    check(lib.hb_attn_set_split_keys(keys), "hb_attn_set_split_keys")


def validate_desc(cfg, max_tokens, max_segs, max_page_ids, n_pages, n_slots, batch):
    """Host-only descriptor validation; returns the status code."""
    return lib.hb_validate_desc(C.byref(cfg), max_tokens, max_segs, max_page_ids, n_pages, n_slots,
                                C.byref(batch.desc))
