"""ctypes binding of ``libecospa.so`` (see ``include/ecospa.h``).

Argument marshalling only: every step runs in the library's HIP kernels.  PyTorch supplies
device memory (tensors) and the HIP stream.  There is no fallback: if the built library is
missing, :func:`load` raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libecospa.so")

OK, ERR_NULL, ERR_SHAPE, ERR_DTYPE, ERR_K, ERR_INDEX, ERR_WORKSPACE, ERR_ALIGN, ERR_HIP = range(9)
F32, BF16 = 0, 1
PAIR_QK, PAIR_VO, PAIR_FFN, PAIR_FFN_GATED = range(4)
BLOCK_ATTN, BLOCK_FFN = 0, 1
ACT_GELU_ERF, ACT_GELU_TANH, ACT_SWIGLU = range(3)
ACT_NONE = -1

EXPORTS = (
    "ecospa_create", "ecospa_destroy", "ecospa_set_workspace", "ecospa_status_string", "ecospa_last_error",
    "ecospa_score_workspace_bytes", "ecospa_coupled_score", "ecospa_select_topk", "ecospa_compact",
    "ecospa_scatter", "ecospa_rope_table", "ecospa_block_workspace_bytes", "ecospa_coupled_fwd",
    "ecospa_coupled_bwd", "ecospa_profile_gemm", "ecospa_profile_gemm_read", "ecospa_contract",
    "ecospa_select_topk_batch", "ecospa_compact_batch", "ecospa_pair_fisher", "ecospa_select_theta",
    "ecospa_select_pairs", "ecospa_rope_table_ragged", "ecospa_adamw", "ecospa_transpose_batch",
    "ecospa_check_indices", "ecospa_contract_workspace_bytes", "ecospa_hbm_probe", "ecospa_contract_colsum", "ecospa_mfma_probe",
    "ecospa_coupled_score_static", "ecospa_coupled_score_static_max_bytes",
    "ecospa_score_select", "ecospa_compact_batch_rope",
    "ecospa_norm_fwd", "ecospa_norm_bwd", "ecospa_norm_bwd_workspace_bytes", "ecospa_embed_fwd", "ecospa_embed_bwd", "ecospa_xent",
    "ecospa_cache_append", "ecospa_prefix_attn", "ecospa_prefix_attn_workspace_bytes", "ecospa_cache_evict",
    "ecospa_logits_process", "ecospa_logits_workspace_bytes",
    "ecospa_quant_rows", "ecospa_contract_quant",
    "ecospa_quant_cache_append", "ecospa_quant_cache_attn", "ecospa_quant_cache_attn_workspace_bytes",
    "ecospa_sample", "ecospa_sample_workspace_bytes",
)
NORM_RMS, NORM_LAYER = 0, 1


class EcospaError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: error {code} ({status_string(code)}) {detail}".strip())


class Pair(C.Structure):
    _fields_ = [("kind", C.c_int), ("dtype", C.c_int), ("groups", C.c_int), ("n", C.c_int), ("unit", C.c_int),
                ("d1", C.c_int), ("d2", C.c_int), ("w1", C.c_void_p), ("w1b", C.c_void_p), ("w2", C.c_void_p),
                ("ld1", C.c_longlong), ("ld1b", C.c_longlong), ("ld2", C.c_longlong), ("rep1", C.c_int), ("rep2", C.c_int),
                ("w2_rows", C.c_int)]


class BlockDesc(C.Structure):
    _fields_ = [("block", C.c_int), ("dtype", C.c_int), ("B", C.c_int), ("L", C.c_int), ("d_model", C.c_int),
                ("h", C.c_int), ("kp_qk", C.c_int), ("kp_vo", C.c_int), ("causal", C.c_int), ("scale", C.c_float),
                ("rope_cos", C.c_void_p), ("rope_sin", C.c_void_p),
                ("w_qkv", C.c_void_p), ("b_qkv", C.c_void_p), ("w_o", C.c_void_p), ("b_o", C.c_void_p),
                ("ld_wqkv", C.c_longlong), ("ld_wo", C.c_longlong),
                ("kp_ff", C.c_int), ("act", C.c_int),
                ("w_1", C.c_void_p), ("b_1", C.c_void_p), ("w_2", C.c_void_p), ("b_2", C.c_void_p),
                ("ld_w1", C.c_longlong), ("ld_w2", C.c_longlong), ("h_kv", C.c_int),
                ("w_qkv_t", C.c_void_p), ("w_o_t", C.c_void_p), ("w_1_t", C.c_void_p), ("w_2_t", C.c_void_p),
                ("ld_wqkvt", C.c_longlong), ("ld_wot", C.c_longlong), ("ld_w1t", C.c_longlong), ("ld_w2t", C.c_longlong)]


class SelectItem(C.Structure):
    _fields_ = [("scores", C.c_void_p), ("groups", C.c_int), ("n_units", C.c_int), ("k", C.c_int),
                ("idx", C.c_void_p)]


class MapItem(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("dtype", C.c_int), ("axis", C.c_int), ("groups", C.c_int),
                ("n", C.c_int), ("unit", C.c_int), ("k", C.c_int), ("kp", C.c_int), ("scatter", C.c_int),
                ("other_extent", C.c_longlong), ("ld_src", C.c_longlong), ("ld_dst", C.c_longlong),
                ("idx", C.c_void_p), ("k_group", C.c_void_p), ("ld_idx", C.c_int), ("idx_div", C.c_int),
                ("dst_t", C.c_void_p), ("ld_dst_t", C.c_longlong), ("src_b", C.c_void_p)]


class RopeItem(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("k_group", C.c_void_p), ("h", C.c_int), ("L", C.c_int), ("k", C.c_int), ("kp", C.c_int),
                ("d_h", C.c_int), ("ld_idx", C.c_int), ("base", C.c_double), ("cos_out", C.c_void_p), ("sin_out", C.c_void_p)]


class TransposeItem(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("dtype", C.c_int), ("rows", C.c_int), ("cols", C.c_int),
                ("ld_src", C.c_longlong), ("ld_dst", C.c_longlong)]


class AdamwItem(C.Structure):
    _fields_ = [("w", C.c_void_p), ("w_lp", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("n", C.c_longlong), ("w_dtype", C.c_int), ("g_dtype", C.c_int), ("s_dtype", C.c_int)]


class AdamwHyper(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("step", C.c_int)]


class Saved(C.Structure):
    _fields_ = [("qkv", C.c_void_p), ("o", C.c_void_p), ("lse", C.c_void_p), ("hpre", C.c_void_p),
                ("act", C.c_void_p)]


class Cache(C.Structure):
    _fields_ = [("dtype", C.c_int), ("B", C.c_int), ("h", C.c_int), ("h_kv", C.c_int), ("kp_qk", C.c_int), ("kp_vo", C.c_int),
                ("cap", C.c_int), ("own_max", C.c_int), ("P", C.c_int), ("scale", C.c_float), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_sb", C.c_longlong), ("k_sh", C.c_longlong), ("k_st", C.c_longlong), ("v_sb", C.c_longlong), ("v_sh", C.c_longlong),
                ("v_st", C.c_longlong), ("pk", C.c_void_p), ("pv", C.c_void_p), ("pk_sh", C.c_longlong), ("pk_st", C.c_longlong),
                ("pv_sh", C.c_longlong), ("pv_st", C.c_longlong), ("lens", C.c_void_p)]


class Logits(C.Structure):
    _fields_ = [("B", C.c_int), ("V", C.c_int), ("dtype", C.c_int), ("out_dtype", C.c_int), ("logits", C.c_void_p), ("out", C.c_void_p),
                ("ld", C.c_longlong), ("ld_out", C.c_longlong), ("history", C.c_void_p), ("history_len", C.c_void_p), ("ld_history", C.c_int),
                ("n_bias", C.c_int), ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p), ("temperature", C.c_void_p),
                ("bias_ids", C.c_void_p), ("bias", C.c_void_p), ("mask", C.c_void_p), ("mask_row", C.c_void_p), ("ld_mask", C.c_longlong),
                ("n_masks", C.c_int), ("pick", C.c_void_p), ("lse", C.c_void_p)]


class QuantCacheDesc(C.Structure):
    _fields_ = [("B", C.c_int), ("h", C.c_int), ("h_kv", C.c_int), ("kp_qk", C.c_int), ("kp_vo", C.c_int), ("cap", C.c_int), ("own_max", C.c_int),
                ("block", C.c_int), ("scale", C.c_float), ("k", C.c_void_p), ("v", C.c_void_p), ("k_sb", C.c_longlong), ("k_sh", C.c_longlong),
                ("k_st", C.c_longlong), ("v_sb", C.c_longlong), ("v_sh", C.c_longlong), ("v_st", C.c_longlong), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("lens", C.c_void_p)]


class SampleArgs(C.Structure):
    _fields_ = [("B", C.c_int), ("V", C.c_int), ("dtype", C.c_int), ("logits", C.c_void_p), ("ld", C.c_longlong), ("u", C.c_void_p),
                ("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p), ("token", C.c_void_p),
                ("prob", C.c_void_p)]


class Grads(C.Structure):
    _fields_ = [("dw_qkv", C.c_void_p), ("db_qkv", C.c_void_p), ("dw_o", C.c_void_p), ("db_o", C.c_void_p),
                ("dw_1", C.c_void_p), ("db_1", C.c_void_p), ("dw_2", C.c_void_p), ("db_2", C.c_void_p),
                ("ld_dwqkv", C.c_longlong), ("ld_dwo", C.c_longlong), ("ld_dw1", C.c_longlong),
                ("ld_dw2", C.c_longlong)]


_lib = None


def load() -> C.CDLL:
    """Load the built library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_11641_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, ci, ll, sz = C.c_void_p, C.c_int, C.c_longlong, C.c_size_t
    lib.ecospa_create.argtypes = [C.POINTER(vp), vp]
    lib.ecospa_create.restype = ci
    lib.ecospa_destroy.argtypes = [vp]
    lib.ecospa_destroy.restype = None
    lib.ecospa_set_workspace.argtypes = [vp, vp, sz]
    lib.ecospa_set_workspace.restype = ci
    lib.ecospa_status_string.argtypes = [ci]
    lib.ecospa_status_string.restype = C.c_char_p
    lib.ecospa_last_error.argtypes = [vp]
    lib.ecospa_last_error.restype = C.c_char_p
    lib.ecospa_score_workspace_bytes.argtypes = [C.POINTER(Pair), ci]
    lib.ecospa_score_workspace_bytes.restype = sz
    lib.ecospa_coupled_score.argtypes = [vp, C.POINTER(Pair), ci, C.POINTER(vp)]
    lib.ecospa_coupled_score.restype = ci
    lib.ecospa_select_topk.argtypes = [vp, vp, ci, ci, ci, vp]
    lib.ecospa_select_topk.restype = ci
    lib.ecospa_pair_fisher.argtypes = [vp, C.POINTER(Pair), ci, C.c_float, C.POINTER(vp)]
    lib.ecospa_pair_fisher.restype = ci
    lib.ecospa_select_theta.argtypes = [vp, vp, ci, ci, C.c_float, vp, vp]
    lib.ecospa_select_theta.restype = ci
    lib.ecospa_select_pairs.argtypes = [vp, vp, ci, ci, vp]
    lib.ecospa_select_pairs.restype = ci
    for f in (lib.ecospa_compact, lib.ecospa_scatter):
        f.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ll, ll, ll, vp]
        f.restype = ci
    lib.ecospa_select_topk_batch.argtypes = [vp, C.POINTER(SelectItem), ci]
    lib.ecospa_select_topk_batch.restype = ci
    lib.ecospa_compact_batch.argtypes = [vp, C.POINTER(MapItem), ci]
    lib.ecospa_compact_batch.restype = ci
    lib.ecospa_compact_batch_rope.argtypes = [vp, C.POINTER(MapItem), ci, C.POINTER(RopeItem)]
    lib.ecospa_compact_batch_rope.restype = ci
    lib.ecospa_rope_table.argtypes = [vp, vp, ci, ci, ci, ci, ci, C.c_double, vp, vp]
    lib.ecospa_rope_table.restype = ci
    lib.ecospa_rope_table_ragged.argtypes = [vp, vp, ci, vp, ci, ci, ci, ci, C.c_double, vp, vp]
    lib.ecospa_rope_table_ragged.restype = ci
    lib.ecospa_transpose_batch.argtypes = [vp, C.POINTER(TransposeItem), ci]
    lib.ecospa_transpose_batch.restype = ci
    lib.ecospa_adamw.argtypes = [vp, C.POINTER(AdamwItem), ci, C.POINTER(AdamwHyper)]
    lib.ecospa_adamw.restype = ci
    lib.ecospa_block_workspace_bytes.argtypes = [C.POINTER(BlockDesc)]
    lib.ecospa_block_workspace_bytes.restype = sz
    lib.ecospa_coupled_fwd.argtypes = [vp, C.POINTER(BlockDesc), vp, vp, C.POINTER(Saved)]
    lib.ecospa_coupled_fwd.restype = ci
    lib.ecospa_coupled_bwd.argtypes = [vp, C.POINTER(BlockDesc), vp, vp, C.POINTER(Saved), vp, C.POINTER(Grads)]
    lib.ecospa_coupled_bwd.restype = ci
    lib.ecospa_profile_gemm.argtypes = [vp, ci]
    lib.ecospa_profile_gemm.restype = ci
    lib.ecospa_profile_gemm_read.argtypes = [vp, C.POINTER(ci), C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.ecospa_profile_gemm_read.restype = ci
    lib.ecospa_contract.argtypes = [vp, ci, ci, ci, ci, vp, ll, ci, vp, ll, ci, vp, ll, vp, ci, ci]
    lib.ecospa_contract.restype = ci
    lib.ecospa_check_indices.argtypes = [vp, vp, ci, ci, ci, vp, ci]
    lib.ecospa_check_indices.restype = ci
    lib.ecospa_contract_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    lib.ecospa_contract_workspace_bytes.restype = sz
    lib.ecospa_score_select.argtypes = [vp, C.POINTER(Pair), ci, C.POINTER(vp), C.POINTER(ci), C.POINTER(vp)]
    lib.ecospa_score_select.restype = ci
    lib.ecospa_coupled_score_static.argtypes = [vp, C.POINTER(Pair), ci, C.POINTER(vp)]
    lib.ecospa_coupled_score_static.restype = ci
    lib.ecospa_coupled_score_static_max_bytes.argtypes = []
    lib.ecospa_coupled_score_static_max_bytes.restype = sz
    lib.ecospa_contract_colsum.argtypes = [vp, ci, ci, ci, vp, ll, vp, ll, vp, ll, vp, ci, ci]
    lib.ecospa_contract_colsum.restype = ci
    lib.ecospa_mfma_probe.argtypes = [vp, vp, vp, ci, C.POINTER(C.c_double)]
    lib.ecospa_mfma_probe.restype = ci
    lib.ecospa_hbm_probe.argtypes = [vp, vp, vp, sz, ci]
    lib.ecospa_norm_fwd.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, C.c_float, vp, vp]
    lib.ecospa_norm_fwd.restype = ci
    lib.ecospa_norm_bwd.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.ecospa_norm_bwd.restype = ci
    lib.ecospa_norm_bwd_workspace_bytes.argtypes = [ci, ci]
    lib.ecospa_norm_bwd_workspace_bytes.restype = sz
    lib.ecospa_embed_fwd.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, ci, vp]
    lib.ecospa_embed_fwd.restype = ci
    lib.ecospa_embed_bwd.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, ci]
    lib.ecospa_embed_bwd.restype = ci
    lib.ecospa_xent.argtypes = [vp, ci, ci, ci, vp, ll, vp, vp, ll, vp, vp]
    lib.ecospa_xent.restype = ci
    lib.ecospa_hbm_probe.restype = ci
    lib.ecospa_cache_append.argtypes = [vp, C.POINTER(Cache), ci, vp, ll, vp, vp, vp, ci, vp, ll, vp]
    lib.ecospa_cache_append.restype = ci
    lib.ecospa_prefix_attn.argtypes = [vp, C.POINTER(Cache), ci, vp, ll, vp, ll, vp, vp, vp]
    lib.ecospa_prefix_attn.restype = ci
    lib.ecospa_prefix_attn_workspace_bytes.argtypes = [C.POINTER(Cache), ci, ci]
    lib.ecospa_prefix_attn_workspace_bytes.restype = sz
    lib.ecospa_cache_evict.argtypes = [vp, C.POINTER(Cache), vp, ci, ci, C.POINTER(Cache), vp, vp, vp]
    lib.ecospa_cache_evict.restype = ci
    lib.ecospa_logits_process.argtypes = [vp, C.POINTER(Logits)]
    lib.ecospa_logits_process.restype = ci
    lib.ecospa_logits_workspace_bytes.argtypes = [ci, ci]
    lib.ecospa_logits_workspace_bytes.restype = sz
    lib.ecospa_quant_rows.argtypes = [vp, ci, ci, ci, vp, ll, vp, ll, vp]
    lib.ecospa_quant_rows.restype = ci
    lib.ecospa_contract_quant.argtypes = [vp, ci, ci, ci, vp, ll, vp, vp, ll, vp, vp, ci, vp, ll]
    lib.ecospa_contract_quant.restype = ci
    lib.ecospa_quant_cache_append.argtypes = [vp, C.POINTER(QuantCacheDesc), ci, vp, ll, vp, vp, vp, ci, vp, ll]
    lib.ecospa_quant_cache_append.restype = ci
    lib.ecospa_quant_cache_attn.argtypes = [vp, C.POINTER(QuantCacheDesc), ci, vp, ll, vp, ll, vp, vp, ll, vp]
    lib.ecospa_quant_cache_attn.restype = ci
    lib.ecospa_quant_cache_attn_workspace_bytes.argtypes = [C.POINTER(QuantCacheDesc), ci]
    lib.ecospa_quant_cache_attn_workspace_bytes.restype = sz
    lib.ecospa_sample.argtypes = [vp, C.POINTER(SampleArgs)]
    lib.ecospa_sample.restype = ci
    lib.ecospa_sample_workspace_bytes.argtypes = [ci, ci]
    lib.ecospa_sample_workspace_bytes.restype = sz
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().ecospa_status_string(int(code)).decode()


def dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return F32
    if t == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dense(t: Optional[torch.Tensor], dtype: torch.dtype, n: int) -> Optional[int]:
    """Address of a contiguous tensor of n elements of this type (None: no tensor)."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"expected a contiguous {dtype} tensor of {n} elements, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def round_up(x: int, m: int) -> int:
    return (x + m - 1) // m * m


class KvCache:
    """A batch's own key/value caches on compact heads, with the prefix that its requests share (ecospa_cache).

    k: [B, h_kv, cap, kp_qk], v: [B, h_kv, cap, kp_vo] (bf16, last dim dense, other strides free); lens: int32 [B], own keys of every
    request; h query heads; scale: the softmax scale; pk: [h_kv, P, kp_qk], pv: [h_kv, P, kp_vo] or None.  own_max (default: cap): no
    request holds more keys than this; calls are cut by it, so a bound near the real lengths saves work and keeps small caches in the
    last-level cache; it may be set between calls.  The object keeps the tensors alive;
    their contents, lens included, are read when the kernels run."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, h: int, scale: float, pk: Optional[torch.Tensor] = None,
                 pv: Optional[torch.Tensor] = None, own_max: Optional[int] = None):
        (Bsz, h_kv, cap, kq), (k_sb, k_sh, k_st, k_unit) = k.shape, k.stride()
        (vB, vh, vcap, kv), (v_sb, v_sh, v_st, v_unit) = v.shape, v.stride()
        assert (vB, vh, vcap) == (Bsz, h_kv, cap) and v.dtype == k.dtype and k_unit == 1 and v_unit == 1 and (pk is None) == (pv is None)
        self.k, self.v, self.lens, self.pk, self.pv = k, v, lens, pk, pv
        self.B, self.h, self.h_kv, self.cap, self.kq, self.kv, self.scale = Bsz, h, h_kv, cap, kq, kv, scale
        self.nq, self.no, self.nqkv, self.n_weights = h * kq, h * kv, (h + h_kv) * kq + h_kv * kv, Bsz * h_kv * cap
        P, prefix = 0, (None, None, 0, 0, 0, 0)
        if pk is not None:
            P = pk.shape[1]
            assert pk.shape == (h_kv, P, kq) and pv.shape == (h_kv, P, kv) and pk.dtype == k.dtype and pv.dtype == k.dtype
            assert pk.stride(2) == 1 and pv.stride(2) == 1
            if P:
                prefix = (pk.data_ptr(), pv.data_ptr(), pk.stride(0), pk.stride(1), pv.stride(0), pv.stride(1))
        self.desc = Cache(dtype_code(k.dtype), Bsz, h, h_kv, kq, kv, cap, cap if own_max is None else own_max, P, scale, k.data_ptr(), v.data_ptr(),
                          k_sb, k_sh, k_st, v_sb, v_sh, v_st, *prefix, _dense(lens, torch.int32, Bsz))
        self._ref = C.byref(self.desc)
        self._need = {}

    @property
    def own_max(self) -> int:
        return self.desc.own_max

    @own_max.setter
    def own_max(self, n: int):
        self.desc.own_max = n

    def workspace_bytes(self, L: int, weights: bool) -> int:
        key = (L, weights, self.desc.own_max)
        if key not in self._need:
            self._need[key] = load().ecospa_prefix_attn_workspace_bytes(self._ref, L, int(weights))
        return self._need[key]


class QuantCache:
    """A batch's own key/value caches in 8-bit floats on compact heads (ecospa_quant_cache).

    k: [B, h_kv, cap, kp_qk], v: [B, h_kv, cap, kp_vo] (float8_e4m3fn, last dim dense, other strides free, multiples of 16); k_scale, v_scale: float32
    [B, h_kv, ceil(cap / block)], dense; lens: int32 [B]; h query heads; scale: the softmax scale; block: rows that share a scale; own_max as
    :class:`KvCache`'s.  The object keeps the tensors alive; their contents are read when the kernels run."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, lens: torch.Tensor, h: int, scale: float,
                 block: int, own_max: Optional[int] = None):
        (Bsz, h_kv, cap, kq), (k_sb, k_sh, k_st, k_unit) = k.shape, k.stride()
        (vB, vh, vcap, kv), (v_sb, v_sh, v_st, v_unit) = v.shape, v.stride()
        f8 = torch.float8_e4m3fn
        if (vB, vh, vcap) != (Bsz, h_kv, cap) or k.dtype != f8 or v.dtype != f8 or k_unit != 1 or v_unit != 1 or block < 1:
            raise ValueError(f"expected {f8} caches of equal length, got {k.dtype} {tuple(k.shape)} and {v.dtype} {tuple(v.shape)}, block {block}")
        self.k, self.v, self.k_scale, self.v_scale, self.lens = k, v, k_scale, v_scale, lens
        self.B, self.h, self.h_kv, self.cap, self.kq, self.kv, self.scale, self.block = Bsz, h, h_kv, cap, kq, kv, scale, block
        self.nq, self.no, self.nqkv = h * kq, h * kv, (h + h_kv) * kq + h_kv * kv
        n = Bsz * h_kv * ((cap + block - 1) // block)
        self.desc = QuantCacheDesc(Bsz, h, h_kv, kq, kv, cap, cap if own_max is None else own_max, block, scale, k.data_ptr(), v.data_ptr(), k_sb, k_sh, k_st,
                                   v_sb, v_sh, v_st, _dense(k_scale, torch.float32, n), _dense(v_scale, torch.float32, n), _dense(lens, torch.int32, Bsz))
        self._ref = C.byref(self.desc)
        self._need = {}

    own_max = KvCache.own_max

    def workspace_bytes(self, L: int) -> int:
        key = (L, self.desc.own_max)
        if key not in self._need:
            self._need[key] = load().ecospa_quant_cache_attn_workspace_bytes(self._ref, L)
        return self._need[key]


class Context:
    """One ecospa_ctx on the current torch stream, with a torch-owned workspace that grows on demand."""

    def __init__(self, device: str = "cuda:0", stream: Optional[torch.cuda.Stream] = None):
        self.lib = load()
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = C.c_void_p()
        rc = self.lib.ecospa_create(C.byref(h), C.c_void_p(self.stream.cuda_stream))
        if rc:
            raise EcospaError(rc, "ecospa_create")
        self.h = h
        self._ws: Optional[torch.Tensor] = None
        self._logits_need: dict = {}      # workspace of a (B, V)
        self._sample_need: dict = {}

    def __del__(self):
        try:
            if getattr(self, "h", None):
                self.lib.ecospa_destroy(self.h)
                self.h = None
        except Exception:
            pass

    def _check(self, rc: int, where: str):
        if rc:
            raise EcospaError(rc, where, self.lib.ecospa_last_error(self.h).decode())

    def reserve(self, nbytes: int):
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=self.device)
            self._check(self.lib.ecospa_set_workspace(self.h, self._ws.data_ptr(), self._ws.numel()),
                        "ecospa_set_workspace")

    def ecospa_profile_gemm(self, enable: bool):
        self._check(self.lib.ecospa_profile_gemm(self.h, int(enable)), "ecospa_profile_gemm")

    def ecospa_profile_gemm_read(self):
        n, ms, fl = C.c_int(), C.c_double(), C.c_double()
        self._check(self.lib.ecospa_profile_gemm_read(self.h, C.byref(n), C.byref(ms), C.byref(fl)),
                    "ecospa_profile_gemm_read")
        return n.value, ms.value, fl.value

    def ecospa_hbm_probe(self, src: torch.Tensor, dst: torch.Tensor, copy: bool):
        """Measurement aid: read src once (copy=False; dst is a small sink) or copy it to dst."""
        nbytes = src.numel() * src.element_size()
        self._check(self.lib.ecospa_hbm_probe(self.h, src.data_ptr(), dst.data_ptr(), nbytes, int(copy)), "ecospa_hbm_probe")

    def ecospa_mfma_probe(self, src: torch.Tensor, sink: torch.Tensor, iters: int) -> float:
        """Measurement aid: launch the pure-MFMA loop on operand bits from src (>= 64 KiB); returns the flops of the launch."""
        assert src.numel() * src.element_size() >= 65536 and sink.dtype == torch.float32 and sink.numel() >= 65536
        fl = C.c_double()
        self._check(self.lib.ecospa_mfma_probe(self.h, src.data_ptr(), sink.data_ptr(), int(iters), C.byref(fl)), "ecospa_mfma_probe")
        return fl.value

    def ecospa_contract(self, A: torch.Tensor, trans_a: bool, Bm: torch.Tensor, trans_b: bool,
                        bias: Optional[torch.Tensor] = None, tile: int = 0, splits: int = 0,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """C[m,n] = sum_k A(m,k) B(n,k) (+ bias[n]); a transposed operand is stored [K, M] / [K, N]."""
        K, M = (A.shape if trans_a else A.shape[::-1])
        K2, N = (Bm.shape if trans_b else Bm.shape[::-1])
        assert K == K2
        if out is None:
            out = torch.empty((M, N), dtype=A.dtype, device=A.device)
        self.reserve(self.lib.ecospa_contract_workspace_bytes(dtype_code(A.dtype), M, N, K, splits))     # fp32 partials of a split contraction
        self._check(self.lib.ecospa_contract(self.h, dtype_code(A.dtype), M, N, K, A.data_ptr(), A.stride(0),
                                             int(trans_a), Bm.data_ptr(), Bm.stride(0), int(trans_b), out.data_ptr(),
                                             out.stride(0), _ptr(bias), tile, splits), "ecospa_contract")
        return out

    def ecospa_contract_colsum(self, A: torch.Tensor, Bm: torch.Tensor, tile: int = 0, splits: int = 0):
        """dY^T X form: A[K, M], Bm[K, N] (bf16) -> (C[M, N] bf16, colsum[M] fp32 = column sums of A)."""
        K, M = A.shape
        K2, N = Bm.shape
        assert K == K2 and A.dtype == torch.bfloat16
        out = torch.empty((M, N), dtype=A.dtype, device=A.device)
        cs = torch.empty((M,), dtype=torch.float32, device=A.device)
        sp = max(splits, 1) if splits else 8
        rows = sp * ((N + 127) // 128)          # at most one row of partial sums per split and 128-wide tile column
        self.reserve(round_up(rows * M * 4, 256) + self.lib.ecospa_contract_workspace_bytes(BF16, M, N, K, splits) + 256)
        self._check(self.lib.ecospa_contract_colsum(self.h, M, N, K, A.data_ptr(), A.stride(0), Bm.data_ptr(), Bm.stride(0),
                                                    out.data_ptr(), out.stride(0), cs.data_ptr(), tile, splits),
                    "ecospa_contract_colsum")
        return out, cs

    # ---- step 1 ------------------------------------------------------------------------------
    @staticmethod
    def make_pair(kind: int, w1: torch.Tensor, w2: torch.Tensor, groups: int, n: int, unit: int = 1,
                  w1b: Optional[torch.Tensor] = None, rep1: int = 1, rep2: int = 1, w2_rows: bool = False) -> Pair:
        """rep1 / rep2: heads of the first / second member that share one group's inner dimensions (Eq. 5).
        w2_rows: the second member of a VO / FFN pair is stored with its units as rows ([units, d])."""
        d1 = w1.shape[1]
        d2 = w2.shape[1] if (kind == PAIR_QK or w2_rows) else w2.shape[0]
        return Pair(kind, dtype_code(w1.dtype), groups, n, unit, d1, d2, _ptr(w1), _ptr(w1b), _ptr(w2),
                    w1.stride(0), 0 if w1b is None else w1b.stride(0), w2.stride(0), rep1, rep2, int(w2_rows))

    def ecospa_coupled_score(self, pairs: Sequence[Pair], out: Optional[Sequence[torch.Tensor]] = None) -> list[torch.Tensor]:
        """Scores of a batch of pairs, one float32 tensor [groups, n/unit] per pair (written into `out` if given)."""
        arr = pairs if isinstance(pairs, C.Array) else (Pair * len(pairs))(*pairs)
        need = self.lib.ecospa_score_workspace_bytes(arr, len(arr))
        self.reserve(need)
        if out is None:
            out = [torch.empty((p.groups, p.n // max(p.unit, 1)), dtype=torch.float32, device=self.device) for p in arr]
        ptrs = (C.c_void_p * len(arr))(*[o.data_ptr() for o in out])
        self._check(self.lib.ecospa_coupled_score(self.h, arr, len(arr), ptrs), "ecospa_coupled_score")
        return list(out)

    def ecospa_score_select(self, pairs: Sequence[Pair], k: Sequence[int], scores: Optional[Sequence[torch.Tensor]] = None,
                            idx: Optional[Sequence[torch.Tensor]] = None):
        """Steps 1 and 2 of a batch of pairs in two launches: (scores, idx) with scores[p] float32 [groups, n/unit] and
        idx[p] int32 [groups, k[p]] (written into the given tensors if any)."""
        arr = pairs if isinstance(pairs, C.Array) else (Pair * len(pairs))(*pairs)
        self.reserve(self.lib.ecospa_score_workspace_bytes(arr, len(arr)))
        if scores is None:
            scores = [torch.empty((p.groups, p.n // max(p.unit, 1)), dtype=torch.float32, device=self.device) for p in arr]
        if idx is None:
            idx = [torch.empty((p.groups, int(kk)), dtype=torch.int32, device=self.device) for p, kk in zip(arr, k)]
        sp = (C.c_void_p * len(arr))(*[o.data_ptr() for o in scores])
        ip = (C.c_void_p * len(arr))(*[o.data_ptr() for o in idx])
        ka = (C.c_int * len(arr))(*[int(kk) for kk in k])
        self._check(self.lib.ecospa_score_select(self.h, arr, len(arr), sp, ka, ip), "ecospa_score_select")
        return list(scores), list(idx)

    def ecospa_coupled_score_static(self, pairs: Sequence[Pair], out: Sequence[torch.Tensor]) -> list[torch.Tensor]:
        """ecospa_coupled_score for callers that cannot allocate: the caller brings the score tensors, the partial sums
        live in the library's own fixed device array (nothing is reserved or allocated here)."""
        arr = pairs if isinstance(pairs, C.Array) else (Pair * len(pairs))(*pairs)
        ptrs = (C.c_void_p * len(arr))(*[o.data_ptr() for o in out])
        self._check(self.lib.ecospa_coupled_score_static(self.h, arr, len(arr), ptrs), "ecospa_coupled_score_static")
        return list(out)

    def ecospa_pair_fisher(self, grads: Sequence[Pair], n_samples: float,
                           out: Optional[Sequence[torch.Tensor]] = None) -> list[torch.Tensor]:
        """Eq. 8 importance of each coupled pair from its gradient matrices (described like the weights): one
        float32 tensor [groups] per pair (written into `out` if given)."""
        arr = grads if isinstance(grads, C.Array) else (Pair * len(grads))(*grads)
        self.reserve(self.lib.ecospa_score_workspace_bytes(arr, len(arr)))
        if out is None:
            out = [torch.empty((p.groups,), dtype=torch.float32, device=self.device) for p in arr]
        ptrs = (C.c_void_p * len(arr))(*[o.data_ptr() for o in out])
        self._check(self.lib.ecospa_pair_fisher(self.h, arr, len(arr), float(n_samples), ptrs), "ecospa_pair_fisher")
        return list(out)

    def ecospa_select_theta(self, scores: torch.Tensor, theta: float):
        """Alg. 1's cumulative-threshold rule per row of scores[groups, n_units]: (idx[groups, n_units] int32 padded
        with -1, k[groups] int32)."""
        assert scores.dtype == torch.float32 and scores.dim() == 2 and scores.is_contiguous()
        groups, n = scores.shape
        idx = torch.empty((groups, n), dtype=torch.int32, device=scores.device)
        k = torch.empty((groups,), dtype=torch.int32, device=scores.device)
        self._check(self.lib.ecospa_select_theta(self.h, scores.data_ptr(), groups, n, float(theta), idx.data_ptr(),
                                                 k.data_ptr()), "ecospa_select_theta")
        return idx, k

    def ecospa_select_pairs(self, fisher: torch.Tensor, n_select: int) -> torch.Tensor:
        """Alg. 1's choice among the pairs: ascending indices (int32[n_select]) of the n_select smallest
        importance values of fisher[n_pairs]."""
        assert fisher.dtype == torch.float32 and fisher.dim() == 1 and fisher.is_contiguous()
        chosen = torch.empty((max(n_select, 1),), dtype=torch.int32, device=fisher.device)
        self._check(self.lib.ecospa_select_pairs(self.h, fisher.data_ptr(), fisher.numel(), n_select,
                                                 chosen.data_ptr()), "ecospa_select_pairs")
        return chosen[:n_select]

    # ---- step 2 ------------------------------------------------------------------------------
    def ecospa_select_topk(self, scores: torch.Tensor, k: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        groups, n_units = scores.shape
        assert scores.dtype == torch.float32 and scores.is_contiguous()
        idx = out if out is not None else torch.empty((groups, max(k, 0)), dtype=torch.int32, device=self.device)
        self._check(self.lib.ecospa_select_topk(self.h, scores.data_ptr(), groups, n_units, k, idx.data_ptr()),
                    "ecospa_select_topk")
        return idx

    def ecospa_select_topk_batch(self, items: Sequence[SelectItem]):
        """items: SelectItem structs (see :meth:`select_item`); one launch for all of them."""
        arr = items if isinstance(items, C.Array) else (SelectItem * len(items))(*items)
        self._check(self.lib.ecospa_select_topk_batch(self.h, arr, len(items)), "ecospa_select_topk_batch")

    @staticmethod
    def select_item(scores: torch.Tensor, k: int, idx: torch.Tensor) -> SelectItem:
        groups, n_units = scores.shape
        assert scores.dtype == torch.float32 and scores.is_contiguous() and idx.dtype == torch.int32
        return SelectItem(scores.data_ptr(), groups, n_units, k, idx.data_ptr())

    def ecospa_check_indices(self, idx: torch.Tensor, n_units: int, k_group: Optional[torch.Tensor] = None) -> bool:
        """Debugging aid (waits for the stream): True if every list idx[g, :k] (k = idx.shape[1], or k_group[g]) is
        strictly ascending with entries in [0, n_units)."""
        assert idx.dtype == torch.int32 and idx.dim() == 2 and idx.is_contiguous()
        self.reserve(256)
        rc = self.lib.ecospa_check_indices(self.h, idx.data_ptr(), idx.shape[0], idx.shape[1], idx.shape[1], _ptr(k_group),
                                           n_units)
        if rc == ERR_INDEX:
            return False
        self._check(rc, "ecospa_check_indices")
        return True

    # ---- step 3 ------------------------------------------------------------------------------
    @staticmethod
    def map_item(src: torch.Tensor, dst: torch.Tensor, idx: torch.Tensor, axis: int, groups: int, n: int,
                 unit: int = 1, kp: Optional[int] = None, scatter: int = 0,
                 k_group: Optional[torch.Tensor] = None, idx_div: int = 1,
                 dst_t: Optional[torch.Tensor] = None, src_b: Optional[torch.Tensor] = None) -> MapItem:
        """Descriptor of one gather (scatter = 0), scatter with zero fill (1) or scatter that leaves the pruned
        slots of dst untouched (2) for :meth:`ecospa_compact_batch`.  With k_group (int32[groups]
        on the device) group g keeps its first k_group[g] entries of idx[g, :] and kp must be given.  dst_t (row gathers
        only): the transposed copy of dst, [other, slots], written by the same launch.  src_b (row gathers only): a
        second source like src; dst then takes the kept rows of both, interleaved (row 2s from src, 2s + 1 from src_b)."""
        assert src_b is None or (src_b.shape == src.shape and src_b.stride(0) == src.stride(0) and src_b.dtype == src.dtype)
        if k_group is not None:
            assert kp is not None and k_group.dtype == torch.int32 and k_group.numel() == groups // idx_div
            assert idx.dtype == torch.int32 and idx.dim() == 2 and idx.is_contiguous() and idx.shape[0] == groups // idx_div
        k = idx.shape[1] if k_group is None else 0
        kp = k if kp is None else kp
        if src.dim() == 1:
            other, ld_s, ld_d, axis = 1, src.numel(), dst.numel(), 1
        else:
            other = src.shape[1] if axis == 0 else src.shape[0]
            ld_s, ld_d = src.stride(0), dst.stride(0)
        return MapItem(src.data_ptr(), dst.data_ptr(), dtype_code(src.dtype), axis, groups, n, unit, k, kp,
                       int(scatter), other, ld_s, ld_d, idx.data_ptr(), _ptr(k_group),
                       idx.shape[1] if k_group is not None else 0, idx_div,
                       _ptr(dst_t), 0 if dst_t is None else dst_t.stride(0), _ptr(src_b))

    def ecospa_compact_ragged(self, src: torch.Tensor, idx: torch.Tensor, k_group: torch.Tensor, axis: int, groups: int,
                              n: int, kp: int, unit: int = 1, scatter: int = 0,
                              out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Gather (or scatter: 1 zero fill, 2 into the contents of `out`) with ragged kept counts, all groups padded
        to kp slots."""
        slots = groups * n if scatter else groups * kp * unit
        if out is None:
            shape = (slots,) if src.dim() == 1 else ((slots, src.shape[1]) if axis == 0 else (src.shape[0], slots))
            out = torch.empty(shape, dtype=src.dtype, device=src.device)
        self.ecospa_compact_batch([self.map_item(src, out, idx, axis, groups, n, unit, kp, scatter, k_group)])
        return out

    def ecospa_compact_batch(self, items: Sequence[MapItem], rope: Optional[RopeItem] = None):
        """All gathers / scatters of `items` in one launch; with `rope` (see :meth:`rope_item`) the same launch also
        fills the cos/sin tables of the kept rotary blocks."""
        arr = items if isinstance(items, C.Array) else (MapItem * len(items))(*items)
        if rope is None:
            self._check(self.lib.ecospa_compact_batch(self.h, arr, len(items)), "ecospa_compact_batch")
        else:
            self._check(self.lib.ecospa_compact_batch_rope(self.h, arr, len(items), C.byref(rope)), "ecospa_compact_batch_rope")

    @staticmethod
    def rope_item(idx: Optional[torch.Tensor], h: int, L: int, k: int, kp: int, d_h: int, base: float, cos: torch.Tensor,
                  sin: torch.Tensor, k_group: Optional[torch.Tensor] = None) -> RopeItem:
        """Descriptor of the cos/sin tables [h, L, kp] of the kept rotary blocks for :meth:`ecospa_compact_batch`: as
        :meth:`ecospa_rope_table` (k blocks per head) or, with k_group, as :meth:`ecospa_rope_table_ragged`."""
        assert cos.shape == (h, L, kp) and sin.shape == (h, L, kp) and cos.dtype == torch.float32 and sin.dtype == torch.float32
        ld_idx = 0 if idx is None else idx.shape[1]
        return RopeItem(_ptr(idx), _ptr(k_group), h, L, 0 if k_group is not None else k, kp, d_h, ld_idx, float(base),
                        cos.data_ptr(), sin.data_ptr())

    def _mapped(self, fn, name, src, dst, axis, groups, n, unit, k, kp, idx):
        if src.dim() == 1:
            other, ld_s, ld_d = 1, src.numel(), dst.numel()
            axis = 1
        else:
            other = src.shape[1] if axis == 0 else src.shape[0]
            ld_s, ld_d = src.stride(0), dst.stride(0)
        self._check(fn(self.h, src.data_ptr(), dst.data_ptr(), dtype_code(src.dtype), axis, groups, n, unit, k, kp,
                       other, ld_s, ld_d, idx.data_ptr()), name)
        return dst

    def ecospa_compact(self, src: torch.Tensor, idx: torch.Tensor, axis: int, groups: int, n: int, unit: int = 1,
                       kp: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        k = idx.shape[1]
        kp = k if kp is None else kp
        slots = groups * kp * unit
        if out is None:
            shape = (slots,) if src.dim() == 1 else ((slots, src.shape[1]) if axis == 0 else (src.shape[0], slots))
            out = torch.empty(shape, dtype=src.dtype, device=src.device)
        return self._mapped(self.lib.ecospa_compact, "ecospa_compact", src, out, axis, groups, n, unit, k, kp, idx)

    def ecospa_scatter(self, src: torch.Tensor, idx: torch.Tensor, axis: int, groups: int, n: int, unit: int = 1,
                       kp: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        k = idx.shape[1]
        kp = k if kp is None else kp
        slots = groups * n
        if out is None:
            shape = (slots,) if src.dim() == 1 else ((slots, src.shape[1]) if axis == 0 else (src.shape[0], slots))
            out = torch.empty(shape, dtype=src.dtype, device=src.device)
        return self._mapped(self.lib.ecospa_scatter, "ecospa_scatter", src, out, axis, groups, n, unit, k, kp, idx)

    def ecospa_rope_table(self, idx: Optional[torch.Tensor], h: int, L: int, k: int, kp: int, d_h: int,
                          base: float = 10000.0, out=None):
        if out is not None:
            cos, sin = out
            assert cos.shape == (h, L, kp) and sin.shape == (h, L, kp) and cos.dtype == torch.float32
        else:
            cos = torch.empty((h, L, kp), dtype=torch.float32, device=self.device)
            sin = torch.empty_like(cos)
        self._check(self.lib.ecospa_rope_table(self.h, _ptr(idx), h, L, k, kp, d_h, float(base), cos.data_ptr(),
                                               sin.data_ptr()), "ecospa_rope_table")
        return cos, sin

    def ecospa_rope_table_ragged(self, idx: torch.Tensor, k_group: torch.Tensor, L: int, kp: int, d_h: int,
                                 base: float = 10000.0, out=None):
        h = idx.shape[0]
        assert idx.dtype == torch.int32 and idx.is_contiguous() and k_group.dtype == torch.int32 and k_group.numel() == h
        if out is not None:
            cos, sin = out
            assert cos.shape == (h, L, kp) and sin.shape == (h, L, kp) and cos.dtype == torch.float32
        else:
            cos = torch.empty((h, L, kp), dtype=torch.float32, device=self.device)
            sin = torch.empty_like(cos)
        self._check(self.lib.ecospa_rope_table_ragged(self.h, idx.data_ptr(), idx.shape[1], k_group.data_ptr(), h, L, kp,
                                                      d_h, float(base), cos.data_ptr(), sin.data_ptr()),
                    "ecospa_rope_table_ragged")
        return cos, sin

    @staticmethod
    def transpose_item(src: torch.Tensor, dst: torch.Tensor) -> TransposeItem:
        assert src.dim() == 2 and dst.shape == (src.shape[1], src.shape[0]) and src.dtype == dst.dtype
        return TransposeItem(src.data_ptr(), dst.data_ptr(), dtype_code(src.dtype), src.shape[0], src.shape[1],
                             src.stride(0), dst.stride(0))

    def ecospa_transpose_batch(self, items: Sequence[TransposeItem]):
        """dst = src^T for every item, one launch (see :meth:`transpose_item`)."""
        arr = items if isinstance(items, C.Array) else (TransposeItem * len(items))(*items)
        self._check(self.lib.ecospa_transpose_batch(self.h, arr, len(arr)), "ecospa_transpose_batch")

    # ---- layer glue ----------------------------------------------------------------------------
    def ecospa_norm_fwd(self, kind: int, x: torch.Tensor, gain: torch.Tensor, bias: Optional[torch.Tensor], eps: float,
                        y: torch.Tensor, res: Optional[torch.Tensor] = None, x_out: Optional[torch.Tensor] = None,
                        stat: Optional[torch.Tensor] = None):
        """y = norm(x + res); x + res -> x_out; the row statistics -> stat (float32 [T] for RMS, [T, 2] for LayerNorm).
        All [T, d] tensors contiguous bf16."""
        T, d = x.shape
        assert all(t is None or (t.is_contiguous() and t.shape == x.shape) for t in (x, y, res, x_out))
        self._check(self.lib.ecospa_norm_fwd(self.h, kind, T, d, dtype_code(x.dtype), x.data_ptr(), _ptr(res), _ptr(x_out),
                                             gain.data_ptr(), _ptr(bias), float(eps), y.data_ptr(), _ptr(stat)), "ecospa_norm_fwd")
        return y

    def ecospa_norm_bwd(self, kind: int, x: torch.Tensor, gain: torch.Tensor, stat: torch.Tensor, dy: torch.Tensor,
                        dx: torch.Tensor, dgain: torch.Tensor, dbias: Optional[torch.Tensor] = None,
                        dres: Optional[torch.Tensor] = None):
        """dx = dres + the gradient of the normalisation; dgain (and dbias) = the parameter gradients."""
        T, d = x.shape
        assert all(t is None or (t.is_contiguous() and t.shape == x.shape) for t in (x, dy, dx, dres))
        self.reserve(self.lib.ecospa_norm_bwd_workspace_bytes(T, d))
        self._check(self.lib.ecospa_norm_bwd(self.h, kind, T, d, dtype_code(x.dtype), x.data_ptr(), gain.data_ptr(), stat.data_ptr(),
                                             dy.data_ptr(), _ptr(dres), dx.data_ptr(), dgain.data_ptr(), _ptr(dbias)), "ecospa_norm_bwd")
        return dx

    def ecospa_embed_fwd(self, ids: torch.Tensor, table: torch.Tensor, out: torch.Tensor, pos: Optional[torch.Tensor] = None):
        """out[t] = table[ids[t]] (+ pos[t mod L]); ids int64."""
        assert ids.dtype == torch.int64 and ids.is_contiguous() and table.is_contiguous() and out.is_contiguous()
        T, (V, d) = ids.numel(), table.shape
        self._check(self.lib.ecospa_embed_fwd(self.h, T, d, V, dtype_code(table.dtype), ids.data_ptr(), table.data_ptr(), _ptr(pos),
                                              0 if pos is None else pos.shape[0], out.data_ptr()), "ecospa_embed_fwd")
        return out

    def ecospa_embed_bwd(self, ids: torch.Tensor, dx: torch.Tensor, dtable: torch.Tensor, dpos: Optional[torch.Tensor] = None):
        """dtable[v] = sum of dx[t] over ids[t] == v (the whole table is written); dpos[l] = sum over the sequences."""
        assert ids.dtype == torch.int64 and ids.is_contiguous() and dx.is_contiguous() and dtable.is_contiguous()
        T, (V, d) = ids.numel(), dtable.shape
        self._check(self.lib.ecospa_embed_bwd(self.h, T, d, V, dtype_code(dx.dtype), ids.data_ptr(), dx.data_ptr(), dtable.data_ptr(),
                                              _ptr(dpos), 0 if dpos is None else dpos.shape[0]), "ecospa_embed_bwd")

    def ecospa_xent(self, logits: torch.Tensor, targets: torch.Tensor, row_loss: torch.Tensor, loss: torch.Tensor,
                    dlogits: Optional[torch.Tensor] = None):
        """Mean cross-entropy of the rows of logits [T, V] (bf16, row stride free) against int64 targets: the row losses,
        the mean (a device float) and dlogits of the mean (may be logits itself)."""
        assert targets.dtype == torch.int64 and targets.is_contiguous() and logits.stride(1) == 1
        assert row_loss.dtype == torch.float32 and loss.dtype == torch.float32
        T, V = logits.shape
        self._check(self.lib.ecospa_xent(self.h, T, V, dtype_code(logits.dtype), logits.data_ptr(), logits.stride(0), targets.data_ptr(),
                                         _ptr(dlogits), 0 if dlogits is None else dlogits.stride(0), row_loss.data_ptr(),
                                         loss.data_ptr()), "ecospa_xent")
        return loss

    # ---- serving -------------------------------------------------------------------------------
    @staticmethod
    def _rows(x: torch.Tensor, width: int):
        """(rows, leading dimension) of a bf16 matrix of at least `width` columns."""
        (T, w), (ld, unit) = x.shape, x.stride()
        if w < width or unit != 1 or x.dtype != torch.bfloat16:
            raise ValueError(f"expected bf16 rows of {width} elements, got {x.dtype} {tuple(x.shape)}")
        return T, ld

    def ecospa_cache_append(self, cache: KvCache, qkv: torch.Tensor, pos: Optional[torch.Tensor] = None, rope=None,
                            q: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None):
        """The L = rows / B new tokens of every request (rows of the projection: Q | K | V columns) become the last L rows of its cache;
        cache.lens counts them already.  rope: (cos, sin) [h_kv, L_tab, kp_qk / 2] turns queries (into q) and keys by the angles of
        positions pos[b] + t; weights [B, h_kv, cap]: the new rows' accumulated weights are set to zero."""
        T, ld = self._rows(qkv, cache.nqkv)
        Tq, ldq = (T, 0) if q is None else self._rows(q, cache.nq)
        if T % cache.B or Tq != T:
            raise ValueError(f"{T} rows (queries {Tq}) for {cache.B} requests")
        cos_ptr = sin_ptr = None
        tab = 0
        if rope is not None:
            cos, sin = rope
            tab = cos.shape[1]
            n = cache.h_kv * tab * (cache.kq // 2)
            cos_ptr, sin_ptr = _dense(cos, torch.float32, n), _dense(sin, torch.float32, n)
        self._check(self.lib.ecospa_cache_append(self.h, cache._ref, T // cache.B, qkv.data_ptr(), ld, _dense(pos, torch.int32, cache.B), cos_ptr,
                                                 sin_ptr, tab, _ptr(q), ldq, _dense(weights, torch.float32, cache.n_weights)), "ecospa_cache_append")

    def ecospa_prefix_attn(self, cache: KvCache, q: torch.Tensor, o: torch.Tensor, lse: Optional[torch.Tensor] = None,
                           weights: Optional[torch.Tensor] = None, weights_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """o [B*L, h * kp_vo] = attention of the new tokens' queries q [B*L, h * kp_qk] over the shared prefix and the own caches; lse
        float32 [B, h, L]; weights_out [B, h_kv, cap] = weights (None: zeros) + what every own key received."""
        T, ldq = self._rows(q, cache.nq)
        To, ldo = self._rows(o, cache.no)
        L = T // cache.B
        if T % cache.B or To != T:
            raise ValueError(f"{T} rows (outputs {To}) for {cache.B} requests")
        self.reserve(cache.workspace_bytes(L, weights_out is not None))
        f32 = torch.float32
        self._check(self.lib.ecospa_prefix_attn(self.h, cache._ref, L, q.data_ptr(), ldq, o.data_ptr(), ldo, _dense(lse, f32, T * cache.h),
                                                _dense(weights, f32, cache.n_weights), _dense(weights_out, f32, cache.n_weights)), "ecospa_prefix_attn")
        return o

    def ecospa_cache_evict(self, cache: KvCache, weights: torch.Tensor, keep: int, recent: int, k_out: torch.Tensor, v_out: torch.Tensor,
                           lens_out: torch.Tensor, weights_out: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None):
        """The last `recent` rows of every cache and, of the others, those with the largest weights, `keep` in all, gathered in order into
        k_out, v_out [B, h_kv, cap_out, kp]; lens_out int32 [B]; weights_out float32 [B, h_kv, cap_out]; idx int32 [B, h_kv, keep]."""
        dst = KvCache(k_out, v_out, lens_out, cache.h, cache.scale)
        if (dst.B, dst.h_kv, dst.kq, dst.kv) != (cache.B, cache.h_kv, cache.kq, cache.kv) or lens_out.data_ptr() == cache.lens.data_ptr():
            raise ValueError("the new cache differs in requests, heads or widths, or shares its lengths with the old one")
        if idx is None:
            self.reserve(cache.B * cache.h_kv * max(keep, 0) * 4)
        f32 = torch.float32
        self._check(self.lib.ecospa_cache_evict(self.h, cache._ref, _dense(weights, f32, cache.n_weights), keep, recent, dst._ref, dst.desc.lens,
                                                _dense(weights_out, f32, dst.n_weights), _dense(idx, torch.int32, cache.B * cache.h_kv * keep)),
                    "ecospa_cache_evict")

    def ecospa_logits_process(self, logits: torch.Tensor, out: Optional[torch.Tensor] = None, history: Optional[torch.Tensor] = None,
                              history_len: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                              frequency: Optional[torch.Tensor] = None, presence: Optional[torch.Tensor] = None,
                              temperature: Optional[torch.Tensor] = None, bias_ids: Optional[torch.Tensor] = None,
                              bias: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                              mask_row: Optional[torch.Tensor] = None, pick: Optional[torch.Tensor] = None,
                              lse: Optional[torch.Tensor] = None):
        """Penalties for the tokens of history [B, H] (int32), biases (ids and values [B, n]), temperature and masks (words [n_masks,
        ceil(V / 32)], int32; mask_row int32 [B], -1: none) on logits [B, V] -> (pick int32 [B], lse float32 [B]); the processed logits go
        to `out` (may be logits itself; None: not wanted).  Parameters: float32 [B]."""
        (Bsz, V), (ld, unit) = logits.shape, logits.stride()
        f32, i32 = torch.float32, torch.int32
        ld_out = out_dtype = n_bias = H = n_masks = ld_mask = 0
        bias_ptr = ids_ptr = mask_ptr = hist_ptr = out_ptr = None
        assert unit == 1
        if out is not None:
            (ld_out, unit), out_dtype, out_ptr = out.stride(), dtype_code(out.dtype), out.data_ptr()
            assert unit == 1 and out.shape == logits.shape
        if history is not None:
            H = history.shape[1]
            hist_ptr = _dense(history, i32, Bsz * H)
        if bias is not None:
            n_bias = bias.shape[1]
            bias_ptr, ids_ptr = _dense(bias, f32, Bsz * n_bias), _dense(bias_ids, i32, Bsz * n_bias)
        if mask is not None:
            (ld_mask, unit), n_masks, mask_ptr = mask.stride(), mask.shape[0], mask.data_ptr()
            assert unit == 1 and mask.dtype == i32 and mask_row is not None
        pick = torch.empty(Bsz, dtype=i32, device=logits.device) if pick is None else pick
        lse = torch.empty(Bsz, dtype=f32, device=logits.device) if lse is None else lse
        need = self._logits_need.get((Bsz, V))
        if need is None:
            need = self._logits_need[Bsz, V] = self.lib.ecospa_logits_workspace_bytes(Bsz, V)
        self.reserve(need)
        a = Logits(Bsz, V, dtype_code(logits.dtype), out_dtype, logits.data_ptr(), out_ptr, ld, ld_out, hist_ptr, _dense(history_len, i32, Bsz), H,
                   n_bias, _dense(repetition, f32, Bsz), _dense(frequency, f32, Bsz), _dense(presence, f32, Bsz), _dense(temperature, f32, Bsz),
                   ids_ptr, bias_ptr, mask_ptr, _dense(mask_row, i32, Bsz), ld_mask, n_masks, _dense(pick, i32, Bsz), _dense(lse, f32, Bsz))
        self._check(self.lib.ecospa_logits_process(self.h, C.byref(a)), "ecospa_logits_process")
        return pick, lse

    def ecospa_sample(self, logits: torch.Tensor, u: torch.Tensor, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
                      top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None,
                      prob: Optional[torch.Tensor] = None) -> torch.Tensor:
        """A token int32 [B] for every row of logits [B, V], drawn by u float32 [B] in [0, 1) from what temperature, top_k (int32), top_p and min_p
        leave (each [B] or None); prob float32 [B]: its probability there.  No token to draw: -1."""
        (Bsz, V), (ld, unit) = logits.shape, logits.stride()
        f32, i32 = torch.float32, torch.int32
        if unit != 1:
            raise ValueError(f"expected dense rows of logits, got strides {logits.stride()}")
        token = torch.empty(Bsz, dtype=i32, device=logits.device) if token is None else token
        need = self._sample_need.get((Bsz, V))
        if need is None:
            need = self._sample_need[Bsz, V] = self.lib.ecospa_sample_workspace_bytes(Bsz, V)
        self.reserve(need)
        a = SampleArgs(Bsz, V, dtype_code(logits.dtype), logits.data_ptr(), ld, _dense(u, f32, Bsz), _dense(temperature, f32, Bsz), _dense(top_k, i32, Bsz),
                       _dense(top_p, f32, Bsz), _dense(min_p, f32, Bsz), _dense(token, i32, Bsz), _dense(prob, f32, Bsz))
        self._check(self.lib.ecospa_sample(self.h, C.byref(a)), "ecospa_sample")
        return token

    # ---- caches in 8-bit floats ------------------------------------------------------------------
    def ecospa_quant_cache_append(self, cache: QuantCache, qkv: torch.Tensor, pos: Optional[torch.Tensor] = None, rope=None,
                                  q: Optional[torch.Tensor] = None):
        """:meth:`ecospa_cache_append` into caches of 8-bit floats: the new tokens become the last L rows, block scales rise where they have to."""
        T, ld = self._rows(qkv, cache.nqkv)
        Tq, ldq = (T, 0) if q is None else self._rows(q, cache.nq)
        if T % cache.B or Tq != T:
            raise ValueError(f"{T} rows (queries {Tq}) for {cache.B} requests")
        cos_ptr = sin_ptr = None
        tab = 0
        if rope is not None:
            cos, sin = rope
            tab = cos.shape[1]
            n = cache.h_kv * tab * (cache.kq // 2)
            cos_ptr, sin_ptr = _dense(cos, torch.float32, n), _dense(sin, torch.float32, n)
        self._check(self.lib.ecospa_quant_cache_append(self.h, cache._ref, T // cache.B, qkv.data_ptr(), ld, _dense(pos, torch.int32, cache.B), cos_ptr,
                                                       sin_ptr, tab, _ptr(q), ldq), "ecospa_quant_cache_append")

    def ecospa_quant_cache_attn(self, cache: QuantCache, q: torch.Tensor, o: torch.Tensor, lse: Optional[torch.Tensor] = None,
                                o_in: Optional[torch.Tensor] = None, lse_in: Optional[torch.Tensor] = None) -> torch.Tensor:
        """o [B*L, h * kp_vo] = attention of the new tokens' queries q [B*L, h * kp_qk] over the own caches; o_in (as o) and lse_in float32
        [B, h, L]: the result over other keys, joined in; lse float32 [B, h, L]: over all of them."""
        T, ldq = self._rows(q, cache.nq)
        To, ldo = self._rows(o, cache.no)
        Ti, ldi = (T, 0) if o_in is None else self._rows(o_in, cache.no)
        L = T // cache.B
        if T % cache.B or To != T or Ti != T:
            raise ValueError(f"{T} rows (outputs {To}, {Ti}) for {cache.B} requests")
        self.reserve(cache.workspace_bytes(L))
        n = T * cache.h
        self._check(self.lib.ecospa_quant_cache_attn(self.h, cache._ref, L, q.data_ptr(), ldq, _ptr(o_in), ldi, _dense(lse_in, torch.float32, n), o.data_ptr(),
                                                     ldo, _dense(lse, torch.float32, n)), "ecospa_quant_cache_attn")
        return o

    # ---- products in 8-bit integers --------------------------------------------------------------
    def ecospa_quant_rows(self, x: torch.Tensor, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
        """(q int8 [rows, cols], scale float32 [rows]) with x[r] ~ scale[r] * q[r]; x: [rows, cols] float32 or bf16, row stride free."""
        (rows, cols), (ld, unit) = x.shape, x.stride()
        if q is None:
            q = torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format) if cols % 16 == 0 else x.new_empty((rows, round_up(cols, 16)), dtype=torch.int8)[:, :cols]
        elif q.dtype != torch.int8 or q.shape != x.shape or q.stride(1) != 1:
            raise ValueError(f"expected int8 codes {tuple(x.shape)}, got {q.dtype} {tuple(q.shape)} {q.stride()}")
        if unit != 1:
            raise ValueError(f"expected rows of {cols} dense elements, got strides {x.stride()}")
        if scale is None:
            scale = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=x.device)
            at_scale = scale.data_ptr()
        else:
            at_scale = _dense(scale, torch.float32, rows)
        rc = self.lib.ecospa_quant_rows(self.h, rows, cols, dtype_code(x.dtype), x.data_ptr(), ld, q.data_ptr(), q.stride(0), at_scale)
        if rc:
            self._check(rc, "ecospa_quant_rows")
        return q, scale

    def ecospa_contract_quant(self, A: torch.Tensor, sa: torch.Tensor, Bm: torch.Tensor, sb: torch.Tensor, bias: Optional[torch.Tensor] = None,
                           act: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """act(sa[m] sb[n] sum_k A[m, k] B[n, k] + bias[n]) in bf16 [M, N] (SwiGLU: [M, N / 2]); A [M, K], Bm [N, K] int8 as
        :meth:`ecospa_quant_rows` leaves them."""
        (M, K), (lda, ua), (N, Kb), (ldb, ub) = A.shape, A.stride(), Bm.shape, Bm.stride()
        act = ACT_NONE if act is None else act
        width = N // 2 if act == ACT_SWIGLU else N
        out = torch.empty((M, width), dtype=torch.bfloat16, device=A.device) if out is None else out
        if A.dtype != torch.int8 or Bm.dtype != torch.int8 or Kb != K or ua != 1 or ub != 1:
            raise ValueError(f"expected int8 rows of equal length, got {A.dtype} {tuple(A.shape)} and {Bm.dtype} {tuple(Bm.shape)}")
        ldc, uc = out.stride()
        if out.dtype != torch.bfloat16 or out.shape != (M, width) or uc != 1:
            raise ValueError(f"expected a bf16 output [{M}, {width}], got {out.dtype} {tuple(out.shape)}")
        rc = self.lib.ecospa_contract_quant(self.h, M, N, K, A.data_ptr(), lda, _dense(sa, torch.float32, M), Bm.data_ptr(), ldb, _dense(sb, torch.float32, N),
                                            _dense(bias, torch.bfloat16, N), act, out.data_ptr(), ldc)
        if rc:
            self._check(rc, "ecospa_contract_quant")
        return out

    # ---- parameter update ----------------------------------------------------------------------
    @staticmethod
    def adamw_item(w: torch.Tensor, g: torch.Tensor, m: torch.Tensor, v: torch.Tensor,
                   w_lp: Optional[torch.Tensor] = None) -> AdamwItem:
        """Descriptor of one tensor for :meth:`ecospa_adamw` (all contiguous, same element count)."""
        n = w.numel()
        assert all(t.is_contiguous() and t.numel() == n for t in (w, g, m, v)) and m.dtype == v.dtype
        assert w_lp is None or (w_lp.is_contiguous() and w_lp.numel() == n and w_lp.dtype == torch.bfloat16)
        return AdamwItem(w.data_ptr(), _ptr(w_lp), g.data_ptr(), m.data_ptr(), v.data_ptr(), n, dtype_code(w.dtype),
                         dtype_code(g.dtype), dtype_code(m.dtype))

    def ecospa_adamw(self, items: Sequence[AdamwItem], step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
                     eps: float = 1e-8, weight_decay: float = 0.01):
        """One fused AdamW step over all tensors in `items` (one launch)."""
        arr = items if isinstance(items, C.Array) else (AdamwItem * len(items))(*items)
        hp = AdamwHyper(lr, beta1, beta2, eps, weight_decay, step)
        self._check(self.lib.ecospa_adamw(self.h, arr, len(arr), C.byref(hp)), "ecospa_adamw")

    # ---- steps 4-5 ---------------------------------------------------------------------------
    def ecospa_coupled_fwd(self, desc: BlockDesc, x: torch.Tensor, y: torch.Tensor, saved: Optional[Saved]):
        self.reserve(self.lib.ecospa_block_workspace_bytes(C.byref(desc)))
        self._check(self.lib.ecospa_coupled_fwd(self.h, C.byref(desc), x.data_ptr(), y.data_ptr(),
                                                None if saved is None else C.byref(saved)), "ecospa_coupled_fwd")
        return y

    def ecospa_coupled_bwd(self, desc: BlockDesc, x: torch.Tensor, dy: torch.Tensor, saved: Saved,
                           dx: Optional[torch.Tensor], grads: Grads):
        self.reserve(self.lib.ecospa_block_workspace_bytes(C.byref(desc)))
        self._check(self.lib.ecospa_coupled_bwd(self.h, C.byref(desc), x.data_ptr(), dy.data_ptr(), C.byref(saved),
                                                _ptr(dx), C.byref(grads)), "ecospa_coupled_bwd")
        return dx
