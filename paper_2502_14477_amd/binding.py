"""Python binding over libesa.so: argument marshalling only.

Every function has the name and meaning of its C entry point (include/esa.h).  Tensors are
torch CUDA tensors (torch provides device memory and the current stream, nothing else); a
leading batch dimension is optional.  The marshalling itself (sizes and strides, output and workspace
allocation, the call) is native code, csrc/binding.cpp: a step is a few tens of microseconds of kernels, and host
time per call is part of what it takes.  The C entry points remain reachable as `lib.esa_*` (ctypes).
Nothing in this module computes: with the library missing, import fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Tuple

import torch

ESA_F32, ESA_BF16, ESA_E4M3 = 0, 1, 2
ESA_W_ROWMAJOR, ESA_W_PACKED = 0, 1
ESA_PAIRS_HALVES, ESA_PAIRS_NEIGHBOURS = 0, 1
ESA_SCALE_NONE, ESA_SCALE_LINEAR, ESA_SCALE_NTK, ESA_SCALE_YARN = 0, 1, 2, 3
_PKG = os.path.dirname(os.path.abspath(__file__))


class EsaError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("libesa error %d: %s" % (code, text))
        self.code = code


class PagedCache(ctypes.Structure):
    """esa_paged_cache of include/esa_paged.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("tok_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("h_kv", ctypes.c_int), ("d", ctypes.c_int), ("dtype", ctypes.c_int)]


class PagedBatch(ctypes.Structure):
    """esa_paged_batch of include/esa_paged.h."""
    _fields_ = [("cu", ctypes.c_void_p), ("start", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("pages_ld", ctypes.c_int64),
                ("n_tok", ctypes.c_int64), ("n_seq", ctypes.c_int), ("max_pages", ctypes.c_int)]


class RopeRows(ctypes.Structure):
    """esa_rope_rows of include/esa_serve.h."""
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("x_tok", ctypes.c_int64), ("x_head", ctypes.c_int64),
                ("out_tok", ctypes.c_int64), ("out_head", ctypes.c_int64), ("heads", ctypes.c_int)]


class PageState(ctypes.Structure):
    """esa_page_state of include/esa_serve.h."""
    _fields_ = [("start_in", ctypes.c_void_p), ("held_in", ctypes.c_void_p), ("ring_at_in", ctypes.c_void_p), ("start", ctypes.c_void_p),
                ("held", ctypes.c_void_p), ("ring_at", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("pages_ld", ctypes.c_int64),
                ("ring", ctypes.c_void_p), ("n_seq", ctypes.c_int), ("max_pages", ctypes.c_int), ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int)]


def lib_path() -> str:
    return os.path.join(_PKG, "libesa.so")


def _load() -> ctypes.CDLL:
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(
            "%s is missing: build it with `python -m paper_2502_14477_amd.build` "
            "(there is no fallback path)" % path)
    L = ctypes.CDLL(path)
    i32, i64, vp, sz, f32 = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
    L.esa_version.restype = i32
    L.esa_version.argtypes = []
    L.esa_last_error.restype = ctypes.c_char_p
    L.esa_last_error.argtypes = []
    L.esa_segments.restype = i32
    L.esa_segments.argtypes = [i64, i64, i64, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.esa_compress.restype = i32
    L.esa_pack_weights.restype = i32
    L.esa_pack_weights.argtypes = [vp, i64, i32, i32, vp, vp]
    L.esa_compress.argtypes = [vp, i64, i64, i64, vp, i32, vp, i32, vp, i64, i32, i32, i64, i64, vp]
    L.esa_compress_qk.restype = i32
    L.esa_compress_qk.argtypes = [vp, i64, i64, vp, vp, vp, i64, i64, i64, vp, i64, i64, vp, vp, vp, i64, i64, i64,
                                  i64, i32, i32, i32, i32, vp]
    L.esa_score_workspace_bytes.restype = sz
    L.esa_score_workspace_bytes.argtypes = [i32, i64, i32, i32]
    L.esa_score.restype = i32
    L.esa_score.argtypes = [vp, i32, vp, i64, i64, i32, i32, vp, i32, i32, i64, i64, i64, vp, sz, vp]
    L.esa_select_topk_workspace_bytes.restype = sz
    L.esa_select_topk_workspace_bytes.argtypes = [i64, i32, i32]
    L.esa_select_topk.restype = i32
    L.esa_select_topk.argtypes = [vp, i64, i32, i64, vp, i32, i64, i64, vp, sz, vp]
    L.esa_score_select_gather_workspace_bytes.restype = sz
    L.esa_score_select_gather_workspace_bytes.argtypes = [i32, i64, i32, i32, i32]
    L.esa_score_select_gather.restype = i32
    L.esa_score_select_gather.argtypes = [vp, i32, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, i64, i32, i32, vp, vp, i32, i32,
                                          i64, i64, i64, i64, i64, i64, vp, sz, vp]
    L.esa_select_topk_static_capacity.restype = sz
    L.esa_select_topk_static_capacity.argtypes = []
    L.esa_select_topk_static_prepare.restype = i32
    L.esa_select_topk_static_prepare.argtypes = []
    L.esa_select_topk_static.restype = i32
    L.esa_select_topk_static.argtypes = [vp, i64, i32, i64, vp, i32, i64, i64, vp]
    L.esa_gather_kv.restype = i32
    L.esa_gather_kv.argtypes = [vp, vp, i64, vp, i32, i32, i32, vp, vp, i32, i32, i64, i64, i64, vp]
    L.esa_attend_workspace_bytes.restype = sz
    L.esa_attend_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
    L.esa_attend.restype = i32
    L.esa_attend.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i64, i64, i64, vp, vp, i32, f32, vp, vp,
                             i32, i32, i64, i64, i64, i64, vp, sz, vp]
    L.esa_attend_indexed_workspace_bytes.restype = sz
    L.esa_attend_indexed_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, i32]
    L.esa_attend_indexed.restype = i32
    L.esa_attend_indexed.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i64, i64, i64, vp, i32, i64, f32, vp, vp,
                                     i32, i32, i64, i64, i64, vp, sz, vp]
    L.esa_attend_finish.restype = i32
    L.esa_attend_finish.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i64, i64, i64, vp, vp, i32, f32, i32, vp, vp,
                                    i32, i32, i64, i64, i64, i64, vp, sz, vp]
    L.esa_attend_local.restype = i32
    L.esa_attend_local.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i64, i64, i64, f32, i32, i32, i32, i64, i64,
                                   vp, sz, vp]
    f64 = ctypes.c_double
    L.esa_rope.restype = i32
    L.esa_rope.argtypes = [vp, i64, i32, i32, i64, f64, f64, f64, vp, i64, i32, i32, i64, i64, vp]
    L.esa_attend_reencoded_workspace_bytes.restype = sz
    L.esa_attend_reencoded_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, i64]
    L.esa_attend_reencoded.restype = i32
    L.esa_attend_reencoded.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i64, i64, i64, vp, vp, i32, f32, f64, f64,
                                       vp, vp, i32, i32, i64, i64, i64, i64, vp, sz, vp]
    batch, cache = ctypes.POINTER(PagedBatch), ctypes.POINTER(PagedCache)
    L.esa_append_paged.restype = i32
    L.esa_append_paged.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, i64, batch, cache, f64, i32, vp]
    L.esa_attend_paged_workspace_bytes.restype = sz
    L.esa_attend_paged_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32]
    L.esa_attend_paged.restype = i32
    L.esa_attend_paged.argtypes = [vp, i64, i32, batch, cache, i64, i64, vp, i32, i64, f32, f32, vp, i64, vp, i32, vp, sz, vp]
    L.esa_rope_frequencies.restype = i32
    L.esa_rope_frequencies.argtypes = [f64, i32, i32, f64, f64, f64, f64, ctypes.POINTER(f64)]
    L.esa_rope_at.restype = i32
    L.esa_rope_at.argtypes = [ctypes.POINTER(RopeRows), i32, vp, i64, i32, i32, vp, i32, f64, i32, i32, vp]
    L.esa_plan_paged_workspace_bytes.restype = sz
    L.esa_plan_paged_workspace_bytes.argtypes = [ctypes.POINTER(PageState)]
    L.esa_plan_paged.restype = i32
    L.esa_plan_paged.argtypes = [ctypes.POINTER(PageState), vp, vp, i64, vp, vp, vp, vp, vp, sz, vp]
    L.esa_verify_drafts_workspace_bytes.restype = sz
    L.esa_verify_drafts_workspace_bytes.argtypes = [i32, i64]
    L.esa_verify_drafts.restype = i32
    L.esa_verify_drafts.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, i32, i64, vp, vp, i32, vp, sz, vp]
    return L


lib = _load()
from . import _native  # noqa: E402  (links against the library loaded above)

EXPORTS = ("esa_version", "esa_last_error", "esa_segments", "esa_pack_weights", "esa_compress", "esa_score_workspace_bytes",
           "esa_score", "esa_select_topk_workspace_bytes", "esa_select_topk", "esa_gather_kv",
           "esa_attend_workspace_bytes", "esa_attend", "esa_attend_local", "esa_attend_finish",
           "esa_attend_indexed_workspace_bytes", "esa_attend_indexed", "esa_rope",
           "esa_attend_reencoded_workspace_bytes", "esa_attend_reencoded", "esa_compress_qk",
           "esa_select_topk_static_capacity", "esa_select_topk_static_prepare", "esa_select_topk_static",
           "esa_score_select_gather_workspace_bytes", "esa_score_select_gather")
PAGED_EXPORTS = ("esa_append_paged", "esa_attend_paged_workspace_bytes", "esa_attend_paged")      # include/esa_paged.h
SERVE_EXPORTS = ("esa_rope_frequencies", "esa_rope_at", "esa_plan_paged_workspace_bytes", "esa_plan_paged",
                 "esa_verify_drafts_workspace_bytes", "esa_verify_drafts")      # include/esa_serve.h


_native.set_error_class(EsaError)


def _check(code: int) -> None:
    if code != 0:
        raise EsaError(code, lib.esa_last_error().decode())


def esa_version() -> int:
    return lib.esa_version()


def esa_segments(t0: int, l_i: int, l_l: int) -> Tuple[int, int]:
    return _native.segments(t0, l_i, l_l)


class PackedWeights:
    """Compression weights in the packed layout [d_c, d_in] (see esa_pack_weights)."""

    def __init__(self, data: torch.Tensor, d_in: int, d_c: int):
        self.data, self.d_in, self.d_c = data, d_in, d_c


def esa_pack_weights(W: torch.Tensor) -> PackedWeights:
    """W [d_in, d_c] -> packed weights; done once per layer."""
    d_in, d_c = W.shape
    assert W.is_contiguous()
    dtype = {torch.float32: ESA_F32, torch.bfloat16: ESA_BF16}.get(W.dtype)
    if dtype is None:
        raise EsaError(-2, "unsupported torch dtype %s" % W.dtype)
    out = torch.empty((d_c, d_in), dtype=W.dtype, device=W.device)
    _check(lib.esa_pack_weights(W.data_ptr(), d_in, d_c, dtype, out.data_ptr(), torch.cuda.current_stream().cuda_stream))
    return PackedWeights(out, d_in, d_c)


def esa_compress(x: torch.Tensor, W, bias: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [B?, n_tok, heads, d] or [B?, n_tok, d_in] -> [B?, n_tok, d_c].  W is a [d_in, d_c] tensor or
    PackedWeights.  `out` may be a row-strided view (e.g. rows t0.. of the compressed-key cache)."""
    if isinstance(W, PackedWeights):
        return _native.compress(x, W.data, ESA_W_PACKED, W.d_in, W.d_c, bias, out)
    d_in, d_c = W.shape
    return _native.compress(x, W, ESA_W_ROWMAJOR, d_in, d_c, bias, out)


def esa_compress_qk(xq: torch.Tensor, Wq, xk: torch.Tensor, Wk, bias_q: Optional[torch.Tensor] = None,
                    bias_k: Optional[torch.Tensor] = None, out_q: Optional[torch.Tensor] = None,
                    out_k: Optional[torch.Tensor] = None):
    """Both compressions of Eq. 5 in one call (shapes per tensor as esa_compress; `out_k` is typically the rows
    t0.. of the compressed-key cache).  Returns (q', k')."""
    if isinstance(Wq, PackedWeights):
        assert isinstance(Wk, PackedWeights), "both weight matrices in the same layout"
        assert Wq.d_c == Wk.d_c
        return _native.compress_qk(xq, Wq.data, Wq.d_in, xk, Wk.data, Wk.d_in, ESA_W_PACKED, Wq.d_c, bias_q, bias_k, out_q, out_k)
    assert not isinstance(Wk, PackedWeights), "both weight matrices in the same layout"
    (dq, dc), (dk, dck) = Wq.shape, Wk.shape
    assert dc == dck
    return _native.compress_qk(xq, Wq, dq, xk, Wk, dk, ESA_W_ROWMAJOR, dc, bias_q, bias_k, out_q, out_k)


def esa_score(qc: torch.Tensor, kc_cache: torch.Tensor, m_lo: int, m_hi: int, eps: int = 0,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """qc [B?, l_c, d_c], kc_cache [B?, S, d_c] -> score [B?, m_hi-m_lo] fp32."""
    return _native.score(qc, kc_cache, m_lo, m_hi, eps, out)


def esa_select_topk(score: torch.Tensor, k: int, base: int = 0) -> torch.Tensor:
    """score [B?, n] fp32 -> idx [B?, min(k, n)] int32, ascending absolute positions."""
    return _native.select_topk(score, k, base)


def esa_score_select_gather(qc: torch.Tensor, kc_cache: torch.Tensor, m_lo: int, m_hi: int, k: int,
                            k_cache: Optional[torch.Tensor] = None, v_cache: Optional[torch.Tensor] = None, eps: int = 0):
    """esa_score + esa_select_topk (+ esa_gather_kv when the caches are given) in one call.
    Returns (score or None, idx, k_sel, v_sel); k_sel / v_sel are None without caches."""
    return _native.score_select_gather(qc, kc_cache, m_lo, m_hi, k, k_cache, v_cache, eps)


def esa_select_topk_static_capacity() -> int:
    return lib.esa_select_topk_static_capacity()


def esa_select_topk_static_prepare() -> None:
    _check(lib.esa_select_topk_static_prepare())


def esa_select_topk_static(score: torch.Tensor, k: int, base: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """esa_select_topk on the library's own scratch.  With `out` given ([B?, min(k, n)] int32) this
    function allocates nothing either."""
    return _native.select_topk_static(score, k, base, out)


def esa_gather_kv(k_cache: torch.Tensor, v_cache: torch.Tensor, idx: torch.Tensor):
    """caches [B?, S, h_kv, d] (GPU memory, or pinned host memory for an offloaded cache), idx [B?, n_sel]
    int32 on the GPU -> (k_sel, v_sel) [B?, n_sel, h_kv, d] on the GPU."""
    return _native.gather_kv(k_cache, v_cache, idx)


ESA_SPLIT_I_EARLY, ESA_SPLIT_ALGORITHM1 = 0, 1


def esa_attend_indexed(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, t0: int, l_i: int, l_l: int,
                       idx: Optional[torch.Tensor], scale: Optional[float] = None, return_lse: bool = False):
    """esa_gather_kv + esa_attend in one call: idx [B?, n_sel] int32 positions of the selected tokens."""
    return _native.attend_indexed(q, k_cache, v_cache, t0, l_i, l_l, idx, scale, return_lse)


def esa_rope(x: torch.Tensor, pos0: float, pos_step: float, base: float, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotary encoding of x [B?, n_tok, heads, d]: row i goes to position pos0 + i*pos_step.  `out` may be
    x itself (in place) or a view with the same shape (e.g. rows of a cache)."""
    return _native.rope(x, pos0, pos_step, base, out)


def esa_attend_reencoded(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, t0: int, l_i: int, l_l: int,
                         k_sel: Optional[torch.Tensor], v_sel: Optional[torch.Tensor], w: float, rope_base: float,
                         scale: Optional[float] = None, return_lse: bool = False):
    """Section 3.2's attention on un-encoded q, key cache and gathered keys (shapes as esa_attend)."""
    return _native.attend_reencoded(q, k_cache, v_cache, t0, l_i, l_l, k_sel, v_sel, w, rope_base, scale, return_lse)


def esa_attend_local(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, t0: int, l_i: int, l_l: int,
                     scale: Optional[float] = None, split: int = ESA_SPLIT_I_EARLY) -> None:
    """First half of the two-call form of esa_attend: the keys that do not depend on the selection
    ([I, L, C], or [L, C] with split = ESA_SPLIT_ALGORITHM1).  Leaves partial results in a buffer that the device's
    two-call attentions share, for esa_attend_finish (same sizes and split, ordered after it, with no other
    esa_attend_local of the device between the two)."""
    _native.attend_local(q, k_cache, v_cache, t0, l_i, l_l, scale, split)


def esa_attend_finish(q, k_cache, v_cache, t0, l_i, l_l, k_sel, v_sel, scale=None, return_lse=False,
                      split: int = ESA_SPLIT_I_EARLY):
    """Second half of the two-call form: the selected keys (with the initial tokens if split =
    ESA_SPLIT_ALGORITHM1), then the merge.  Arguments as esa_attend."""
    return esa_attend(q, k_cache, v_cache, t0, l_i, l_l, k_sel, v_sel, scale, return_lse, _split=split)


def esa_attend(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, t0: int, l_i: int, l_l: int,
               k_sel: Optional[torch.Tensor], v_sel: Optional[torch.Tensor], scale: Optional[float] = None,
               return_lse: bool = False, _split: Optional[int] = None):
    """q [B?, l_c, h, d]; caches [B?, S, h_kv, d] holding the current tokens at rows t0..; gathered
    buffers [B?, n_sel, h_kv, d] -> out [B?, l_c, h, d] (and lse [B?, l_c, h] fp32)."""
    return _native.attend(q, k_cache, v_cache, t0, l_i, l_l, k_sel, v_sel, scale, return_lse, _split)


def esa_append_paged(k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, start: torch.Tensor, pages: torch.Tensor,
                     k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                     v_scale: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, rope_base: Optional[float] = None,
                     out_q: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Appends k, v [n_tok, h_kv, d] to a paged cache, keys turned to their positions (rope_base=None: as they are), and returns q
    [n_tok, h, d] turned likewise (None without q).  Rows cu[b] .. cu[b+1] are sequence b's positions start[b], start[b]+1, ...; cu [n_seq+1],
    start [n_seq] and pages [n_seq, max_pages] are int32.  Caches [n_pages, h_kv, page_size, d] in any order of strides, of k's type or
    float8_e4m3fn with scales [n_pages, h_kv] uint8 (exponents: 2^(byte - 127)).  `out_q` may be q itself.  Rows behind cu[n_seq] are left
    as they are, undefined in a new tensor."""
    return _native.append_paged(k, v, cu, start, pages, k_cache, v_cache, k_scale, v_scale, q, rope_base, out_q)


def esa_attend_paged(q: torch.Tensor, cu: torch.Tensor, start: torch.Tensor, pages: torch.Tensor, k_cache: torch.Tensor,
                     v_cache: torch.Tensor, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                     l_i: Optional[int] = None, l_l: int = 0, idx: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                     cap: float = 0.0, out: Optional[torch.Tensor] = None, return_lse: bool = False):
    """Attention of q [n_tok, h, d] over the pages of its sequences, to which the rows' keys and values have been appended (arguments as
    esa_append_paged, `start` from before it) -> out [n_tok, h, d] (and lse [n_tok, h] fp32).  l_i=None: a token sees everything up to
    itself; else the initial, the local and the selected positions idx [n_seq, n_sel] int32 (-1: none), segments as esa_segments.
    cap > 0: scores become cap * tanh(score / cap).  Rows behind cu[n_seq] are left as they are, undefined in new tensors."""
    return _native.attend_paged(q, cu, start, pages, k_cache, v_cache, k_scale, v_scale, l_i, l_l, idx, scale, cap, out, return_lse)


def esa_rope_frequencies(base: float, rot: int, scaling: int = ESA_SCALE_NONE, factor: float = 1.0, length: float = 0.0, fast: float = 32.0,
                         slow: float = 1.0, device="cuda") -> torch.Tensor:
    """Angles a position of the rot/2 pairs, float64, made once per model: base^(-2j/rot), or scaled for contexts `factor` times as long
    (ESA_SCALE_YARN: pairs that make more than `fast` turns in `length` tokens stay, those that make less than `slow` are divided)."""
    return _native.rope_frequencies(base, rot, scaling, factor, length, fast, slow).to(device)


class _Turn(torch.autograd.Function):
    """esa_rope_at where gradients are wanted: the map is linear in the rows, and the transposed call is its way back."""

    @staticmethod
    def forward(ctx, q, k, pos, freq, pairs, gain, transposed, zeros):
        ctx.save_for_backward(pos, freq)
        ctx.how = pairs, gain, transposed
        # rows of negative position have no influence: their gradients are 0
        out = [torch.zeros(x.shape, dtype=x.dtype, device=x.device) if zeros and x is not None else None for x in (q, k)]
        got = _native.rope_at(q, pos, freq, k, pairs, gain, transposed, *out)
        if k is not None:
            ctx.mark_non_differentiable(*(x for x, needed in zip(got, ctx.needs_input_grad) if not needed))
        return got

    @staticmethod
    def backward(ctx, *grads):
        pos, freq = ctx.saved_tensors
        pairs, gain, transposed = ctx.how
        wanted = [(g if g.stride(2) == 1 else g.contiguous()) if needed else None for g, needed in zip(grads, ctx.needs_input_grad)]
        rows = [g for g in wanted if g is not None]
        got = _Turn.apply(rows[0], rows[1] if len(rows) > 1 else None, pos, freq, pairs, gain, not transposed, True)
        back = iter(got if len(rows) > 1 else (got,))
        wanted = [None if g is None else next(back) for g in wanted]
        return (*wanted, *[None] * (8 - len(wanted)))


def esa_rope_at(q: torch.Tensor, pos: torch.Tensor, freq: torch.Tensor, k: Optional[torch.Tensor] = None, pairs: int = ESA_PAIRS_HALVES,
                gain: float = 1.0, transposed: bool = False, out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None):
    """Rotary encoding of q [n_tok, h, d], and k [n_tok, h_kv, d] in the same call, at positions pos [n_tok] int32 on the GPU; tokens and heads may
    lie in any order of strides.  freq: esa_rope_frequencies' or any float64 on the GPU; the first 2 * len(freq) elements of a head
    turn, the others are copied.  transposed=True takes gradients of the outputs to gradients of the inputs.  Rows of negative
    position are left as they are, undefined in a new tensor.  `out_q`, `out_k` may be q and k.  Returns q, or (q, k).  Where q or k requires a
    gradient the result has one (pos and freq have to stay as they are until then); outputs are not to be given then."""
    got = _native.rope_at(q, pos, freq, k, pairs, gain, transposed, out_q, out_k)
    return got if got is not None else _Turn.apply(q, k, pos, freq, pairs, gain, transposed, False)


class PagePlan(NamedTuple):
    """What esa_plan_paged writes: cu [n_seq + 1], start, held [n_seq], ring_at [2], pos [n_tok], lack [1] int32, slot [n_tok] int64."""
    cu: torch.Tensor
    start: torch.Tensor
    held: torch.Tensor
    ring_at: torch.Tensor
    pos: torch.Tensor
    slot: torch.Tensor
    lack: torch.Tensor

    @staticmethod
    def empty(n_seq: int, n_tok: int, device) -> "PagePlan":
        def ints(n, dtype=torch.int32):
            return torch.empty(n, dtype=dtype, device=device)
        return PagePlan(ints(n_seq + 1), ints(n_seq), ints(n_seq), ints(2), ints(n_tok), ints(n_tok, torch.int64), ints(1))


def esa_plan_paged(new: torch.Tensor, start: torch.Tensor, held: torch.Tensor, pages: torch.Tensor, ring: torch.Tensor, ring_at: torch.Tensor,
                   page_size: int, n_tok: int, grow: Optional[torch.Tensor] = None, out: Optional[PagePlan] = None) -> PagePlan:
    """Begins a step of new[b] tokens of sequence b [n_seq], which has start[b] (+ grow[b]) in the cache and holds the pages pages[b, :held[b]] of a
    pool of len(ring) pages; ring holds those that nobody holds, ring_at[1] of them from place ring_at[0] on.  Pages that are no longer needed go
    back to the ring, those that are needed come from it: pages [n_seq, max_pages] and ring are changed in place.  n_tok is the number of
    rows that there is room for.  Returns cu, start and (with pages) what esa_append_paged and esa_attend_paged take, pos as esa_rope_at
    takes it, slot = page * page_size + pos % page_size (-1: none), the next call's held and ring_at, and lack, the pages that were not to be
    had: a sequence with held[b] * page_size < start[b] + its rows repeats its step (grow[b] = 0).  A page is held once.  `out` is written into and returned; its start, held and ring_at may be the arguments of these names."""
    if out is None:
        out = PagePlan.empty(pages.shape[0], n_tok, pages.device)
    _native.plan_paged(new, start, held, pages, ring, ring_at, page_size, n_tok, grow, *out)
    return out


def esa_verify_drafts(target: torch.Tensor, tokens: torch.Tensor, cu: torch.Tensor, u: torch.Tensor, draft: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None):
    """Rows cu[b] .. cu[b+1] are sequence b's last token and the drafted ones behind it: tokens [n_tok] int32, target [n_tok, vocab] the target's
    probabilities behind each row, draft [n_tok, vocab] those that the row's token was drawn from (None: it was looked up), u [n_tok] fp32 random numbers
    (a drafted row's decides whether it stands, the first row's draws the token behind the last that stands).  Returns (out [n_tok],
    count [n_seq]) int32: the token behind each row, -1 behind the drawn one (and drawn from a row without any probability), and how many there are.  A prompt's
    tokens are no drafts: rows that are not verified are left out, by offsets of the others' own.  Rows behind cu[n_seq] are left as they are, undefined in
    a new tensor."""
    return _native.verify_drafts(target, tokens, cu, u, draft, out, count)
