"""ctypes binding of libmustdrop.so: argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

F32, BF16 = 0, 1
FILTER_BUDGET, FILTER_THRESHOLD = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
# MUSTDROP_LIBRARY selects another build of the same ABI (e.g. one compiled with different tile parameters)
_LIB_PATH = os.environ.get("MUSTDROP_LIBRARY") or os.path.join(_HERE, "libmustdrop.so")
_lib = None

EXPORTS = [
    "mustdrop_last_error", "mustdrop_version",
    "mustdrop_encode_merge_workspace_bytes", "mustdrop_encode_merge", "mustdrop_encode_merge_adaptive",
    "mustdrop_encode_merge_noalloc",
    "mustdrop_prefill_filter_workspace_bytes", "mustdrop_prefill_filter",
    "mustdrop_decode_evict_workspace_bytes", "mustdrop_decode_evict", "mustdrop_decode_append", "mustdrop_decode_keep",
    "mustdrop_prefill_filter_strided", "mustdrop_decode_evict_strided", "mustdrop_decode_append_strided",
    "mustdrop_decode_keep_strided",
    "mustdrop_cache4_bytes", "mustdrop_cache4_pages_workspace_bytes", "mustdrop_cache4_pages", "mustdrop_cache4_write",
    "mustdrop_cache4_read", "mustdrop_cache4_attend_workspace_bytes", "mustdrop_cache4_attend",
    "mustdrop_rotate", "mustdrop_cache4_append", "mustdrop_cache4_bounds", "mustdrop_cache4_choose_workspace_bytes", "mustdrop_cache4_choose",
    "mustdrop_cache4_attend_chosen_workspace_bytes", "mustdrop_cache4_attend_chosen",
    "mustdrop_profile_start", "mustdrop_profile_stop",
]


class KvLayout(C.Structure):
    """md_kv_layout: element strides of the batch, token and head axes."""
    _fields_ = [("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class Rotary(C.Structure):
    """md_rotary: how many pairs of channels turn, on how many axes, which channels a pair is, and each pair's axis."""
    _fields_ = [("pairs", C.c_int32), ("axes", C.c_int32), ("adjacent", C.c_int32), ("axis", C.c_uint8 * 128)]


class MustDropError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"mustdrop error {code}: {message}")
        self.code = code


def library_path() -> str:
    return _LIB_PATH


def library() -> C.CDLL:
    """Loads the HIP library built in-tree (python -m paper_2411_10803_amd.build).  No fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2411_10803_amd.build` "
                              "(there is no CPU fallback)")
        lib = C.CDLL(_LIB_PATH)
        lib.mustdrop_last_error.restype = C.c_char_p
        lib.mustdrop_version.restype = C.c_int
        for n in ("mustdrop_encode_merge_workspace_bytes", "mustdrop_prefill_filter_workspace_bytes",
                  "mustdrop_decode_evict_workspace_bytes", "mustdrop_cache4_bytes", "mustdrop_cache4_pages_workspace_bytes",
                  "mustdrop_cache4_attend_workspace_bytes", "mustdrop_cache4_choose_workspace_bytes",
                  "mustdrop_cache4_attend_chosen_workspace_bytes"):
            getattr(lib, n).restype = C.c_size_t
        for n in ("mustdrop_encode_merge", "mustdrop_encode_merge_adaptive", "mustdrop_encode_merge_noalloc", "mustdrop_prefill_filter", "mustdrop_decode_evict", "mustdrop_decode_append",
                  "mustdrop_decode_keep", "mustdrop_prefill_filter_strided", "mustdrop_decode_evict_strided",
                  "mustdrop_decode_append_strided", "mustdrop_decode_keep_strided", "mustdrop_cache4_pages",
                  "mustdrop_cache4_write", "mustdrop_cache4_read", "mustdrop_cache4_attend", "mustdrop_rotate", "mustdrop_cache4_append",
                  "mustdrop_cache4_bounds", "mustdrop_cache4_choose", "mustdrop_cache4_attend_chosen"):
            getattr(lib, n).restype = C.c_int
        _lib = lib
    return _lib


# Argument types of the calls, one letter each: p pointer, i int, l int64, f float, z size_t.  The conversion then
# happens inside ctypes: an object per argument made in Python cost 10 of the 20 us that the host spent on a call.
_TYPES = {"p": C.c_void_p, "i": C.c_int, "l": C.c_int64, "f": C.c_float, "z": C.c_size_t}
_ENCODE = "pippipp" + "i" * 10 + "f"
_PREFILL = "p" * 8 + "i" * 6 + "fiiff" + "i" + "p" * 10
_EVICT = "p" * 7 + "i" * 4 + "ffi" + "pp"
_APPEND = "p" * 8 + "i" * 6
_KEEP = "p" * 7 + "i" * 5 + "pp"
_SIGNATURES = {
    "mustdrop_encode_merge": _ENCODE + "i" + "p" * 9 + "pzp",
    "mustdrop_encode_merge_noalloc": _ENCODE + "i" + "p" * 9 + "p",
    "mustdrop_encode_merge_adaptive": _ENCODE + "fi" + "p" * 10 + "pzp",
    "mustdrop_prefill_filter": _PREFILL + "pzp",
    "mustdrop_prefill_filter_strided": _PREFILL + "ppp" + "pzp",
    "mustdrop_decode_evict": _EVICT + "pzp",
    "mustdrop_decode_evict_strided": _EVICT + "p" + "pzp",
    "mustdrop_decode_append": _APPEND + "p",
    "mustdrop_decode_append_strided": _APPEND + "p" + "p",
    "mustdrop_decode_keep": _KEEP + "pzp",
    "mustdrop_decode_keep_strided": _KEEP + "pl" + "pzp",
    "mustdrop_cache4_pages": "p" * 7 + "i" * 5 + "pzp",
    "mustdrop_cache4_write": "ppipp" + "i" * 6 + "pp",
    "mustdrop_cache4_read": "p" * 6 + "i" * 8 + "pp",
    "mustdrop_cache4_attend": "pi" + "p" * 5 + "i" * 8 + "f" + "p" * 4 + "pzp",
    "mustdrop_rotate": "ppi" + "p" * 4 + "i" * 7 + "pipp" + "p" * 4 + "p",
    "mustdrop_cache4_append": "pppi" + "p" * 5 + "i" * 9 + "pp" + "p" * 3 + "p",
    "mustdrop_cache4_bounds": "p" * 6 + "i" * 7 + "p",
    "mustdrop_cache4_choose": "pi" + "p" * 5 + "i" * 11 + "pp" + "pzp",
    "mustdrop_cache4_attend_chosen": "pi" + "p" * 6 + "i" * 9 + "f" + "p" * 4 + "pzp",
}
_functions: Dict[str, object] = {}


def _call(name: str, *args):
    """Calls an entry point with plain Python values and device pointers, and raises on an error code."""
    fn = _functions.get(name)
    if fn is None:
        fn = library()[name]                               # a function object of its own: library().<name> stays untyped
        fn.restype = C.c_int
        fn.argtypes = [_TYPES[t] for t in _SIGNATURES[name]]
        _functions[name] = fn
    try:
        rc = fn(*args)
    except C.ArgumentError as e:
        for t, value in zip(_SIGNATURES[name], args):
            if t != "p":
                _TYPES[t](value)                           # raises what the conversion itself raises, e.g. OverflowError
        raise TypeError(f"{name}: {e}") from None
    _check(rc)


def _check(rc: int):
    if rc != 0:
        raise MustDropError(rc, library().mustdrop_last_error().decode())


def _ptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None or isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors handed to the C ABI must be contiguous"
    return t.data_ptr()


def _view_ptr(t) -> int:
    """Device pointer of a [.., tokens, H, d] view whose last axis is contiguous (any other strides)."""
    assert t.stride(-1) == 1, "the head dimension must be contiguous"
    return t.data_ptr()


def _layout(t):
    """md_kv_layout of a [B, tokens, H, d] view (the last three axes of a [layers, B, tokens, H, d] one)."""
    st = t.stride()
    return KvLayout(st[-4], st[-3], st[-2])


def _stream(stream=None) -> int:
    import torch
    if stream is not None:
        return stream.cuda_stream
    # the handle alone; torch.cuda.current_stream() wraps it in an object first
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _workspace(nbytes: int, device):
    import torch
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def encode_workspace(B, T, Hg, Wg, Hc, kt, kh, kw, device="cuda"):
    n = library().mustdrop_encode_merge_workspace_bytes(B, T, Hg, Wg, Hc, kt, kh, kw)
    return _workspace(n, device)


def prefill_workspace(B, Mv, N, H, Rcap, device="cuda"):
    n = library().mustdrop_prefill_filter_workspace_bytes(B, Mv, N, H, Rcap)
    return _workspace(n, device)


def decode_workspace(B, Lcap, H, device="cuda"):
    n = library().mustdrop_decode_evict_workspace_bytes(B, Lcap, H)
    return _workspace(n, device)


def mustdrop_encode_merge(x, q_cls, k_cls, mass_in, valid, T, Hg, Wg, kt, kh, kw, tau, key_budget,
                          out: Optional[Dict] = None, workspace=None, stream=None, want_scores=True) -> Dict:
    """Sec. 3.3.  x [B, M, D] (f32 / bf16); q_cls [B, Hc, dc]; k_cls [B, 1+M, Hc, dc]; returns the output tensors."""
    import torch
    B, M, D = x.shape
    dev = x.device
    if key_budget > 0:
        Hc, dc = q_cls.shape[1], q_cls.shape[2]
        qk_dtype = _dtype_code(q_cls)
    else:
        Hc, dc, qk_dtype = 1, D, _dtype_code(x)
    W = -(-T // kt) * -(-Hg // kh) * -(-Wg // kw)          # border windows are clipped to the grid
    if out is None:
        out = {
            "out_x": torch.zeros_like(x),
            "out_index": torch.full((B, M), -1, dtype=torch.int32, device=dev),
            "out_mass": torch.zeros((B, M), dtype=torch.float32, device=dev),
            "out_is_key": torch.zeros((B, M), dtype=torch.uint8, device=dev),
            "out_valid": torch.zeros((B, M), dtype=torch.uint8, device=dev),
            "out_count": torch.zeros((B,), dtype=torch.int32, device=dev),
            "key_index": torch.full((B, max(key_budget, 1)), -1, dtype=torch.int32, device=dev),
            "a_cls": torch.zeros((B, M), dtype=torch.float32, device=dev) if want_scores else None,
            "window_sim": torch.zeros((B, max(W, 1)), dtype=torch.float32, device=dev) if want_scores else None,
        }
    if workspace is None:
        workspace = encode_workspace(B, T, Hg, Wg, Hc, kt, kh, kw, dev)
    out["workspace"] = workspace
    _call("mustdrop_encode_merge",
        _ptr(x), _dtype_code(x), _ptr(q_cls), _ptr(k_cls), qk_dtype, _ptr(mass_in), _ptr(valid),
        B, T, Hg, Wg, D, Hc, dc,
        kt, kh, kw, tau, key_budget,
        _ptr(out["out_x"]), _ptr(out["out_index"]), _ptr(out["out_mass"]), _ptr(out["out_is_key"]),
        _ptr(out["out_valid"]), _ptr(out["out_count"]), _ptr(out["key_index"]),
        _ptr(out.get("a_cls")), _ptr(out.get("window_sim")),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return out


def mustdrop_encode_merge_noalloc(x, q_cls, k_cls, mass_in, valid, T, Hg, Wg, kt, kh, kw, tau, key_budget, out: Dict,
                                  stream=None) -> Dict:
    """mustdrop_encode_merge on the library's static scratch buffer (no workspace argument; the call allocates
    nothing, so `out` must hold every output tensor; "a_cls" and "window_sim" may be None)."""
    B, M, D = x.shape
    if key_budget > 0:
        Hc, dc = q_cls.shape[1], q_cls.shape[2]
        qk_dtype = _dtype_code(q_cls)
    else:
        Hc, dc, qk_dtype = 1, D, _dtype_code(x)
    _call("mustdrop_encode_merge_noalloc",
        _ptr(x), _dtype_code(x), _ptr(q_cls), _ptr(k_cls), qk_dtype, _ptr(mass_in), _ptr(valid),
        B, T, Hg, Wg, D, Hc, dc,
        kt, kh, kw, tau, key_budget,
        _ptr(out["out_x"]), _ptr(out["out_index"]), _ptr(out["out_mass"]), _ptr(out["out_is_key"]),
        _ptr(out["out_valid"]), _ptr(out["out_count"]), _ptr(out["key_index"]),
        _ptr(out.get("a_cls")), _ptr(out.get("window_sim")), _stream(stream))
    return out


def mustdrop_encode_merge_adaptive(x, q_cls, k_cls, mass_in, valid, T, Hg, Wg, kt, kh, kw, tau, key_lambda, key_cap,
                                   out: Optional[Dict] = None, workspace=None, stream=None, want_scores=True) -> Dict:
    """Sec. 3.3 with Eq. 7 as printed: keys = {a_cls > mean + key_lambda * std}; key_index holds the first key_cap
    of them, key_count their number."""
    import torch
    B, M, D = x.shape
    dev = x.device
    Hc, dc = q_cls.shape[1], q_cls.shape[2]
    W = -(-T // kt) * -(-Hg // kh) * -(-Wg // kw)          # border windows are clipped to the grid
    if out is None:
        out = {
            "out_x": torch.zeros_like(x),
            "out_index": torch.full((B, M), -1, dtype=torch.int32, device=dev),
            "out_mass": torch.zeros((B, M), dtype=torch.float32, device=dev),
            "out_is_key": torch.zeros((B, M), dtype=torch.uint8, device=dev),
            "out_valid": torch.zeros((B, M), dtype=torch.uint8, device=dev),
            "out_count": torch.zeros((B,), dtype=torch.int32, device=dev),
            "key_index": torch.full((B, max(key_cap, 1)), -1, dtype=torch.int32, device=dev),
            "key_count": torch.zeros((B,), dtype=torch.int32, device=dev),
            "a_cls": torch.zeros((B, M), dtype=torch.float32, device=dev) if want_scores else None,
            "window_sim": torch.zeros((B, max(W, 1)), dtype=torch.float32, device=dev) if want_scores else None,
        }
    if workspace is None:
        workspace = encode_workspace(B, T, Hg, Wg, Hc, kt, kh, kw, dev)
    out["workspace"] = workspace
    _call("mustdrop_encode_merge_adaptive",
        _ptr(x), _dtype_code(x), _ptr(q_cls), _ptr(k_cls), _dtype_code(q_cls), _ptr(mass_in), _ptr(valid),
        B, T, Hg, Wg, D, Hc, dc,
        kt, kh, kw, tau, key_lambda, key_cap,
        _ptr(out["out_x"]), _ptr(out["out_index"]), _ptr(out["out_mass"]), _ptr(out["out_is_key"]),
        _ptr(out["out_valid"]), _ptr(out["out_count"]), _ptr(out["key_index"]), _ptr(out["key_count"]),
        _ptr(out.get("a_cls")), _ptr(out.get("window_sim")),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return out


def mustdrop_prefill_filter(q_txt, k, v, hidden, vis_valid, txt_len, is_key, Mv, softmax_scale, mode, budget,
                            gamma, alpha, Rcap=None, out: Optional[Dict] = None, workspace=None, stream=None,
                            want_scores=True, row_lse=None) -> Dict:
    """Sec. 3.4.  q_txt [B,N,H,d]; k, v [B,L,H,d]; hidden [B,L,C] (bf16); row_lse [B,H,N] f32 or None."""
    import torch
    B, N, H, d = q_txt.shape
    Cdim = hidden.shape[2]
    dev = q_txt.device
    if Rcap is None:
        Rcap = budget if mode == FILTER_BUDGET else Mv
    if out is None:
        out = {
            "hidden_out": torch.zeros((B, Rcap + N, Cdim), dtype=hidden.dtype, device=dev),
            "k_out": torch.zeros((B, Rcap + N, H, d), dtype=k.dtype, device=dev),
            "v_out": torch.zeros((B, Rcap + N, H, d), dtype=v.dtype, device=dev),
            "kept_index": torch.full((B, Rcap), -1, dtype=torch.int32, device=dev),
            "kept_count": torch.zeros((B,), dtype=torch.int32, device=dev),
            "out_len": torch.zeros((B,), dtype=torch.int32, device=dev),
            "out_protect": torch.zeros((B, Rcap + N), dtype=torch.uint8, device=dev),
            "out_ids": torch.full((B, Rcap + N), -1, dtype=torch.int32, device=dev),
            "score_global": torch.zeros((B, Mv), dtype=torch.float32, device=dev) if want_scores else None,
            "score_indiv": torch.zeros((B, Mv), dtype=torch.float32, device=dev) if want_scores else None,
        }
    if workspace is None:
        workspace = prefill_workspace(B, Mv, N, H, Rcap, dev)
    out["workspace"] = workspace
    _call("mustdrop_prefill_filter",
        _ptr(q_txt), _ptr(k), _ptr(v), _ptr(hidden), _ptr(vis_valid), _ptr(txt_len), _ptr(is_key), _ptr(row_lse),
        B, Mv, N, H, d, Cdim,
        softmax_scale, mode, budget, gamma, alpha,
        Rcap,
        _ptr(out["hidden_out"]), _ptr(out["k_out"]), _ptr(out["v_out"]),
        _ptr(out["kept_index"]), _ptr(out["kept_count"]), _ptr(out.get("out_len")), _ptr(out.get("out_protect")), _ptr(out.get("out_ids")),
        _ptr(out.get("score_global")), _ptr(out.get("score_indiv")),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return out


def mustdrop_decode_evict(q, k_cache, v_cache, acc, ids, protect, length, softmax_scale, decay, budget,
                          evicted_ids=None, evicted_count=None, workspace=None, stream=None):
    """Sec. 3.5, one decode step; the cache state is updated in place.  Returns the workspace used."""
    B, Lcap, H, d = k_cache.shape
    if workspace is None:
        workspace = decode_workspace(B, Lcap, H, k_cache.device)
    _call("mustdrop_decode_evict",
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(acc), _ptr(ids), _ptr(protect), _ptr(length),
        B, Lcap, H, d,
        softmax_scale, decay, budget,
        _ptr(evicted_ids), _ptr(evicted_count),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return workspace


def mustdrop_decode_append(k_new, v_new, k_cache, v_cache, acc, ids, protect, length, new_id, protect_new=1,
                           stream=None):
    """Eq. 3: appends one entry per sample at slot len[b] (device-side, asynchronous)."""
    B, Lcap, H, d = k_cache.shape
    _call("mustdrop_decode_append",
        _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(acc), _ptr(ids), _ptr(protect), _ptr(length),
        B, Lcap, H, d, int(new_id), int(protect_new),
        _stream(stream))


def mustdrop_decode_keep(k_caches, v_caches, keep, acc, ids, protect, length, evicted_ids=None, evicted_count=None,
                         workspace=None, stream=None):
    """Sec. 3.5, the static policy: only the entries flagged in ``keep`` stay, in the caches of all layers
    (k_caches, v_caches [n_layers,B,Lcap,H,d]); the state is updated in place.  Returns the workspace used."""
    n_layers, B, Lcap, H, d = k_caches.shape
    if workspace is None:
        workspace = decode_workspace(B, Lcap, H, k_caches.device)
    _call("mustdrop_decode_keep",
        _ptr(k_caches), _ptr(v_caches), _ptr(keep), _ptr(acc), _ptr(ids), _ptr(protect), _ptr(length),
        n_layers, B, Lcap, H, d,
        _ptr(evicted_ids), _ptr(evicted_count),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return workspace


def mustdrop_prefill_filter_strided(q_txt, k, v, hidden, vis_valid, txt_len, is_key, Mv, softmax_scale, mode, budget,
                                    gamma, alpha, out: Dict, Rcap=None, workspace=None, stream=None, row_lse=None) -> Dict:
    """Sec. 3.4 on Q / K / V in any layout: q_txt, k, v and out["k_out"], out["v_out"] are [B, tokens, H, d] VIEWS
    (e.g. a permuted head-major tensor); their strides are handed over as md_kv_layout.  k and v share one
    layout, k_out and v_out another.  `out` must hold every output tensor (see mustdrop_prefill_filter)."""
    B, N, H, d = q_txt.shape
    Cdim = hidden.shape[2]
    if Rcap is None:
        Rcap = budget if mode == FILTER_BUDGET else Mv
    assert k.stride() == v.stride() and out["k_out"].stride() == out["v_out"].stride()
    assert tuple(out["k_out"].shape) == (B, Rcap + N, H, d)
    if workspace is None:
        workspace = prefill_workspace(B, Mv, N, H, Rcap, q_txt.device)
    out["workspace"] = workspace
    lq, lkv, lo = _layout(q_txt), _layout(k), _layout(out["k_out"])
    _call("mustdrop_prefill_filter_strided",
        _view_ptr(q_txt), _view_ptr(k), _view_ptr(v), _ptr(hidden), _ptr(vis_valid), _ptr(txt_len), _ptr(is_key), _ptr(row_lse),
        B, Mv, N, H, d, Cdim,
        softmax_scale, mode, budget, gamma, alpha,
        Rcap,
        _ptr(out["hidden_out"]), _view_ptr(out["k_out"]), _view_ptr(out["v_out"]),
        _ptr(out["kept_index"]), _ptr(out["kept_count"]), _ptr(out.get("out_len")), _ptr(out.get("out_protect")), _ptr(out.get("out_ids")),
        _ptr(out.get("score_global")), _ptr(out.get("score_indiv")),
        C.byref(lq), C.byref(lkv), C.byref(lo),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return out


def mustdrop_decode_evict_strided(q, k_cache, v_cache, acc, ids, protect, length, softmax_scale, decay, budget,
                                  evicted_ids=None, evicted_count=None, workspace=None, stream=None):
    """Sec. 3.5, one decode step on caches given as [B, Lcap, H, d] views of any layout."""
    B, Lcap, H, d = k_cache.shape
    assert k_cache.stride() == v_cache.stride()
    if workspace is None:
        workspace = decode_workspace(B, Lcap, H, k_cache.device)
    lay = _layout(k_cache)
    _call("mustdrop_decode_evict_strided",
        _ptr(q), _view_ptr(k_cache), _view_ptr(v_cache), _ptr(acc), _ptr(ids), _ptr(protect), _ptr(length),
        B, Lcap, H, d,
        softmax_scale, decay, budget,
        _ptr(evicted_ids), _ptr(evicted_count), C.byref(lay),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return workspace


def mustdrop_decode_append_strided(k_new, v_new, k_cache, v_cache, acc, ids, protect, length, new_id, protect_new=1,
                                   stream=None):
    """Eq. 3 on caches given as [B, Lcap, H, d] views of any layout."""
    B, Lcap, H, d = k_cache.shape
    assert k_cache.stride() == v_cache.stride()
    lay = _layout(k_cache)
    _call("mustdrop_decode_append_strided",
        _ptr(k_new), _ptr(v_new), _view_ptr(k_cache), _view_ptr(v_cache), _ptr(acc), _ptr(ids), _ptr(protect),
        _ptr(length), B, Lcap, H, d, int(new_id),
        int(protect_new), C.byref(lay), _stream(stream))


def mustdrop_decode_keep_strided(k_caches, v_caches, keep, acc, ids, protect, length, evicted_ids=None,
                                 evicted_count=None, workspace=None, stream=None):
    """Sec. 3.5, the static policy on caches given as [n_layers, B, Lcap, H, d] views of any layout."""
    n_layers, B, Lcap, H, d = k_caches.shape
    assert k_caches.stride() == v_caches.stride()
    if workspace is None:
        workspace = decode_workspace(B, Lcap, H, k_caches.device)
    lay = _layout(k_caches)
    _call("mustdrop_decode_keep_strided",
        _view_ptr(k_caches), _view_ptr(v_caches), _ptr(keep), _ptr(acc), _ptr(ids), _ptr(protect), _ptr(length),
        n_layers, B, Lcap, H, d,
        _ptr(evicted_ids), _ptr(evicted_count), C.byref(lay), k_caches.stride(0),
        _ptr(workspace), workspace.numel(), _stream(stream))
    return workspace


def _typed(dtype, **tensors):
    for name, t in tensors.items():
        if t is not None and t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, not {t.dtype}")


def _shaped(name, t, shape):
    if t is not None and t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")


def _here(stream, *tensors) -> int:
    """The stream of a call, on the current device: a launch goes there, so every tensor has to be there."""
    import torch
    at = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ValueError(f"tensors must be on one GPU: {t.device}, {tensors[0].device}")
    if at < 0:
        raise ValueError(f"tensors must be on one GPU: {tensors[0].device}")
    if at != torch._C._cuda_getDevice():                   # (torch.cuda.current_device() asks first whether there is a GPU at all)
        raise ValueError(f"tensors on device {at} in a call on device {torch.cuda.current_device()}: make theirs the current one")
    return torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream


def _made_on(stream):
    """What a call makes for itself is made on the stream that it runs on: memory of another one could be in use there until the
    call's own stream writes it, or be given away while that still reads it."""
    import contextlib
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _pool(cache, d):
    """(pages, heads, tokens of a page) of a cache held in 4 bits, uint8 [n_pages, H, page * (d + d / 16)]."""
    import torch
    if cache.dtype is not torch.uint8:
        raise TypeError(f"cache must be torch.uint8, not {cache.dtype}")
    shape, size = cache.shape, d + d // 16
    if len(shape) != 3 or d % 16 or shape[2] % size:
        raise ValueError(f"cache must be [n_pages, H, page * (d + d / 16)] with d = {d}, not {tuple(shape)}")
    return shape[0], shape[1], shape[2] // size


def _rows(t, what):
    """(pointer, md_kv_layout or None) of a [B, N, H, d] view; None for dense token-major memory.  An axis of one element gets a
    stride that the library takes (torch leaves any number there)."""
    if t.is_contiguous():
        return t.data_ptr(), None
    if t.dim() != 4 or t.stride(3) != 1:
        raise ValueError(f"{what} must be [B, N, H, d] with contiguous d")
    n, st = t.shape, list(t.stride())
    for a in range(3):
        if n[a] == 1:
            st[a] = max([n[3]] + [st[c] * n[c] for c in range(3) if c != a and n[c] > 1])
    return t.data_ptr(), KvLayout(st[0], st[1], st[2])


def _row_pair(k, v, names):
    """Pointers and the one layout of two [B, N, H, d] views of one type and shape."""
    if v.dtype is not k.dtype or v.shape != k.shape:
        _typed(k.dtype, **{names[1]: v})
        _shaped(names[1], v, k.shape)
    if k.is_contiguous() and v.is_contiguous():
        return k.data_ptr(), v.data_ptr(), None
    (kp, lay), (vp, other) = _rows(k, names[0]), _rows(v, names[1])
    if (lay is None) != (other is None) or (lay and (lay.batch, lay.token, lay.head) != (other.batch, other.token, other.head)):
        raise ValueError(f"{names[0]} and {names[1]} must have one layout")
    return kp, vp, lay and C.byref(lay)


def cache4_buffer(n_pages, page, H, d, device="cuda"):
    """The pool of a cache held in 4 bits: uint8 [n_pages, H, page * (d + d / 16)]."""
    import torch
    nbytes = library().mustdrop_cache4_bytes(int(n_pages), int(page), int(H), int(d))
    if nbytes == 0:
        raise ValueError(library().mustdrop_last_error().decode())
    return torch.zeros(nbytes, dtype=torch.uint8, device=device).view(n_pages, H, nbytes // (n_pages * H))


def cache4_pages_workspace(B, device="cuda"):
    return _workspace(library().mustdrop_cache4_pages_workspace_bytes(B), device)


def cache4_workspace(q, cache, table):
    """Workspace of mustdrop_cache4_attend for queries [B, N, Hq, d] on this pool with block tables [B, max_pages]."""
    B, N, Hq, d = q.shape
    _, H, page = _pool(cache, d)
    n = library().mustdrop_cache4_attend_workspace_bytes(B, N, Hq, H, d, table.shape[1], page)
    return _workspace(n, q.device)


def mustdrop_cache4_pages(new_len, length, table, free_pages, n_free, missing, page, slots=None, workspace=None, stream=None):
    """Block tables and slots: every sample is to hold new_len entries; length, table, free_pages and n_free are updated in
    place, slots [B, N] (or None) receives the slots of the new entries, missing [1] what the pool is short of (then nothing
    else changes).  All int32.  Returns the workspace used."""
    import torch
    B, max_pages = table.shape
    N = 0 if slots is None else slots.shape[1]
    _typed(torch.int32, new_len=new_len, length=length, table=table, free_pages=free_pages, n_free=n_free, missing=missing, slots=slots)
    _shaped("new_len", new_len, (B,))
    _shaped("length", length, (B,))
    _shaped("n_free", n_free, (1,))
    _shaped("missing", missing, (1,))
    _shaped("slots", slots, (B, N))
    raw = _here(stream, new_len, length, table, free_pages, n_free, missing, slots, workspace)
    if workspace is None:
        with _made_on(stream):
            workspace = cache4_pages_workspace(B, table.device)
    _call("mustdrop_cache4_pages",
        _ptr(new_len), _ptr(length), _ptr(table), _ptr(free_pages), _ptr(n_free), _ptr(slots), _ptr(missing),
        B, max_pages, free_pages.shape[0], int(page), N,
        _ptr(workspace), workspace.numel(), raw)
    return workspace


def mustdrop_cache4_write(k_new, v_new, slots, cache, stream=None):
    """Rows [B, N, H, d] (bf16 / f32 views of one layout) into the cache, at slots [B, N]."""
    import torch
    B, N, H, d = k_new.shape
    n_pages, heads, page = _pool(cache, d)
    _typed(torch.int32, slots=slots)
    _shaped("slots", slots, (B, N))
    kp, vp, lay = _row_pair(k_new, v_new, ("k_new", "v_new"))
    if heads != H:
        raise ValueError(f"rows of {H} heads for a cache of {heads} heads")
    raw = _here(stream, k_new, v_new, slots, cache)
    _call("mustdrop_cache4_write",
        kp, vp, _dtype_code(k_new), _ptr(slots), _ptr(cache),
        B, N, H, d, n_pages, page, lay, raw)


def mustdrop_cache4_read(cache, table, length, k_out, v_out, first=None, stream=None):
    """Entries first .. of the cache into k_out, v_out [B, N, H, d] (bf16 / f32 views of one layout); rows of entries from length on
    are left as they are."""
    import torch
    B, N, H, d = k_out.shape
    n_pages, heads, page = _pool(cache, d)
    max_pages = table.shape[-1]
    _typed(torch.int32, table=table, length=length, first=first)
    _shaped("table", table, (B, max_pages))
    _shaped("length", length, (B,))
    _shaped("first", first, (B,))
    kp, vp, lay = _row_pair(k_out, v_out, ("k_out", "v_out"))
    if heads != H:
        raise ValueError(f"rows of {H} heads for a cache of {heads} heads")
    raw = _here(stream, cache, table, length, k_out, v_out, first)
    _call("mustdrop_cache4_read",
        _ptr(cache), _ptr(table), _ptr(length), _ptr(first), kp, vp, _dtype_code(k_out),
        B, N, H, d, n_pages, page, max_pages, lay, raw)


def mustdrop_cache4_attend(q, cache, table, length, softmax_scale, out=None, lse=None, q_len=None, keep=None, workspace=None, stream=None):
    """Attention of q [B, N, Hq, d] (bf16 / f32, any layout) over the cache, each sample's rows at its last entries (causal).
    Returns out (made as zeros if None); lse [B, Hq, N] f32, q_len [B] int32 and keep [B, max_pages * page] uint8 may be None."""
    import torch
    B, N, Hq, d = q.shape
    n_pages, H, page = _pool(cache, d)
    max_pages = table.shape[-1]
    if out is None:
        with _made_on(stream):
            out = torch.zeros((B, N, Hq, d), dtype=q.dtype, device=q.device)
    _typed(torch.int32, table=table, length=length, q_len=q_len)
    if lse is not None:
        _typed(torch.float32, lse=lse)
        _shaped("lse", lse, (B, Hq, N))
    if keep is not None:
        _typed(torch.uint8, keep=keep)
        _shaped("keep", keep, (B, max_pages * page))
    _typed(q.dtype, out=out)
    _shaped("out", out, q.shape)
    _shaped("table", table, (B, max_pages))
    _shaped("length", length, (B,))
    _shaped("q_len", q_len, (B,))
    raw = _here(stream, q, cache, table, length, out, lse, q_len, keep, workspace)
    if workspace is None:
        with _made_on(stream):
            workspace = cache4_workspace(q, cache, table)
    qp, lq = _rows(q, "q")
    op, lo = _rows(out, "out")
    _call("mustdrop_cache4_attend",
        qp, _dtype_code(q), _ptr(cache), _ptr(table), _ptr(length), _ptr(q_len), _ptr(keep),
        B, N, Hq, H, d, n_pages, page, max_pages, softmax_scale,
        op, _ptr(lse), lq and C.byref(lq), lo and C.byref(lo),
        _ptr(workspace), workspace.numel(), raw)
    return out


def rotary(sections, adjacent=False, axis=None) -> Rotary:
    """How rows turn: sections[a] pairs of channels by axis a, one axis after the other, or pair i by axis[i] (0, 1, ..: as many entries as
    there are pairs; sections then says how many axes there are and pairs in all).  A program keeps it."""
    pairs = sum(int(n) for n in sections)
    which = [a for a, n in enumerate(sections) for _ in range(int(n))] if axis is None else [int(a) for a in axis]
    if len(which) != pairs or not 0 < pairs <= 128 or min(which) < 0 or max(which) >= len(sections) or min(sections) < 0:
        raise ValueError(f"sections {list(sections)} and axis {axis} do not name an axis for each of 1 to 128 pairs")
    return Rotary(pairs, len(sections), int(bool(adjacent)), (C.c_uint8 * 128)(*which))


def rotary_table(n_pos, pairs, base=10000.0, device="cuda"):
    """Cosines and sines [n_pos, pairs, 2] f32 of the angles p * base^(-i / pairs), worked out in 64 bits; a program keeps it.  (Any other
    table of that shape will do, for other frequencies or scalings.)"""
    import numpy as np
    import torch
    at = np.arange(n_pos, dtype=np.float64)[:, None] * float(base) ** (-np.arange(pairs, dtype=np.float64) / pairs)
    return torch.from_numpy(np.stack([np.cos(at), np.sin(at)], axis=-1).astype(np.float32)).to(device)


def _needed(name, t, dtype, shape):
    """Says what is wrong with a tensor that is not contiguous, of this type and of this shape.  (The calls below look at these three
    themselves: a function for each of a call's tensors took a third of the time that the host spends on it.)"""
    _typed(dtype, **{name: t})
    _shaped(name, t, shape)
    assert t.is_contiguous(), "tensors handed to the C ABI must be contiguous"


def _given(name, t, dtype, shape):
    """Device pointer of a tensor that may be None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _needed(name, t, dtype, shape)
    return t.data_ptr()


def _angles(positions, table, turn, B, f32, i32):
    """Checks positions [axes, B, L] and table [n_pos, pairs, 2]; returns (L, n_pos)."""
    at, angles = positions.shape, table.shape
    if positions.dtype is not i32 or len(at) != 3 or at != (turn.axes, B, at[2]) or not positions.is_contiguous():
        _needed("positions", positions, i32, (turn.axes, B, at[-1]))
    if table.dtype is not f32 or len(angles) != 3 or angles != (angles[0], turn.pairs, 2) or not table.is_contiguous():
        _needed("table", table, f32, (angles[0], turn.pairs, 2))
    return at[2], angles[0]


def _side(t, out, shape, names):
    """Pointers and layouts of rows of this shape and of what they become (None: themselves)."""
    if out is not None and (out.dtype is not t.dtype or out.shape != shape):
        _typed(t.dtype, **{names[1]: out})
        _shaped(names[1], out, shape)
    if out is not None and t.is_contiguous() and out.is_contiguous():
        return out, t.data_ptr(), None, out.data_ptr(), None
    p, lay = _rows(t, names[0])
    lay = lay and C.byref(lay)
    if out is None:
        return t, p, lay, p, lay
    o, out_lay = _rows(out, names[1])
    return out, p, lay, o, out_lay and C.byref(out_lay)


def mustdrop_rotate(q, positions, table, turn, k=None, q_out=None, k_out=None, index=None, rows=None, inverse=False, stream=None):
    """Rows q [B, N, Hq, d] and k [B, N, H, d] or None (bf16 / f32, any layout) turned by their positions [axes, B, L] int32 (row (b, i) at
    [:, b, index[b, i]], or [:, b, i] without index [B, N] int32), with table [n_pos, pairs, 2] f32 (rotary_table) and turn = rotary(..).  q_out and
    k_out: None for in place.  rows [B] int32: rows from there on stay.  inverse: the way back.  Returns (q_out, k_out)."""
    import torch
    i32 = torch.int32
    B, N, Hq, d = q.shape
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    L, n_pos = _angles(positions, table, turn, B, torch.float32, i32)
    at, count = _given("index", index, i32, (B, N)), _given("rows", rows, i32, (B,))
    q_out, qp, ql, qo, qol = _side(q, q_out, (B, N, Hq, d), ("q", "q_out"))
    H, kp, kl, ko, kol = 0, None, None, None, None
    if k is not None:
        shape = k.shape
        if k.dtype is not q.dtype or len(shape) != 4 or shape != (B, N, shape[2], d):
            _typed(q.dtype, k=k)
            _shaped("k", k, (B, N, shape[2], d))
        H = shape[2]
        k_out, kp, kl, ko, kol = _side(k, k_out, shape, ("k", "k_out"))
    raw = _here(stream, q, k, positions, table, q_out, k_out, index, rows)
    _call("mustdrop_rotate",
        qp, kp, BF16 if q.dtype is torch.bfloat16 else _dtype_code(q), positions.data_ptr(), at, table.data_ptr(), count,
        B, N, L, Hq, H, d, n_pos, C.byref(turn), 1 if inverse else 0, qo, ko, ql, kl, qol, kol, raw)
    return q_out, k_out


def mustdrop_cache4_append(q, k_new, v_new, positions, table, turn, slots, cache, q_out=None, index=None, stream=None):
    """Rows k_new, v_new [B, N, H, d] (bf16 / f32 views of one layout) into the cache at slots [B, N], k_new turned on the way; q
    [B, N, Hq, d] (or None) turned into q_out (None: in place), which is returned.  Rows without a slot stay out, and their queries.  For
    positions, table, turn and index see mustdrop_rotate."""
    import torch
    i32 = torch.int32
    B, N, H, d = k_new.shape
    n_pages, heads, page = _pool(cache, d)
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    L, n_pos = _angles(positions, table, turn, B, torch.float32, i32)
    if slots.dtype is not i32 or slots.shape != (B, N) or not slots.is_contiguous():
        _needed("slots", slots, i32, (B, N))
    at = _given("index", index, i32, (B, N))
    kp, vp, lay = _row_pair(k_new, v_new, ("k_new", "v_new"))
    if heads != H:
        raise ValueError(f"rows of {H} heads for a cache of {heads} heads")
    Hq, qp, ql, qo, qol = 0, None, None, None, None
    if q is not None:
        shape = q.shape
        if q.dtype is not k_new.dtype or len(shape) != 4 or shape != (B, N, shape[2], d):
            _typed(k_new.dtype, q=q)
            _shaped("q", q, (B, N, shape[2], d))
        Hq = shape[2]
        q_out, qp, ql, qo, qol = _side(q, q_out, shape, ("q", "q_out"))
    raw = _here(stream, k_new, v_new, q, q_out, positions, table, slots, cache, index)
    _call("mustdrop_cache4_append",
        qp, kp, vp, BF16 if k_new.dtype is torch.bfloat16 else _dtype_code(k_new), positions.data_ptr(), at, table.data_ptr(), slots.data_ptr(),
        _ptr(cache), B, N, L, Hq, H, d, n_pos, n_pages, page, C.byref(turn), qo, ql, lay, qol, raw)
    return q_out


def cache4_bounds_buffer(n_pages, H, d, device="cuda"):
    """What mustdrop_cache4_bounds writes: bounds int8 [n_pages, H, 2, d] and scales uint8 [n_pages, H]."""
    import torch
    return torch.zeros((n_pages, H, 2, d), dtype=torch.int8, device=device), torch.zeros((n_pages, H), dtype=torch.uint8, device=device)


def _bounds(bounds, scales, i8, u8):
    """(pages, heads, channels) of a cache's bounds."""
    shape = bounds.shape
    n_pages, H, two, d = shape
    if bounds.dtype is not i8 or two != 2 or not bounds.is_contiguous():
        _needed("bounds", bounds, i8, (n_pages, H, 2, d))
    if scales.dtype is not u8 or scales.shape != (n_pages, H) or not scales.is_contiguous():
        _needed("scales", scales, u8, (n_pages, H))
    return n_pages, H, d


def _requests(table, length, q_len, B, i32):
    """Checks a block table [B, max_pages], lengths [B] and row counts [B] or None; returns (max_pages, pointer of q_len)."""
    shape = table.shape
    if table.dtype is not i32 or len(shape) != 2 or shape[0] != B or not table.is_contiguous():
        _needed("table", table, i32, (B, shape[-1]))
    if length.dtype is not i32 or length.shape != (B,) or not length.is_contiguous():
        _needed("length", length, i32, (B,))
    return shape[1], None if q_len is None else _given("q_len", q_len, i32, (B,))


def mustdrop_cache4_bounds(cache, table, length, n, bounds, scales, first=None, stream=None):
    """Bounds of the keys of the pages that hold entries first .. first + n - 1 (below length) of every sample, into bounds int8
    [n_pages, H, 2, d] and scales uint8 [n_pages, H] (cache4_bounds_buffer)."""
    import torch
    i32 = torch.int32
    pages, H, d = _bounds(bounds, scales, torch.int8, torch.uint8)
    n_pages, heads, page = _pool(cache, d)
    if pages != n_pages or H != heads:
        raise ValueError(f"bounds of {pages} pages and {H} heads for a cache of {n_pages} and {heads}")
    B = table.shape[0]
    max_pages, _ = _requests(table, length, None, B, i32)
    start = _given("first", first, i32, (B,))
    raw = _here(stream, cache, table, length, bounds, scales, first)
    _call("mustdrop_cache4_bounds",
        _ptr(cache), table.data_ptr(), length.data_ptr(), start, bounds.data_ptr(), scales.data_ptr(), B, int(n), H, d, n_pages, page, max_pages, raw)


def cache4_choose_workspace(q, bounds, table, page=16):
    """Workspace of mustdrop_cache4_choose for queries [B, N, Hq, d] on these bounds with block tables [B, max_pages]."""
    B, N, Hq, d = q.shape
    n = library().mustdrop_cache4_choose_workspace_bytes(B, N, Hq, bounds.shape[1], d, table.shape[1], page)
    return _workspace(n, q.device)


def mustdrop_cache4_choose(q, bounds, scales, table, length, page, chosen, q_len=None, first_pages=0, last_pages=1, workspace=None, stream=None):
    """The pages that each of the last q_len tokens of every sample is to read, for each K/V head: chosen [B, N, H, budget] int32
    receives entries of the block table in ascending order, then -1.  q [B, N, Hq, d] (bf16 / f32, any layout); bounds and scales from
    mustdrop_cache4_bounds; the first first_pages and the last last_pages are always among them.  Returns chosen."""
    import torch
    i32 = torch.int32
    B, N, Hq, d = q.shape
    n_pages, H, channels = _bounds(bounds, scales, torch.int8, torch.uint8)
    if channels != d:
        raise ValueError(f"bounds of {channels} channels for queries of {d}")
    max_pages, rows = _requests(table, length, q_len, B, i32)
    lists = chosen.shape
    if chosen.dtype is not i32 or len(lists) != 4 or lists != (B, N, H, lists[3]) or not chosen.is_contiguous():
        _needed("chosen", chosen, i32, (B, N, H, lists[-1]))
    raw = _here(stream, q, bounds, scales, table, length, chosen, q_len, workspace)
    if workspace is None:
        with _made_on(stream):
            workspace = cache4_choose_workspace(q, bounds, table, int(page))
    qp, lq = _rows(q, "q")
    _call("mustdrop_cache4_choose",
        qp, BF16 if q.dtype is torch.bfloat16 else _dtype_code(q), bounds.data_ptr(), scales.data_ptr(), table.data_ptr(), length.data_ptr(), rows,
        B, N, Hq, H, d, n_pages, int(page), max_pages, int(first_pages), int(last_pages), lists[3],
        chosen.data_ptr(), lq and C.byref(lq), _ptr(workspace), workspace.numel(), raw)
    return chosen


def cache4_attend_chosen_workspace(q, cache, chosen):
    """Workspace of mustdrop_cache4_attend_chosen for queries [B, N, Hq, d] on this pool with lists [B, N, H, budget]."""
    B, N, Hq, d = q.shape
    _, H, page = _pool(cache, d)
    n = library().mustdrop_cache4_attend_chosen_workspace_bytes(B, N, Hq, H, d, chosen.shape[3], page)
    return _workspace(n, q.device)


def mustdrop_cache4_attend_chosen(q, cache, table, length, chosen, softmax_scale, out=None, lse=None, q_len=None, keep=None, workspace=None, stream=None):
    """mustdrop_cache4_attend over the pages that chosen [B, N, H, budget] int32 names for each token and K/V head (ascending; what does
    not ascend or is no entry of the table does not count).  Returns out (made as zeros if None)."""
    import torch
    i32 = torch.int32
    shape = q.shape
    B, N, Hq, d = shape
    n_pages, H, page = _pool(cache, d)
    if out is None:
        with _made_on(stream):
            out = torch.zeros((B, N, Hq, d), dtype=q.dtype, device=q.device)
    elif out.dtype is not q.dtype or out.shape != shape:
        _typed(q.dtype, out=out)
        _shaped("out", out, shape)
    max_pages, rows = _requests(table, length, q_len, B, i32)
    lists = chosen.shape
    if chosen.dtype is not i32 or len(lists) != 4 or lists != (B, N, H, lists[3]) or not chosen.is_contiguous():
        _needed("chosen", chosen, i32, (B, N, H, lists[-1]))
    sums, mask = _given("lse", lse, torch.float32, (B, Hq, N)), _given("keep", keep, torch.uint8, (B, max_pages * page))
    raw = _here(stream, q, cache, table, length, chosen, out, lse, q_len, keep, workspace)
    if workspace is None:
        with _made_on(stream):
            workspace = cache4_attend_chosen_workspace(q, cache, chosen)
    qp, lq = _rows(q, "q")
    op, lo = _rows(out, "out")
    _call("mustdrop_cache4_attend_chosen",
        qp, BF16 if q.dtype is torch.bfloat16 else _dtype_code(q), _ptr(cache), table.data_ptr(), length.data_ptr(), rows, mask, chosen.data_ptr(),
        B, N, Hq, H, d, n_pages, page, max_pages, lists[3], softmax_scale,
        op, sums, lq and C.byref(lq), lo and C.byref(lo),
        _ptr(workspace), workspace.numel(), raw)
    return out


def profile_start():
    """Benchmarking aid: bracket every kernel launch with HIP events until profile_stop()."""
    _check(library().mustdrop_profile_start())


def profile_stop(cap: int = 64) -> Dict[str, Dict[str, float]]:
    """Returns {kernel name: {"ms": summed milliseconds, "calls": launches}}."""
    names = C.create_string_buffer(64 * cap)
    ms = (C.c_float * cap)()
    calls = (C.c_int * cap)()
    n = C.c_int(0)
    _check(library().mustdrop_profile_stop(names, ms, calls, C.c_int(cap), C.byref(n)))
    out = {}
    for i in range(n.value):
        nm = names.raw[64 * i:64 * (i + 1)].split(b"\0", 1)[0].decode()
        out[nm] = {"ms": float(ms[i]), "calls": int(calls[i])}
    return out
