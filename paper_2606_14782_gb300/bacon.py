"""Python binding of the BACON C ABI (``include/bacon.h``).

Argument marshalling only: every step of the compression runs in the CUDA
kernels of ``libbacon.so``.  torch tensors provide device memory and streams;
their raw pointers cross the ABI.  There is no CPU fallback: if the library
is missing, loading it raises.
"""

from __future__ import annotations

import ctypes
import os
import struct
from array import array

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbacon.so")

BACON_OK, BACON_EINVAL, BACON_ENOMEM, BACON_ECUDA, BACON_ESTATE, BACON_ETIMEOUT, \
    BACON_EUNSUPPORTED = range(7)
STATUS_NAMES = {0: "BACON_OK", 1: "BACON_EINVAL", 2: "BACON_ENOMEM", 3: "BACON_ECUDA",
                4: "BACON_ESTATE", 5: "BACON_ETIMEOUT", 6: "BACON_EUNSUPPORTED"}
SCORE_KINDS = {"B": 0, "Q": 1, "E": 2, "V": 3, "Bpool": 4, "S": 5, "lambda": 6}

# every symbol include/bacon.h declares
EXPORTS = ("bacon_default_params", "bacon_init", "bacon_destroy", "bacon_last_error",
           "bacon_state_create", "bacon_state_reset", "bacon_state_destroy",
           "bacon_score_layer", "bacon_select", "bacon_compact",
           "bacon_compress_all_layers", "bacon_compress_host", "bacon_get_scores",
           "bacon_profile_enable", "bacon_profile_read", "bacon_window_scores_noalloc",
           "bacon_compress_layer_budgets", "bacon_pyramid_budgets",
           "bacon_compress_adaptive", "bacon_compress_with_lse", "bacon_sweep",
           "bacon_sync", "bacon_cache_create", "bacon_cache_destroy", "bacon_cache_plan",
           "bacon_cache_locate", "bacon_cache_release", "bacon_cache_shorten",
           "bacon_cache_store", "bacon_cache_load", "bacon_cache_attend", "bacon_cache_sync",
           "bacon_rotary_frequencies", "bacon_rotary_create", "bacon_rotary_destroy",
           "bacon_rotary_apply", "bacon_cache_store_rotated", "bacon_block_norm",
           "bacon_logits_create", "bacon_logits_destroy", "bacon_logits_process",
           "bacon_logits_sync")
MAX_VARIANTS = 32
PROFILE_STAGES = ("window_stats", "window_combine", "window_scores", "calibrate_select",
                  "gather")


CACHE_FORMATS = {"e4m3": 0, "int8": 1}
CACHE_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ROPE_SCALINGS = {None: 0, "linear": 1, "base": 2, "rotations": 3, "dims": 4}
NORMS = {None: 0, "rms": 1, "layer": 2}
GATES = {"linear": 0, "sigmoid": 1, "tanh": 2, "silu": 3}


class BaconError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class Params(ctypes.Structure):
    """Mirror of ``bacon_params``."""
    _fields_ = [("r", ctypes.c_int), ("m", ctypes.c_int), ("rho", ctypes.c_int),
                ("gamma", ctypes.c_float), ("eps", ctypes.c_float),
                ("use_E", ctypes.c_int), ("use_L", ctypes.c_int), ("use_T", ctypes.c_int),
                ("keep_window", ctypes.c_int), ("max_seq_len", ctypes.c_int),
                ("max_requests", ctypes.c_int), ("keep_scores", ctypes.c_int)]


class Variant(ctypes.Structure):
    """Mirror of ``bacon_variant``."""
    _fields_ = [("r", ctypes.c_int), ("m", ctypes.c_int), ("rho", ctypes.c_int),
                ("gamma", ctypes.c_float), ("use_E", ctypes.c_int), ("use_L", ctypes.c_int),
                ("use_T", ctypes.c_int)]


class CacheDesc(ctypes.Structure):
    """Mirror of ``bacon_cache_desc``."""
    _fields_ = ([(n, ctypes.c_int) for n in ("layers", "kv_heads", "q_heads", "head_dim", "page",
                                             "pages", "max_requests", "max_blocks", "format",
                                             "dtype")]
                + [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")])


class Rows(ctypes.Structure):
    """Mirror of ``bacon_rows``."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("in_", "out", "weight")]
                + [("heads", ctypes.c_int)]
                + [(n, ctypes.c_longlong) for n in ("in_request", "in_token", "in_head",
                                                    "out_request", "out_token", "out_head")])


class Block(ctypes.Structure):
    """Mirror of ``bacon_block``."""
    _fields_ = ([(n, ctypes.c_int) for n in ("tokens", "width", "dtype", "residual_dtype",
                                             "weight_dtype", "post", "pre", "activation")]
                + [(n, ctypes.c_float) for n in ("scale", "eps", "weight_offset")]
                + [("gate_channel", ctypes.c_int)]
                + [(n, ctypes.c_longlong) for n in ("gate_token", "y_token", "x_token",
                                                    "sum_token", "normed_token")]
                + [(n, ctypes.c_void_p) for n in ("y", "x", "gate", "post_weight", "post_bias",
                                                  "pre_weight", "pre_bias", "sum", "normed")])


class LogitsRows(ctypes.Structure):
    """Mirror of ``bacon_logits_rows``."""
    _fields_ = ([(n, ctypes.c_int) for n in ("rows", "dtype", "out_dtype", "requests", "capacity",
                                             "biases")]
                + [(n, ctypes.c_longlong) for n in ("row_stride", "out_stride", "token_stride",
                                                    "mask_stride")]
                + [(n, ctypes.c_void_p) for n in ("logits", "out", "tokens", "request", "prompt",
                                                  "lengths", "repetition", "frequency", "presence",
                                                  "temperature", "bias_tokens", "bias_values",
                                                  "mask", "best", "logprob", "lse")])


def _packer(cls):
    """Values of a mirror's fields, in order, as its bytes: a call's descriptor
    in a third of the time that setting the fields takes."""
    codes = {ctypes.c_int: "i", ctypes.c_float: "f", ctypes.c_longlong: "q", ctypes.c_void_p: "P"}
    return struct.Struct("@" + "".join(codes[t] for _, t in cls._fields_)).pack


_pack_rows, _pack_block, _pack_logits = _packer(Rows), _packer(Block), _packer(LogitsRows)

_lib = None
_vp = ctypes.c_void_p
_int = ctypes.c_int
_i64 = ctypes.c_longlong


def load() -> ctypes.CDLL:
    """Load libbacon.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2606_14782_gb300.build` (needs nvcc)")
    lib = ctypes.CDLL(LIB_PATH)
    lib.bacon_default_params.argtypes = [ctypes.POINTER(Params)]
    lib.bacon_default_params.restype = None
    lib.bacon_init.argtypes = [ctypes.POINTER(_vp), _int, _int, _int, _int, _int, _int, _int,
                               ctypes.POINTER(Params)]
    lib.bacon_destroy.argtypes = [_vp]
    lib.bacon_destroy.restype = None
    lib.bacon_last_error.argtypes = []
    lib.bacon_last_error.restype = ctypes.c_char_p
    lib.bacon_state_create.argtypes = [_vp, ctypes.POINTER(_vp)]
    lib.bacon_state_reset.argtypes = [_vp]
    lib.bacon_state_destroy.argtypes = [_vp]
    lib.bacon_state_destroy.restype = None
    lib.bacon_score_layer.argtypes = [_vp, _vp, _int, _vp, _vp, _int, _vp, _vp]
    lib.bacon_select.argtypes = [_vp, _vp, _int, _vp, _vp]
    lib.bacon_compact.argtypes = [_vp, _vp, _vp, _vp, _int, _int, _vp, _vp, _vp]
    lib.bacon_compress_all_layers.argtypes = [_vp, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                              ctypes.POINTER(_vp), _int, _int, ctypes.POINTER(_vp),
                                              ctypes.POINTER(_vp), _vp, _vp]
    lib.bacon_compress_host.argtypes = [_vp, _int, _vp, _vp, _vp, _int, _int, _vp, _vp, _vp, _vp]
    lib.bacon_get_scores.argtypes = [_vp, _int, _vp, ctypes.c_size_t, _vp]
    lib.bacon_sync.argtypes = [_vp, _vp]
    lib.bacon_compress_layer_budgets.argtypes = [_vp, _int, ctypes.POINTER(_vp),
                                                 ctypes.POINTER(_vp), ctypes.POINTER(_vp), _int,
                                                 ctypes.POINTER(_int), ctypes.POINTER(_vp),
                                                 ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp]
    lib.bacon_pyramid_budgets.argtypes = [_int, _int, _int, _int, ctypes.POINTER(_int)]
    lib.bacon_compress_with_lse.argtypes = [_vp, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp), _int, _int,
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, _vp]
    lib.bacon_compress_adaptive.argtypes = [_vp, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), _int, _int, ctypes.c_float,
                                            ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                            ctypes.POINTER(_vp), _vp, _vp]
    lib.bacon_sweep.argtypes = [_vp, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _int, _int,
                                _int, ctypes.POINTER(Variant), _vp, _vp, _vp]
    lib.bacon_pyramid_budgets.restype = None
    lib.bacon_window_scores_noalloc.argtypes = [_int, _int, _int, _int, _vp, _vp, _int, _vp,
                                                _vp, _vp, _vp]
    lib.bacon_profile_enable.argtypes = [_vp, _int]
    lib.bacon_profile_read.argtypes = [_vp, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(_int), _int]
    lib.bacon_cache_create.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(CacheDesc)]
    lib.bacon_cache_destroy.argtypes = [_vp]
    lib.bacon_cache_destroy.restype = None
    lib.bacon_cache_plan.argtypes = [_vp, _int, _vp, _vp, _int, _vp, _vp, _vp, _int, _vp, _vp,
                                     _vp, _vp]
    lib.bacon_cache_locate.argtypes = [_vp, _int, _vp, _vp, _vp, _int, _vp, _vp]
    lib.bacon_cache_release.argtypes = [_vp, _int, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.bacon_cache_shorten.argtypes = [_vp, _int, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.bacon_cache_store.argtypes = [_vp, _int, _int, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp]
    lib.bacon_cache_load.argtypes = [_vp, _int, _vp, _vp, _vp, _vp]
    lib.bacon_cache_attend.argtypes = [_vp, _int, _int, _int, _vp, _i64, _i64, _vp, _vp, _vp,
                                       _int, ctypes.c_float, _vp, _vp, _vp]
    lib.bacon_cache_sync.argtypes = [_vp, _vp]
    lib.bacon_rotary_frequencies.argtypes = [_int] + [ctypes.c_double, _int] + [ctypes.c_double] * 4 + [
        ctypes.POINTER(ctypes.c_double)]
    lib.bacon_rotary_create.argtypes = [ctypes.POINTER(_vp), _int, _int, _int, ctypes.c_float,
                                        ctypes.POINTER(ctypes.c_double), ctypes.c_char_p]
    lib.bacon_rotary_destroy.argtypes = [_vp]
    lib.bacon_rotary_destroy.restype = None
    lib.bacon_rotary_apply.argtypes = [_vp, _int, _int, ctypes.c_char_p, ctypes.c_char_p, _int, _int,
                                       ctypes.c_float, ctypes.c_float, _int, _vp, _vp]
    lib.bacon_cache_store_rotated.argtypes = [_vp, _vp, _int, ctypes.c_char_p, ctypes.c_char_p, _vp,
                                              _i64, _i64, _int, ctypes.c_float, ctypes.c_float, _vp,
                                              _vp, _vp]
    lib.bacon_block_norm.argtypes = [ctypes.c_char_p, _vp]
    lib.bacon_logits_create.argtypes = [ctypes.POINTER(_vp), _int]
    lib.bacon_logits_destroy.argtypes = [_vp]
    lib.bacon_logits_destroy.restype = None
    lib.bacon_logits_process.argtypes = [_vp, ctypes.c_char_p, _vp]
    lib.bacon_logits_sync.argtypes = [_vp, _vp]
    for name in ("bacon_cache_create", "bacon_cache_plan", "bacon_cache_locate",
                 "bacon_cache_release", "bacon_cache_shorten", "bacon_cache_store",
                 "bacon_cache_load",
                 "bacon_cache_attend", "bacon_cache_sync", "bacon_rotary_frequencies",
                 "bacon_rotary_create", "bacon_rotary_apply", "bacon_cache_store_rotated",
                 "bacon_block_norm", "bacon_logits_create", "bacon_logits_process",
                 "bacon_logits_sync",
                 "bacon_sweep", "bacon_compress_with_lse", "bacon_compress_adaptive",
                 "bacon_compress_layer_budgets",
                 "bacon_window_scores_noalloc",
                 "bacon_profile_enable", "bacon_profile_read",
                 "bacon_init", "bacon_state_create", "bacon_state_reset", "bacon_score_layer",
                 "bacon_select", "bacon_compact", "bacon_compress_all_layers",
                 "bacon_compress_host", "bacon_get_scores", "bacon_sync"):
        getattr(lib, name).restype = _int
    _lib = lib
    return lib


def _check(status: int):
    if status != BACON_OK:
        msg = load().bacon_last_error().decode(errors="replace")
        raise BaconError(status, msg)


def default_params(**overrides) -> Params:
    p = Params()
    load().bacon_default_params(ctypes.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def _stream_ptr(stream) -> int:
    if stream is None:  # the current stream, without building a Stream object
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _empty(shape, dtype, device, stream):
    """An output that a call on `stream` allocates.  It is that stream's memory:
    memory of the current one may have been freed there with work on it still to
    run.  The current stream, where the caller goes on with it, is recorded."""
    if stream is not None and torch.device(device).type == "cuda":
        here = torch.cuda.current_stream(device)
        if stream.cuda_stream != here.cuda_stream:
            if not hasattr(stream, "stream_id"):  # not torch's own: its address is enough
                stream = torch.cuda.ExternalStream(stream.cuda_stream, device)
            with torch.cuda.stream(stream):
                t = torch.empty(shape, dtype=dtype, device=device)
            t.record_stream(here)
            return t
    return torch.empty(shape, dtype=dtype, device=device)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _ptr_array(ptrs):
    arr = (_vp * len(ptrs))()
    for i, p in enumerate(ptrs):
        arr[i] = p
    return arr


def _pair_table(t, pairs):
    """Pointers of t[r, l] for pair i = r * layers + l of a contiguous
    [R, layers, ...] tensor."""
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    base = t.data_ptr()
    stride = t.numel() // (t.shape[0] * t.shape[1]) * t.element_size()
    # one buffer of addresses instead of one ctypes store per pair: 28 pairs
    # take 1.5 us instead of 8
    ptrs = array("Q", range(base, base + stride * pairs, stride) if stride else [base] * pairs)
    return (_vp * pairs).from_buffer(ptrs)


class Context:
    """Owns a ``bacon_ctx`` (one model shape)."""

    def __init__(self, layers, kv_heads, q_heads, head_dim, window, pool=7, budget=None,
                 params: Params | None = None, **param_overrides):
        lib = load()
        if params is None:
            params = default_params(**param_overrides)
        self.params = params
        self.layers, self.kv_heads, self.q_heads = layers, kv_heads, q_heads
        self.head_dim, self.window, self.pool = head_dim, window, pool
        self.budget = budget if budget is not None else window
        h = _vp()
        _check(lib.bacon_init(ctypes.byref(h), layers, kv_heads, q_heads, head_dim, window,
                              pool, self.budget, ctypes.byref(params)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load().bacon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -------------------------------------------------------- whole step
    def compress_all_layers(self, qwin, k, v, budget, k_out=None, v_out=None, idx_out=None,
                            stream=None):
        """qwin [R, layers, Hq, W, d], k/v [R, layers, Hkv, N, d] (bf16, cuda,
        contiguous).  Returns (k_out, v_out, idx) with shapes
        [R, layers, Hkv, kept, d] and [R, layers, Hkv, kept]."""
        R, Ly, Hq, W, d = qwin.shape
        N = k.shape[3]
        kept = min(budget, N)
        shape_o = (R, Ly, self.kv_heads, kept, d)
        if k_out is None:
            k_out = _empty(shape_o, k.dtype, k.device, stream)
        if v_out is None:
            v_out = _empty(shape_o, v.dtype, v.device, stream)
        if idx_out is None:
            idx_out = _empty(shape_o[:-1], torch.int32, k.device, stream)
        if not idx_out.is_contiguous():
            raise ValueError("tensors must be contiguous")
        tq, tk, tv, tko, tvo = (_pair_table(t, R * Ly) for t in (qwin, k, v, k_out, v_out))
        _check(load().bacon_compress_all_layers(self.handle, R, tq, tk, tv, N, budget, tko, tvo,
                                                idx_out.data_ptr(), _stream_ptr(stream)))
        self._last_units, self._last_N = R * Ly * self.kv_heads, N
        return k_out, v_out, idx_out

    def compress_layer_budgets(self, qwin, k, v, layer_budgets, stream=None):
        """Per-layer budgets (window included).  Returns lists indexed
        [request][layer] of k_out [Hkv, kept_l, d], v_out and idx [Hkv, kept_l]."""
        R, Ly, Hq, W, d = qwin.shape
        N = k.shape[3]
        assert len(layer_budgets) == Ly
        kept = [min(int(b), N) for b in layer_budgets]
        ko = [[_empty((self.kv_heads, kept[l], d), k.dtype, k.device, stream)
               for l in range(Ly)] for _ in range(R)]
        vo = [[_empty(ko[r][l].shape, k.dtype, k.device, stream) for l in range(Ly)] for r in range(R)]
        ix = [[_empty((self.kv_heads, kept[l]), torch.int32, k.device, stream)
               for l in range(Ly)] for _ in range(R)]
        pairs = [(r, l) for r in range(R) for l in range(Ly)]
        # (a tensor of other requests or layers is indexed pair by pair)
        tq, tk, tv = (_pair_table(t, len(pairs))
                      if t.is_contiguous() and tuple(t.shape[:2]) == (R, Ly) else
                      _ptr_array([t[r, l].data_ptr() for r, l in pairs]) for t in (qwin, k, v))
        tko = _ptr_array([ko[r][l].data_ptr() for r, l in pairs])
        tvo = _ptr_array([vo[r][l].data_ptr() for r, l in pairs])
        tix = _ptr_array([ix[r][l].data_ptr() for r, l in pairs])
        b = (_int * Ly)(*[int(x) for x in layer_budgets])
        _check(load().bacon_compress_layer_budgets(self.handle, R, tq, tk, tv, N, b, tko, tvo,
                                                   tix, _stream_ptr(stream)))
        self._last_units, self._last_N = R * Ly * self.kv_heads, N
        return ko, vo, ix

    def compress_with_lse(self, qwin, k, v, lse, budget, k_out=None, v_out=None, idx_out=None,
                          stream=None):
        """As compress_all_layers, with the window rows' natural-log softmax
        normalisers lse [R, layers, Hq, W] (fp32, cuda) from the prefill."""
        R, Ly, Hq, W, d = qwin.shape
        N = k.shape[3]
        kept = min(budget, N)
        shape_o = (R, Ly, self.kv_heads, kept, d)
        k_out = _empty(shape_o, k.dtype, k.device, stream) if k_out is None else k_out
        v_out = _empty(shape_o, v.dtype, v.device, stream) if v_out is None else v_out
        if idx_out is None:
            idx_out = _empty(shape_o[:-1], torch.int32, k.device, stream)
        tq, tk, tv, tl, tko, tvo = (_pair_table(t, R * Ly) for t in (qwin, k, v, lse, k_out, v_out))
        _check(load().bacon_compress_with_lse(self.handle, R, tq, tk, tv, tl, N, budget, tko, tvo,
                                              idx_out.data_ptr(), _stream_ptr(stream)))
        self._last_units, self._last_N = R * Ly * self.kv_heads, N
        return k_out, v_out, idx_out

    def compress_adaptive(self, qwin, k, v, budget, alpha=0.2, stream=None):
        """AdaKV-style head budgets.  Returns (k_out, v_out, idx, counts):
        k_out/v_out [R, layers, Hkv * kept, d] and idx [R, layers, Hkv * kept]
        flat per layer (heads in order), counts [R, layers, Hkv]."""
        R, Ly, Hq, W, d = qwin.shape
        N = k.shape[3]
        kept = min(budget, N)
        ko = _empty((R, Ly, self.kv_heads * kept, d), k.dtype, k.device, stream)
        vo = _empty(ko.shape, k.dtype, k.device, stream)
        ix = _empty((R, Ly, self.kv_heads * kept), torch.int32, k.device, stream)
        counts = _empty((R, Ly, self.kv_heads), torch.int32, k.device, stream)
        tq, tk, tv, tko, tvo, tix = (_pair_table(t, R * Ly) for t in (qwin, k, v, ko, vo, ix))
        _check(load().bacon_compress_adaptive(self.handle, R, tq, tk, tv, N, budget,
                                              float(alpha), tko, tvo, tix, counts.data_ptr(),
                                              _stream_ptr(stream)))
        self._last_units, self._last_N = R * Ly * self.kv_heads, N
        return ko, vo, ix, counts

    def sweep(self, qwin, k, budget, variants, idx_out=None, lambda_out=None, stream=None):
        """Selections under several hyper-parameter sets from one set of
        window passes.  variants: sequence of dicts with any of r, m, rho,
        gamma, use_E, use_L, use_T (the rest from the context's parameters).
        Returns (idx [V, R, layers, Hkv, kept] int32, lambda [V, R, layers,
        Hkv] fp32)."""
        R, Ly, Hq, W, d = qwin.shape
        N = k.shape[3]
        kept = min(budget, N)
        nv = len(variants)
        arr = (Variant * max(nv, 1))()
        for j, x in enumerate(variants):
            for f, _ in Variant._fields_:
                setattr(arr[j], f, x.get(f, getattr(self.params, f)))
        if idx_out is None:
            idx_out = _empty((nv, R, Ly, self.kv_heads, kept), torch.int32, k.device, stream)
        if lambda_out is None:
            lambda_out = _empty((nv, R, Ly, self.kv_heads), torch.float32, k.device, stream)
        tq, tk = (_pair_table(t, R * Ly) for t in (qwin, k))
        _check(load().bacon_sweep(self.handle, R, tq, tk, N, budget, nv, arr,
                                  idx_out.data_ptr(), lambda_out.data_ptr(),
                                  _stream_ptr(stream)))
        return idx_out, lambda_out

    def compress_host(self, qwin, k, v, budget, k_out=None, v_out=None, idx_out=None,
                      stream=None):
        """The same step on host (CPU, ideally pinned) tensors; blocks until
        the outputs are on the host."""
        R, Ly, Hq, W, d = qwin.shape
        N = k.shape[3]
        kept = min(budget, N)
        shape_o = (R, Ly, self.kv_heads, kept, d)
        pin = k.is_pinned()
        if k_out is None:
            k_out = torch.empty(shape_o, dtype=k.dtype, pin_memory=pin)
        if v_out is None:
            v_out = torch.empty(shape_o, dtype=v.dtype, pin_memory=pin)
        if idx_out is None:
            idx_out = torch.empty(shape_o[:-1], dtype=torch.int32, pin_memory=pin)
        _check(load().bacon_compress_host(self.handle, R, qwin.data_ptr(), k.data_ptr(),
                                          v.data_ptr(), N, budget, k_out.data_ptr(),
                                          v_out.data_ptr(), idx_out.data_ptr(),
                                          _stream_ptr(stream)))
        self._last_units, self._last_N = R * Ly * self.kv_heads, N
        return k_out, v_out, idx_out

    def scores(self, kind: str, out=None, stream=None):
        """Intermediate per-token arrays of the last whole-step call (fp32)."""
        n = self._last_count(kind)
        if out is None:
            out = _empty(n, torch.float32, "cuda", stream)
        _check(load().bacon_get_scores(self.handle, SCORE_KINDS[kind], out.data_ptr(),
                                       out.numel(), _stream_ptr(stream)))
        return out

    def _last_count(self, kind):
        return self._last_units * (1 if kind == "lambda" else self._last_N)

    def sync(self, stream=None):
        _check(load().bacon_sync(self.handle, _stream_ptr(stream)))

    def profile(self, enable: bool):
        _check(load().bacon_profile_enable(self.handle, int(enable)))

    def profile_read(self):
        """{stage: (total ms, launches)} since the previous read."""
        n = len(PROFILE_STAGES)
        ms = (ctypes.c_double * n)()
        cnt = (_int * n)()
        _check(load().bacon_profile_read(self.handle, ms, cnt, n))
        return {name: (ms[i], cnt[i]) for i, name in enumerate(PROFILE_STAGES)}

    # ----------------------------------------------- layer by layer
    def compact(self, k, v, idx, k_out=None, v_out=None, stream=None):
        """k/v [Hkv, N, d], idx [Hkv, count] int32 (cuda)."""
        Hkv, N, d = k.shape
        count = idx.shape[-1]
        if k_out is None:
            k_out = _empty((Hkv, count, d), k.dtype, k.device, stream)
        if v_out is None:
            v_out = _empty((Hkv, count, d), v.dtype, v.device, stream)
        _check(load().bacon_compact(self.handle, k.data_ptr(), v.data_ptr(), idx.data_ptr(), N,
                                    count, k_out.data_ptr(), v_out.data_ptr(),
                                    _stream_ptr(stream)))
        return k_out, v_out


def pyramid_budgets(layers, window, budget, beta=20):
    """The library's pyramid budget schedule (bacon_pyramid_budgets)."""
    out = (_int * layers)()
    load().bacon_pyramid_budgets(layers, window, budget, beta, out)
    return list(out)


class State:
    """Per-request persistence state for layer-by-layer scoring."""

    def __init__(self, ctx: Context):
        self.ctx = ctx
        h = _vp()
        _check(load().bacon_state_create(ctx.handle, ctypes.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load().bacon_state_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self):
        _check(load().bacon_state_reset(self.handle))

    def score_layer(self, layer, qwin, k, scores_out=None, stream=None):
        """qwin [Hq, W, d], k [Hkv, N, d] of one layer; returns S [Hkv, N]
        when scores_out is given or requested (pass True)."""
        N = k.shape[1]
        if scores_out is True:
            scores_out = _empty((self.ctx.kv_heads, N), torch.float32, k.device, stream)
        _check(load().bacon_score_layer(self.ctx.handle, self.handle, layer, qwin.data_ptr(),
                                        k.data_ptr(), N, _ptr(scores_out), _stream_ptr(stream)))
        return scores_out

    def select(self, budget, N, idx_out=None, stream=None, device="cuda"):
        kept = min(budget, N)
        if idx_out is None:
            idx_out = _empty((self.ctx.kv_heads, kept), torch.int32, device, stream)
        _check(load().bacon_select(self.ctx.handle, self.handle, budget, idx_out.data_ptr(),
                                   _stream_ptr(stream)))
        return idx_out


_i32 = torch.int32


class Cache:
    """Kept rows and the tokens after them in pages of 8-bit values
    (``bacon_cache``): block tables, storing, and attention over them.

    A unit is one (request, layer, kv-head).  Per-unit arrays are int32 on the
    GPU: lengths [R, layers, kv_heads], table [R, layers, kv_heads,
    max_blocks]; ring [pages] and state [2] hold the free pages.  The pools
    k, v [pages, page, head_dim] uint8 and their scales [pages] fp32 may be
    given, else they are allocated here.  The cache lives on the pools' device,
    and so must everything that its calls are given.  A call on another stream
    than the current one (stream=) runs when that stream gets to it: its inputs
    have to be complete there, and are the caller's to keep until it has run."""

    def __init__(self, layers, kv_heads, q_heads, head_dim, pages, page=64, format="e4m3",
                 dtype=torch.bfloat16, max_requests=4, max_blocks=None, k=None, v=None,
                 k_scale=None, v_scale=None):
        lib = load()
        if format not in CACHE_FORMATS or dtype not in CACHE_DTYPES:
            raise ValueError("format must be e4m3 or int8, dtype bfloat16 or float16")
        self.layers, self.kv_heads, self.q_heads = layers, kv_heads, q_heads
        self.head_dim, self.pages, self.page = head_dim, pages, page
        self.format, self.dtype = format, dtype
        self.max_requests = max_requests
        self.max_blocks = (min(pages, ((1 << 31) - 1025) // page) if max_blocks is None
                           else max_blocks)
        codes, scales = (pages, page, head_dim), (pages,)
        given = [t for t in (k, v, k_scale, v_scale) if t is not None]
        self.device = given[0].device if given else torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.k, self.v = (torch.empty(codes, dtype=torch.uint8, device=self.device) if t is None
                          else t for t in (k, v))
        self.k_scale, self.v_scale = (torch.empty(scales, device=self.device) if t is None else t
                                      for t in (k_scale, v_scale))
        for t, shape, kind in ((self.k, codes, torch.uint8), (self.v, codes, torch.uint8),
                               (self.k_scale, scales, torch.float32),
                               (self.v_scale, scales, torch.float32)):
            if not t.is_cuda or not self._fits(t, shape, kind):
                raise ValueError(f"the pools must be on one GPU, contiguous, and this one {kind} of "
                                 f"shape {shape}")
        desc = CacheDesc(layers, kv_heads, q_heads, head_dim, page, pages, max_requests,
                         self.max_blocks, CACHE_FORMATS[format], CACHE_DTYPES[dtype],
                         self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(),
                         self.v_scale.data_ptr())
        h = _vp()
        with torch.cuda.device(self.device):
            _check(lib.bacon_cache_create(ctypes.byref(h), ctypes.byref(desc)))
        self.handle, self._lib = h, lib
        self._unit, self._row = (layers, kv_heads), (layers, kv_heads, self.max_blocks)

    def _fits(self, t, shape, dtype):
        """Whether a tensor is contiguous, of this shape and type, on the cache's device."""
        return (t.dtype is dtype and t.shape == shape and t.get_device() == self._index
                and t.is_contiguous())

    def _int32(self, t, shape, what):
        """The address of a contiguous int32 tensor of this shape."""
        if self._fits(t, shape, _i32):
            return t.data_ptr()
        raise ValueError(f"{what} must be a contiguous int32 tensor of shape {tuple(shape)} on "
                         f"{self.device}")

    def _stream(self, stream):
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        if getattr(stream, "device_index", self._index) != self._index:
            raise ValueError(f"the stream must be one of {self.device}")
        return stream.cuda_stream

    def close(self):
        if getattr(self, "handle", None):
            self._lib.bacon_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def sync(self, stream=None):
        _check(self._lib.bacon_cache_sync(self.handle, self._stream(stream)))

    def tables(self, requests):
        """(lengths, table, ring, state) of `requests` empty requests: every
        page is free."""
        shape = (requests, self.layers, self.kv_heads)
        dev = self.k.device
        return (torch.zeros(shape, dtype=torch.int32, device=dev),
                torch.full(shape + (self.max_blocks,), -1, dtype=torch.int32, device=dev),
                torch.arange(self.pages, dtype=torch.int32, device=dev),
                torch.tensor([0, self.pages], dtype=torch.int32, device=dev))

    def plan(self, lengths, added, table, ring, state, rows, slots=None, lengths_out=None,
             state_out=None, stream=None):
        """Pages and slots for the tokens the units are about to get.  added
        [R, layers, kv_heads]: each unit its own number, slots [rows] in the
        units' order (that of compress_adaptive's rows); added [R] or None
        (one): tokens of a request, slots [layers, rows, kv_heads].  rows: the
        tokens in all.  The table gets the new pages; returns (slots,
        lengths_out, state_out)."""
        R = lengths.shape[0]
        units = (R,) + self._unit
        per_unit = added is not None and added.dim() == 3
        shape = (rows,) if per_unit else (self.layers, rows, self.kv_heads)
        p_lengths, p_state = self._int32(lengths, units, "lengths"), self._int32(state, (2,), "state")
        if slots is None:
            slots = _empty(shape, _i32, self.device, stream)
        if lengths_out is None:
            lengths_out = _empty(units, _i32, self.device, stream)
        if state_out is None:
            state_out = _empty((2,), _i32, self.device, stream)
        _check(self._lib.bacon_cache_plan(
            self.handle, R, p_lengths,
            None if added is None else self._int32(added, units if per_unit else (R,), "added"),
            per_unit, self._int32(table, (R,) + self._row, "table"),
            self._int32(ring, (self.pages,), "ring"), p_state, rows, self._int32(slots, shape, "slots"),
            self._int32(lengths_out, units, "lengths_out"), self._int32(state_out, (2,), "state_out"),
            self._stream(stream)))
        return slots, lengths_out, state_out

    def locate(self, count, table, rows, first=None, slots=None, stream=None):
        """Slots [rows] of the positions [first, first + count) of each unit
        (first None: 0), the units one after the other; -1 beyond them."""
        R = count.shape[0]
        units = (R,) + self._unit
        if slots is None:
            slots = _empty((rows,), _i32, self.device, stream)
        _check(self._lib.bacon_cache_locate(
            self.handle, R, None if first is None else self._int32(first, units, "first"),
            self._int32(count, units, "count"), self._int32(table, (R,) + self._row, "table"),
            rows, self._int32(slots, (rows,), "slots"), self._stream(stream)))
        return slots

    def release(self, done, lengths, table, ring, state, stream=None):
        """Gives the pages of the requests with done [R] != 0 back, in place."""
        R = lengths.shape[0]
        units = (R,) + self._unit
        _check(self._lib.bacon_cache_release(
            self.handle, R, self._int32(done, (R,), "done"), self._int32(lengths, units, "lengths"),
            self._int32(table, (R,) + self._row, "table"),
            self._int32(ring, (self.pages,), "ring"), self._int32(state, (2,), "state"),
            self._stream(stream)))

    def shorten(self, fewer, lengths, table, ring, state, stream=None):
        """Takes the last fewer[r] tokens (fewer [R]; rejected drafts, say) of
        every unit of request r back, and gives the pages that held no other
        back, in place."""
        R = lengths.shape[0]
        units = (R,) + self._unit
        _check(self._lib.bacon_cache_shorten(
            self.handle, R, self._int32(fewer, (R,), "fewer"), self._int32(lengths, units, "lengths"),
            self._int32(table, (R,) + self._row, "table"),
            self._int32(ring, (self.pages,), "ring"), self._int32(state, (2,), "state"),
            self._stream(stream)))

    def _rows(self, t, what):
        """(address, token stride, head stride) of rows [T, H, d] or [T, d]."""
        stride = t.stride()
        if (t.dtype is not self.dtype or t.get_device() != self._index
                or t.shape[-1] != self.head_dim or len(stride) not in (2, 3) or stride[-1] != 1):
            raise ValueError(f"{what} must be {self.dtype} rows of {self.head_dim} values on "
                             f"{self.device}, [tokens, heads, d] or [tokens, d], the last "
                             "dimension contiguous")
        return t.data_ptr(), stride[0], stride[1] if len(stride) == 3 else 0

    def store(self, k, v, slots, stream=None):
        """Rows k, v [T, H, d] (slots [T, H]) or [T, d] (slots [T]) into their
        slots; any strides with contiguous rows."""
        if k.shape != v.shape:
            raise ValueError("k and v must have the same shape")
        kp, vp = self._rows(k, "k"), self._rows(v, "v")
        _check(self._lib.bacon_cache_store(
            self.handle, k.shape[0], k.shape[1] if k.dim() == 3 else 1, *kp, *vp,
            self._int32(slots, k.shape[:-1], "slots"), self._stream(stream)))

    def store_rotated(self, rotary, q, k, v, positions, slots, q_weight=None, k_weight=None,
                      eps=1e-6, offset=0.0, q_out=None, stream=None):
        """``rotary.apply`` to q [T, Hq, d] (may be None) and k [T, H, d], and
        ``store`` of the turned k and of v, in one launch with the same results:
        positions int32 [T] (or [3, T]), slots [T, H].  Returns the turned q."""
        if k.shape != v.shape or k.dim() != 3:
            raise ValueError("k and v must have the same shape [tokens, heads, d]")
        T = k.shape[0]
        kp, vp = self._rows(k, "k"), self._rows(v, "v")
        weights = _weights_dtype((q_weight, k_weight), (self.head_dim,), self.dtype, self._index)
        rows = None
        if q is not None:
            qp = self._rows(q, "q")
            if q.dim() != 3 or q.shape[0] != T:
                raise ValueError("q must be [tokens, heads, d], of k's tokens")
            if q_out is None:
                q_out = _empty(q.shape, self.dtype, self.device, stream)
                op = q_out.data_ptr(), q.shape[1] * self.head_dim, self.head_dim
            elif q_out.shape != q.shape:
                raise ValueError("q_out must have q's shape")
            else:
                op = self._rows(q_out, "q_out")
            rows = _pack_rows(qp[0], op[0], _ptr(q_weight) or 0, q.shape[1], 0, qp[1], qp[2], 0,
                              op[1], op[2])
        _check(self._lib.bacon_cache_store_rotated(
            self.handle, rotary.handle, T, rows,
            _pack_rows(kp[0], 0, _ptr(k_weight) or 0, k.shape[1], 0, kp[1], kp[2], 0, 0, 0), *vp,
            weights, eps, offset, self._int32(positions, rotary.shape(T), "positions"),
            self._int32(slots, k.shape[:-1], "slots"), self._stream(stream)))
        return q_out

    def load(self, slots, k_out=None, v_out=None, stream=None):
        """The values of the slots' rows, shape [*slots.shape, d] each."""
        shape = slots.shape + (self.head_dim,)
        if k_out is None:
            k_out = _empty(shape, self.dtype, self.device, stream)
        if v_out is None:
            v_out = _empty(shape, self.dtype, self.device, stream)
        for t in (k_out, v_out):
            if not self._fits(t, shape, self.dtype):
                raise ValueError(f"outputs must be contiguous {self.dtype} of shape {tuple(shape)} "
                                 f"on {self.device}")
        _check(self._lib.bacon_cache_load(self.handle, slots.numel(),
                                          self._int32(slots, slots.shape, "slots"), k_out.data_ptr(),
                                          v_out.data_ptr(), self._stream(stream)))
        return k_out, v_out

    def attend(self, layer, q, lengths, table, starts=None, causal=True, scale=None, out=None,
               lse=None, stream=None):
        """Attention of the queries q [T, q_heads, d] of one layer's new tokens
        (already stored) over their units.  starts [R + 1] int32: where each
        request's queries begin; None: T / R each.  Returns out [T, q_heads,
        d], with lse=True (or a tensor) also the log-sum-exp [T, q_heads]."""
        R, shape = lengths.shape[0], q.shape
        if len(shape) != 3 or shape[1] != self.q_heads:
            raise ValueError(f"q must be [tokens, {self.q_heads}, {self.head_dim}]")
        qp = self._rows(q, "q")
        if out is None:
            out = _empty(shape, self.dtype, self.device, stream)
        elif not self._fits(out, shape, self.dtype):
            raise ValueError(f"out must be contiguous, of q's shape and type, on {self.device}")
        if lse is True:
            lse = _empty(shape[:2], torch.float32, self.device, stream)
        elif lse is not None and not self._fits(lse, shape[:2], torch.float32):
            raise ValueError(f"lse must be contiguous float32 [tokens, q_heads] on {self.device}")
        _check(self._lib.bacon_cache_attend(
            self.handle, R, layer, shape[0], *qp,
            None if starts is None else self._int32(starts, (R + 1,), "starts"),
            self._int32(lengths, (R,) + self._unit, "lengths"),
            self._int32(table, (R,) + self._row, "table"), bool(causal),
            0.0 if scale is None else scale, out.data_ptr(), _ptr(lse), self._stream(stream)))
        return out if lse is None else (out, lse)


# ------------------------------------------------------------------------
# a token between its matrix products and the cache

_device = torch._C._cuda_getDevice


def _on(index, call, *args):
    """A call of the library with device `index` current."""
    if _device() == index:
        _check(call(*args))
    else:
        with torch.cuda.device(index):
            _check(call(*args))


def _stream_of(stream, index):
    """The address of a stream of device `index` (None: its current one)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index)
    if getattr(stream, "device_index", index) != index:
        raise ValueError(f"the stream must be one of cuda:{index}")
    return stream.cuda_stream


def _weights_dtype(weights, shape, dtype, index):
    """The type of the weights that there are: the rows' or float32, one for all."""
    kind = None
    for w in weights:
        if w is None:
            continue
        if (w.shape != shape or w.get_device() != index or not w.is_contiguous()
                or w.dtype is not (kind or w.dtype) or w.dtype not in (dtype, torch.float32)):
            raise ValueError(f"weights must be contiguous, of shape {tuple(shape)}, all {dtype} or "
                             f"all float32, on cuda:{index}")
        if not w.data_ptr():  # its storage was freed; NULL would mean that there is no weight
            raise ValueError("a weight has no memory")
        kind = w.dtype
    return DTYPES[kind or dtype]


class Rotary:
    """Rotary positions of rows of `head_dim` values (``bacon_rotary``).

    The first `rotary_dim` values (None: all) turn, in pairs (i, i + half) or
    interleaved (2i, 2i + 1).  Frequencies: base^(-2i / rotary_dim), with
    `scaling` "linear" (by `factor`), "base" (the base grows), "rotations" or
    "dims" (pairs that turn fewer than `low` times over `original` positions are
    scaled, those that turn more than `high` times are not); or the caller's
    `frequencies` (rotary_dim / 2 radians a position).  `axes`: for each pair the
    position axis 0, 1 or 2 that it turns with (e.g. time, height, width); None:
    one axis.  Host memory only: a handle serves every device."""

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, interleaved=False, scaling=None,
                 factor=1.0, original=0, low=1.0, high=32.0, amplitude=1.0, frequencies=None,
                 axes=None):
        self._lib = load()
        self.head_dim = head_dim
        self.rotary_dim = head_dim if rotary_dim is None else rotary_dim
        half = self.rotary_dim // 2
        table = (ctypes.c_double * max(half, 1))()
        if frequencies is not None:
            if len(frequencies) != half:
                raise ValueError(f"{half} frequencies are needed")
            table[:half] = [float(f) for f in frequencies]
        else:
            if scaling not in ROPE_SCALINGS:
                raise ValueError(f"scaling must be one of {list(ROPE_SCALINGS)}")
            _check(self._lib.bacon_rotary_frequencies(self.rotary_dim, base, ROPE_SCALINGS[scaling],
                                                      factor, original, low, high, table))
        self.frequencies = list(table)[:half]
        if axes is not None and (len(axes) != half or not all(x in (0, 1, 2) for x in axes)):
            raise ValueError(f"axes must be {half} numbers in 0, 1, 2")
        self.axes = 1 if axes is None else 3
        h = _vp()
        _check(self._lib.bacon_rotary_create(ctypes.byref(h), head_dim, self.rotary_dim,
                                             int(interleaved), amplitude, table,
                                             None if axes is None else bytes([int(x) for x in axes])))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            self._lib.bacon_rotary_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def shape(self, *tokens):
        """The shape of the positions of tokens of this shape."""
        return tokens if self.axes == 1 else (3,) + tokens

    def _rows(self, t, out, weight, dtype, index, places, stream, what):
        """Packed rows and the output (allocated if None)."""
        shape, stride = t.shape, t.stride()
        if (t.dtype is not dtype or t.get_device() != index or shape[:-2] != places
                or shape[-1] != self.head_dim or (stride[-1] != 1 and t.numel())):
            raise ValueError(f"{what} must be {dtype} rows of {self.head_dim} values on cuda:{index}, "
                             "[tokens, heads, d] or [requests, tokens, heads, d] like the other, "
                             "the last dimension contiguous")
        if out is None:
            out = _empty(shape, dtype, t.device, stream)
        elif (out.dtype is not dtype or out.get_device() != index or out.shape != shape
              or (out.stride(-1) != 1 and t.numel())):
            raise ValueError(f"the output of {what} must have its shape, type and device, the last "
                             "dimension contiguous")
        to = out.stride()
        if len(stride) == 4:
            return out, _pack_rows(t.data_ptr(), out.data_ptr(), 0 if weight is None else weight.data_ptr(),
                                   shape[2], *stride[:3], *to[:3])
        return out, _pack_rows(t.data_ptr(), out.data_ptr(), 0 if weight is None else weight.data_ptr(),
                               shape[1], 0, stride[0], stride[1], 0, to[0], to[1])

    def apply(self, q, k, positions, q_weight=None, k_weight=None, eps=1e-6, offset=0.0,
              transposed=False, q_out=None, k_out=None, stream=None):
        """Positions into q [T, Hq, d] and k [T, H, d], or [R, N, Hq, d] and
        [R, N, H, d], bf16, fp16 or fp32 of any strides with contiguous rows
        (either may be None); positions int32, contiguous, [T] or [R, N], with a
        leading dimension of 3 when there are axes.  With q_weight or k_weight [d]
        a row is first divided by its root mean square (`eps`) and multiplied by
        offset + weight.  transposed: by the negative angles, the call's gradient
        and, for amplitude 1, its inverse.  Outputs may be the inputs, or views
        such as k_out.transpose(1, 2) of head-major rows.  Returns (q_out,
        k_out)."""
        t = k if q is None else q
        if t is None or not t.is_cuda or t.dim() not in (3, 4) or t.dtype not in DTYPES:
            raise ValueError("q or k must be bf16, fp16 or fp32 rows on a GPU, [tokens, heads, d] or "
                             "[requests, tokens, heads, d]")
        dtype, index, places = t.dtype, t.get_device(), t.shape[:-2]
        kind = weights = DTYPES[dtype]
        if q_weight is not None or k_weight is not None:
            weights = _weights_dtype((q_weight, k_weight), (self.head_dim,), dtype, index)
        rows = [None, None]
        if q is not None:
            q_out, rows[0] = self._rows(q, q_out, q_weight, dtype, index, places, stream, "q")
        if k is not None:
            k_out, rows[1] = self._rows(k, k_out, k_weight, dtype, index, places, stream, "k")
        if (positions.dtype is not _i32
                or positions.shape != (places if self.axes == 1 else (3,) + places)
                or positions.get_device() != index or not positions.is_contiguous()):
            raise ValueError("positions must be a contiguous int32 tensor of shape "
                             f"{tuple(self.shape(*places))} on cuda:{index}")
        _on(index, self._lib.bacon_rotary_apply, self.handle, places[0] if len(places) == 2 else 1,
            places[-1], *rows, kind, weights, eps, offset, transposed, positions.data_ptr(),
            _stream_of(stream, index))
        return q_out, k_out


class BlockNorm:
    """What lies between two blocks of `width` channels (``bacon_block_norm``):
    a = post(y) gate(g), s = x + scale a, n = pre(s).

    post, pre: None, "rms" or "layer", with weights and biases [width] (any may be
    None) in the rows' type or float32; eps is both norms', and both multiply by
    offset + weight.  gate: "linear", "sigmoid", "tanh" or "silu", of the gate that
    a call gives.  The object holds the tensors of the weights, and each call reads what
    they are then; it may be used from several threads and streams."""

    def __init__(self, width, pre="rms", post=None, pre_weight=None, pre_bias=None,
                 post_weight=None, post_bias=None, gate="linear", scale=1.0, eps=1e-6, offset=0.0):
        if pre not in NORMS or post not in NORMS or gate not in GATES:
            raise ValueError(f"norms must be of {list(NORMS)}, gate of {list(GATES)}")
        self._lib = load()
        self.width, self.pre, self.post = width, pre, post
        self._kinds = NORMS[post], NORMS[pre], GATES[gate], scale, eps, offset
        self._weights = post_weight, post_bias, pre_weight, pre_bias
        self._given = [(i, w) for i, w in enumerate(self._weights) if w is not None]
        if not all(w.is_cuda for _, w in self._given):
            raise ValueError("weights must be on a GPU")
        self._shape = torch.Size((width,))

    def _bound(self, dtype, index):
        """The type and places of the weights, as they are now: a parameter may have got
        other data since the last call."""
        places, shape, first = [0, 0, 0, 0], self._shape, self._given[0][1].dtype
        for i, w in self._given:
            at = w.data_ptr()
            if (w.dtype is not first or w.shape != shape or w.get_device() != index or not at
                    or not w.is_contiguous()):
                break
            places[i] = at
        else:
            if first is dtype or first is torch.float32:
                return DTYPES[first], places
        kind = _weights_dtype(self._weights, shape, dtype, index)  # says what is wrong
        return kind, [_ptr(w) or 0 for w in self._weights]

    def _rows(self, t, shape, dtypes, index, what, one):
        """The distance of rows [..., width], with the last dimension contiguous
        and one distance for all rows; `one`: of a single row among others."""
        if t.dtype not in dtypes or t.get_device() != index or t.shape != shape:
            raise ValueError(f"{what} must be of shape {tuple(shape)} and one of {dtypes} on "
                             f"cuda:{index}")
        if t.is_contiguous():
            return t.stride()[-2] if one else self.width
        return self._distance(t, what)

    def _distance(self, t, what):
        shape, stride = t.shape, t.stride()
        if stride[-1] == 1 or self.width == 1:
            flat = [(n, s) for n, s in zip(shape[:-1], stride[:-1]) if n > 1]
            if all(s == n * r for (_, s), (n, r) in zip(flat, flat[1:])):
                return flat[-1][1] if flat else self.width
        raise ValueError(f"the rows of {what} must be contiguous, and the same distance apart")

    def __call__(self, y, x=None, gate=None, sum_out=None, norm_out=None, stream=None):
        """y [..., width]; x (the residual) of its shape, in its type or float32;
        gate of its type: [width], [..., 1] or [..., width].  Returns (sum, normed):
        the sum in x's type (None for a norm alone: without x, post and gate), normed
        in y's (None without a pre norm).  sum_out may be x, norm_out y."""
        shape, dtype, width = y.shape, y.dtype, self.width
        index = y.get_device()
        if not y.is_cuda or len(shape) < 1 or shape[-1] != width:
            raise ValueError(f"y must be [..., {width}] on a GPU")
        kind = weight_kind = wide_kind = DTYPES.get(dtype)
        if kind is None:
            raise ValueError("rows must be bf16, fp16 or fp32")
        weights = 0, 0, 0, 0
        if self._given:
            weight_kind, weights = self._bound(dtype, index)
        tokens = y.numel() // width
        one = tokens == 1 and len(shape) > 1
        if y.is_contiguous():
            y_stride = y.stride()[-2] if one else width
        else:
            y_stride = self._distance(y, "y")
        gate_stride = x_stride = sum_stride = norm_stride = 0
        wide = x if x is not None else sum_out
        residual = dtype if wide is None else wide.dtype
        if x is not None:
            x_stride = self._rows(x, shape, (dtype, torch.float32), index, "x", one)
        channel = 0
        if gate is not None:
            g = gate.shape
            if gate.dtype is not dtype or gate.get_device() != index:
                raise ValueError("the gate must have y's type and device")
            if g == shape:
                channel = 1
                gate_stride = self._rows(gate, shape, (dtype,), index, "gate", one)
            elif g == (width,) and gate.is_contiguous():
                channel = 1
            elif g == shape[:-1] + (1,) and gate.is_contiguous():
                gate_stride = 1
            else:
                raise ValueError(f"the gate must be contiguous [{width}] or {tuple(shape[:-1])} + "
                                 "(1,), or have y's shape")
        if sum_out is not None:
            sum_stride = self._rows(sum_out, shape, (residual,) if x is not None else
                                    (dtype, torch.float32), index, "sum_out", one)
        elif x is not None or self.post is not None or gate is not None:
            sum_out = _empty(shape, residual, y.device, stream)
            sum_stride = width
        if self.pre is None:
            if norm_out is not None:
                raise ValueError("there is no pre norm")
        elif norm_out is None:
            norm_out = _empty(shape, dtype, y.device, stream)
            norm_stride = width
        else:
            norm_stride = self._rows(norm_out, shape, (dtype,), index, "norm_out", one)
        if residual is not dtype:
            wide_kind = DTYPES[residual]
        post, pre, activation, scale, eps, offset = self._kinds
        desc = _pack_block(tokens, width, kind, wide_kind, weight_kind, post, pre, activation,
                           scale, eps, offset, channel, gate_stride, y_stride, x_stride,
                           sum_stride, norm_stride, y.data_ptr(), 0 if x is None else x.data_ptr(),
                           0 if gate is None else gate.data_ptr(), *weights,
                           0 if sum_out is None else sum_out.data_ptr(),
                           0 if norm_out is None else norm_out.data_ptr())
        at = _stream_of(stream, index)
        if _device() == index:
            _check(self._lib.bacon_block_norm(desc, at))
        else:
            _on(index, self._lib.bacon_block_norm, desc, at)
        return sum_out, norm_out


class Logits:
    """Rules on rows of `vocab` logits (``bacon_logits``), on the current device or
    `device`: penalties, biases, masks, temperature, and the greedy token."""

    def __init__(self, vocab, device=None):
        self._lib = load()
        self.vocab = vocab
        index = None if device is None else torch.device(device).index
        self.device = torch.device("cuda", torch.cuda.current_device() if index is None else index)
        self._index = self.device.index
        h = _vp()
        with torch.cuda.device(self.device):
            _check(self._lib.bacon_logits_create(ctypes.byref(h), vocab))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            self._lib.bacon_logits_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def sync(self, stream=None):
        _check(self._lib.bacon_logits_sync(self.handle, _stream_of(stream, self._index)))

    def _fits(self, t, shape, dtype, what):
        """The address of a contiguous tensor of this shape and type, 0 for None."""
        if t is None:
            return 0
        if (t.dtype is dtype and t.shape == shape and t.get_device() == self._index
                and t.is_contiguous()):
            return t.data_ptr()
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"{self.device}")

    def _lines(self, t, dtypes, rows, least, what):
        """(address, stride) of [rows, ...] of at least `least` values, each row
        contiguous; a row may be shared (stride 0) where that is read only."""
        if (t.dim() != 2 or t.dtype not in dtypes or t.get_device() != self._index
                or t.shape[0] != rows or t.shape[1] < least or (t.shape[1] > 1 and t.stride(1) != 1)):
            raise ValueError(f"{what} must be [{rows}, {least}], of {dtypes}, on {self.device}, each "
                             "row contiguous")
        return t.data_ptr(), t.stride(0)

    def process(self, logits, tokens=None, lengths=None, prompt=None, request=None,
                repetition=None, frequency=None, presence=None, temperature=None,
                bias_tokens=None, bias_values=None, mask=None, out=None, greedy=True, stream=None):
        """logits [rows, vocab] in bf16, fp16 or fp32.  History: tokens int32
        [requests, capacity]; of line request[row] (None: the row's own) the first
        lengths[row] entries, the first prompt[row] of them (None: 0) the prompt; a
        row of length -1 is left out.  repetition, frequency, presence, temperature:
        float32 [rows].  bias_tokens int32, bias_values float32 [rows, n] (-1:
        unused).  mask int32 [rows or 1, ceil(vocab / 32)], a bit for each token
        that is allowed.  out: None (a new float32 tensor), False (not wanted), or a
        tensor in float32 or the logits' type, the logits themselves too.  Returns
        (out, best, logprob, lse), the last three [rows] or, without `greedy`,
        None."""
        if logits.dim() != 2 or logits.shape[1] != self.vocab:
            raise ValueError(f"logits must be [rows, {self.vocab}]")
        rows, dtype = logits.shape[0], logits.dtype
        p_logits, stride = self._lines(logits, DTYPES, rows, self.vocab, "logits")
        p_out = out_stride = 0
        out_dtype = torch.float32
        if out is None:
            out = _empty((rows, self.vocab), torch.float32, self.device, stream)
            p_out, out_stride = out.data_ptr(), self.vocab
        elif out is False:
            out = None
        else:
            if out.shape != logits.shape:
                raise ValueError("out must have the logits' shape")
            out_dtype = out.dtype
            p_out, out_stride = self._lines(out, (dtype, torch.float32), rows, self.vocab, "out")
        each = (rows,)
        requests = capacity = token_stride = p_tokens = 0
        if tokens is not None:
            requests, capacity = tokens.shape
            p_tokens, token_stride = self._lines(tokens, (_i32,), requests, 0, "tokens")
            if not p_tokens:
                # no entries have no address, and without one lengths would not be looked at;
                # nobody follows this one
                p_tokens, requests, capacity = 16, max(1, requests), 0
        biases = p_bias = p_value = 0
        if bias_tokens is not None and bias_values is not None:
            biases = bias_tokens.shape[-1]
            p_bias = self._fits(bias_tokens, (rows, biases), _i32, "bias_tokens")
            p_value = self._fits(bias_values, (rows, biases), torch.float32, "bias_values")
        elif bias_tokens is not None or bias_values is not None:
            raise ValueError("bias_tokens and bias_values come together")
        p_mask = mask_stride = 0
        if mask is not None:
            one = mask.dim() == 2 and mask.shape[0] == 1
            p_mask, mask_stride = self._lines(mask, (_i32,), 1 if one else rows,
                                              -(-self.vocab // 32), "mask")
            if one:
                mask_stride = 0
        best = logprob = lse = None
        if greedy:
            best = _empty(each, _i32, self.device, stream)
            logprob = _empty(each, torch.float32, self.device, stream)
            lse = _empty(each, torch.float32, self.device, stream)
        f32, fits = torch.float32, self._fits
        desc = _pack_logits(
            rows, DTYPES[dtype], DTYPES[out_dtype], requests, capacity, biases, stride, out_stride,
            token_stride, mask_stride, p_logits, p_out, p_tokens, fits(request, each, _i32, "request"),
            fits(prompt, each, _i32, "prompt"), fits(lengths, each, _i32, "lengths"),
            fits(repetition, each, f32, "repetition"), fits(frequency, each, f32, "frequency"),
            fits(presence, each, f32, "presence"), fits(temperature, each, f32, "temperature"),
            p_bias, p_value, p_mask, _ptr(best) or 0, _ptr(logprob) or 0, _ptr(lse) or 0)
        _check(self._lib.bacon_logits_process(self.handle, desc, _stream_of(stream, self._index)))
        return out, best, logprob, lse
