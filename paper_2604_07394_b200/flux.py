"""ctypes binding of ``libflux_attn.so`` -- argument marshalling only.

Every function named ``flux_*`` forwards to the C entry point of the same name
(declared in ``include/flux_attn.h``).  :class:`Plan` wraps them for torch
tensors: it passes ``data_ptr()`` and the current CUDA stream, nothing else.
There is no fallback: if the library is missing or a call fails, an exception
is raised.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflux_attn.so")

FLUX_OK = 0
FLUX_E_INVALID_ARG = -1
FLUX_E_UNSUPPORTED_SHAPE = -2
FLUX_E_CAPACITY = -3
FLUX_E_WORKSPACE = -4
FLUX_E_DEVICE_TIMEOUT = -5
FLUX_E_CUDA = -6
FLUX_E_DEVICE_FLAG = -7

FLUX_STATUS_BAD_MASK = 1
FLUX_STATUS_NAN_LOGIT = 2
FLUX_STATUS_BAD_LENGTH = 4
FLUX_STATUS_WAIT_EXPIRED = 8
FLUX_STATUS_NONFINITE = 16
FLUX_STATUS_BAD_POINTER = 32

FLUX_KERNEL_DECODE = 0
FLUX_KERNEL_PREFILL = 1

FLUX_DECODE_AUTO = 0
FLUX_DECODE_TWO_LAUNCH = 1
FLUX_DECODE_SINGLE_LAUNCH = 2

FLUX_KVQ_E4M3 = 0
FLUX_KVQ_INT8 = 1

FLUX_KV_FULL = 0
FLUX_KV_COMPACT_SA = 1

EXPORTS = [
    "flux_plan_create", "flux_plan_destroy", "flux_workspace_size", "flux_plan_set_workspace",
    "flux_router_apply", "flux_router_forward", "flux_attn_prefill", "flux_attn_prefill_blocks", "flux_kv_retain", "flux_kv_append",
    "flux_attn_prefill_packed", "flux_kvq_cache_size", "flux_kvq_store", "flux_kvq_load", "flux_attn_decode_kvq", "flux_attn_decode_step_kvq",
    "flux_attn_decode", "flux_attn_decode_heads", "flux_attn_decode_partial", "flux_attn_combine", "flux_attn_decode_partial_push", "flux_attn_combine_wait", "flux_attn_decode_step", "flux_attn_decode_noalloc", "flux_attn_decode_host", "flux_attn_prefill_host", "flux_plan_status",
    "flux_debug_dispatch", "flux_debug_touched", "flux_debug_decode_kernel", "flux_plan_set_launch_overlap", "flux_debug_wait_probe", "flux_profile_enable", "flux_profile_read", "flux_launch_count", "flux_last_error", "flux_version",
]


class FluxConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("sink", ctypes.c_int32), ("window", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("max_batch", ctypes.c_int32),
        ("max_context", ctypes.c_int32), ("kv_layout", ctypes.c_int32),
    ]


class FluxRouterWeights(ctypes.Structure):
    _fields_ = [
        ("enc_dim", ctypes.c_int32), ("head_hidden", ctypes.c_int32),
        ("w_enc1", ctypes.c_void_p), ("b_enc1", ctypes.c_void_p),
        ("w_enc2", ctypes.c_void_p), ("b_enc2", ctypes.c_void_p),
        ("w_head1", ctypes.c_void_p), ("b_head1", ctypes.c_void_p),
        ("w_head2", ctypes.c_void_p), ("b_head2", ctypes.c_void_p),
    ]


class PeerSet(ctypes.Structure):
    _fields_ = [
        ("world", ctypes.c_int32), ("rank", ctypes.c_int32),
        ("gather_o", ctypes.c_void_p * 8), ("gather_ml", ctypes.c_void_p * 8), ("flags", ctypes.c_void_p * 8),
    ]


class FluxError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("flux_attn error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load():
    """Load the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            LIB_PATH + " is missing: build it with `python -m paper_2604_07394_b200.build` "
            "(there is no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cfgp = ctypes.POINTER(FluxConfig)
    L.flux_plan_create.argtypes = [cfgp, ctypes.POINTER(vp)]
    L.flux_plan_destroy.argtypes = [vp]
    L.flux_workspace_size.argtypes = [cfgp, ctypes.POINTER(sz)]
    L.flux_plan_set_workspace.argtypes = [vp, vp, sz]
    L.flux_router_apply.argtypes = [vp, vp, vp, i32, vp, vp]
    L.flux_router_forward.argtypes = [vp, ctypes.POINTER(FluxRouterWeights), vp, i32, vp, i32, vp, vp]
    L.flux_attn_prefill.argtypes = [vp, i32, i32, vp, vp, vp, i32, i32, vp, vp]
    L.flux_attn_prefill_blocks.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, vp]
    L.flux_kv_retain.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, vp]
    L.flux_kv_append.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    L.flux_attn_decode.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    L.flux_attn_decode_partial.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.flux_attn_combine.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    L.flux_attn_decode_partial_push.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, ctypes.c_uint32, vp]
    L.flux_attn_combine_wait.argtypes = [vp, i32, i32, vp, vp, vp, ctypes.c_uint32, ctypes.c_int64, vp, vp]
    L.flux_attn_decode_heads.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp]
    L.flux_attn_decode_step.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.flux_attn_decode_noalloc.argtypes = [cfgp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.flux_attn_decode_host.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.flux_attn_prefill_host.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp]
    L.flux_attn_prefill_packed.argtypes = [vp, i32, i32, vp, vp, vp, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, vp, vp, vp, vp]
    L.flux_kvq_cache_size.argtypes = [cfgp, i32, i32, ctypes.POINTER(sz)]
    L.flux_kvq_store.argtypes = [vp, i32, i32, i32, vp, vp, ctypes.c_int64, ctypes.c_int64, i32, vp, vp, vp, vp, vp]
    L.flux_kvq_load.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    L.flux_attn_decode_kvq.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    L.flux_attn_decode_step_kvq.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.flux_plan_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32), vp]
    L.flux_debug_dispatch.argtypes = [vp, vp, i32, ctypes.POINTER(i32), vp]
    L.flux_debug_decode_kernel.argtypes = [vp, i32]
    L.flux_plan_set_launch_overlap.argtypes = [vp, i32]
    L.flux_debug_touched.argtypes = [vp, vp, i32]
    L.flux_debug_wait_probe.argtypes = [vp, ctypes.c_int64, vp]
    L.flux_profile_enable.argtypes = [vp, i32]
    L.flux_profile_read.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_int64), vp]
    L.flux_launch_count.argtypes = [vp]
    L.flux_launch_count.restype = ctypes.c_int64
    L.flux_last_error.restype = ctypes.c_char_p
    L.flux_version.restype = ctypes.c_char_p
    for name in EXPORTS:
        fn = getattr(L, name)
        if name not in ("flux_launch_count", "flux_last_error", "flux_version"):
            fn.restype = ctypes.c_int
    _lib = L
    return L


def last_error() -> str:
    return load().flux_last_error().decode()


def _check(rc: int) -> None:
    if rc != FLUX_OK:
        raise FluxError(rc, last_error())


def _ptr(t):
    """Address of a torch tensor / numpy array / int / None."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return int(t)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _rows(t, heads, what, dev=-1):
    """Row stride in elements of a bf16 tensor [rows][heads][128] on CUDA device dev (-1: in host memory) whose rows are contiguous
    inside (a slice of a wider projection output qualifies); anything else is an error."""
    stride = t.stride()
    if t.dtype is not torch.bfloat16 or t.shape[1:] != (heads, 128) or (stride[1:] != (128, 1) and (heads > 1 or stride[2] != 1)) or t.get_device() != dev:
        raise ValueError("%s: expected bf16 [rows][%d][128] with contiguous rows on cuda:%d, got %s %s with strides %s on %s"
                         % (what, heads, dev, t.dtype, tuple(t.shape), stride, t.device))
    return stride[0] if stride[0] >= heads * 128 or t.shape[0] > 1 else heads * 128


def _flat_rows(t, n, heads, what, dev=-1):
    """Address of a contiguous bf16 tensor of at least n rows [heads][128] on CUDA device dev."""
    if t.dtype is torch.bfloat16 and t.is_contiguous() and t.get_device() == dev:
        shape = t.shape
        if len(shape) == 3 and shape[0] >= n and shape[1] == heads and shape[2] == 128:
            return t.data_ptr()
    raise ValueError("%s: expected contiguous bf16 [%d][%d][128] on cuda:%d, got %s %s with strides %s on %s"
                     % (what, n, heads, dev, t.dtype, tuple(t.shape), t.stride(), t.device))


def _vector(t, n, dtype, what, dev):
    """Address of a contiguous tensor of at least n entries of a type on CUDA device dev."""
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError("%s: expected contiguous %s [%d] on cuda:%d, got %s %s on %s" % (what, dtype, n, dev, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _int32(t, n, what, dev=-1):
    return _vector(t, n, torch.int32, what, dev)


def _table(t, n, what, dev=-1):
    """Address of a table of n device addresses (pointer_table), or an address as it is."""
    if type(t) is torch.Tensor and t.dtype is torch.int64 and t.numel() >= n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    return _vector(t, n, torch.int64, what, dev) if isinstance(t, torch.Tensor) else _ptr(t)


def _bounds(rows, what):
    """Row bounds as a contiguous host array of int32; anything that is not a whole number of that size is an error."""
    rows = np.asarray(rows)
    if rows.dtype != np.int32:
        given = rows
        if given.dtype.kind not in "iu" or (rows := given.astype(np.int32)).tolist() != given.tolist():
            raise ValueError("%s: expected whole numbers below 2^31, got %s %s" % (what, given.dtype, given))
    return np.ascontiguousarray(rows)


def make_config(n_layers, n_q_heads, n_kv_heads, sink, window, max_batch, max_context,
                kv_layout=FLUX_KV_FULL, softmax_scale=0.0, head_dim=128) -> FluxConfig:
    return FluxConfig(n_layers, n_q_heads, n_kv_heads, head_dim, sink, window, softmax_scale,
                      max_batch, max_context, kv_layout)


def flux_workspace_size(cfg: FluxConfig) -> int:
    out = ctypes.c_size_t()
    _check(load().flux_workspace_size(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def flux_kvq_cache_size(cfg: FluxConfig, compact: bool, max_len: int) -> int:
    """Bytes of one 8-bit cache (K or V of one layer and request)."""
    out = ctypes.c_size_t()
    _check(load().flux_kvq_cache_size(ctypes.byref(cfg), 1 if compact else 0, max_len, ctypes.byref(out)))
    return out.value


class Plan:
    """Owns a ``flux_plan`` and the torch-allocated workspace it was given."""

    def __init__(self, cfg: FluxConfig, device="cuda:0"):
        L = load()
        self.cfg = cfg
        self.device = torch.device(device)
        self._index = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self._h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(L.flux_plan_create(ctypes.byref(cfg), ctypes.byref(self._h)))
            nbytes = flux_workspace_size(cfg)
            self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
            self._bf16 = torch.empty(0, dtype=torch.bfloat16, device=self.device)
            _check(L.flux_plan_set_workspace(self._h, self.workspace.data_ptr(), nbytes))
        self.mask = None

    def close(self):
        if self._h:
            load().flux_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self):
        """The stream that is current on the plan's device, as a raw handle (torch.cuda.current_stream().cuda_stream builds a
        Stream object each time: 3 us, as much as the launch)."""
        return torch._C._cuda_getCurrentRawStream(self._index)

    def _tables(self, k_caches, v_caches, B):
        """Addresses of the two pointer tables of a call (a batch beyond the plan's is refused by the call itself)."""
        n, dev = min(B, self.cfg.max_batch), self._index
        return _table(k_caches, n, "k_caches", dev), _table(v_caches, n, "v_caches", dev)

    # -- entry points, same names as the C ABI ------------------------------------------------
    def flux_router_apply(self, logits=None, mask=None, B=None, mask_out=None):
        """logits fp32 [B][L][2] or mask uint8 [B][L] (torch on device, or numpy on host)."""
        src = mask if mask is not None else logits
        if B is None:
            B = int(src.shape[0])
        if mask_out is None:
            mask_out = torch.empty((B, self.cfg.n_layers), dtype=torch.uint8, device=self.device)
        _check(load().flux_router_apply(self._h, _ptr(logits), _ptr(mask), B, _ptr(mask_out), _stream()))
        self.mask = mask_out          # keep the cached decision alive
        return mask_out

    def flux_router_forward(self, weights, q_first, q_last, logits_out=None):
        """weights: dict of device tensors (w_enc1, b_enc1, w_enc2, b_enc2, w_head1, b_head1, w_head2,
        b_head2); q_first / q_last: bf16 [tokens][Hq][D] device tensors; logits_out: fp32 [2] device."""
        if logits_out is None:
            logits_out = torch.empty(2, dtype=torch.float32, device=self.device)
        w = FluxRouterWeights(int(weights["w_enc1"].shape[0]), int(weights["w_head1"].shape[0]),
                              *[_ptr(weights[k]) for k in ("w_enc1", "b_enc1", "w_enc2", "b_enc2",
                                                           "w_head1", "b_head1", "w_head2", "b_head2")])
        _check(load().flux_router_forward(self._h, ctypes.byref(w), _ptr(q_first), int(q_first.shape[0]),
                                          _ptr(q_last), int(q_last.shape[0]), _ptr(logits_out), _stream()))
        return logits_out

    def flux_attn_prefill(self, layer, req, q, k, v, q_start, out=None):
        Nq = int(q.shape[0])
        if out is None:
            out = torch.empty_like(q)
        _check(load().flux_attn_prefill(self._h, layer, req, _ptr(q), _ptr(k), _ptr(v), q_start, Nq,
                                        _ptr(out), _stream()))
        return out

    def flux_attn_prefill_blocks(self, q, k, v, q_start, block_mask, out=None):
        """block_mask: uint8 device tensor [n_q_blocks][n_kv_blocks], rows = absolute query blocks."""
        Nq = int(q.shape[0])
        if out is None:
            out = torch.empty_like(q)
        _check(load().flux_attn_prefill_blocks(self._h, _ptr(q), _ptr(k), _ptr(v), q_start, Nq,
                                               _ptr(block_mask), int(block_mask.shape[1]), _ptr(out), _stream()))
        return out

    def flux_attn_prefill_host(self, layer, req, q_host, q_dev, k, v, q_start, out_dev, out_host):
        Nq = int(q_host.shape[0])
        _check(load().flux_attn_prefill_host(self._h, layer, req, _ptr(q_host), _ptr(q_dev), _ptr(k),
                                             _ptr(v), q_start, Nq, _ptr(out_dev), _ptr(out_host),
                                             _stream()))
        return out_host

    def flux_kv_retain(self, layer, req, k_src, v_src, n, k_cache, v_cache):
        _check(load().flux_kv_retain(self._h, layer, req, _ptr(k_src), _ptr(v_src), n, _ptr(k_cache),
                                     _ptr(v_cache), _stream()))

    def flux_kv_append(self, layer, B, k_new, v_new, k_caches, v_caches, pos):
        _check(load().flux_kv_append(self._h, layer, B, _ptr(k_new), _ptr(v_new), _ptr(k_caches),
                                     _ptr(v_caches), _ptr(pos), _stream()))

    def flux_attn_decode(self, layer, B, q, k_caches, v_caches, ctx_len, out=None):
        if out is None:
            out = torch.empty_like(q)
        _check(load().flux_attn_decode(self._h, layer, B, _ptr(q), _ptr(k_caches), _ptr(v_caches),
                                       _ptr(ctx_len), _ptr(out), _stream()))
        return out

    def flux_attn_decode_partial(self, layer, B, q, k_caches, v_caches, ctx_len, key_begin, key_end, part_o=None, part_ml=None):
        """One piece of a decode step over the key positions [key_begin[b], key_end[b]) -> (part_o fp32 [B][Hq][D],
        part_ml fp32 [B][Hq][2])."""
        if part_o is None:
            part_o = torch.empty((B, self.cfg.n_q_heads, 128), dtype=torch.float32, device=self.device)
        if part_ml is None:
            part_ml = torch.empty((B, self.cfg.n_q_heads, 2), dtype=torch.float32, device=self.device)
        _check(load().flux_attn_decode_partial(self._h, layer, B, _ptr(q), _ptr(k_caches), _ptr(v_caches), _ptr(ctx_len),
                                               _ptr(key_begin), _ptr(key_end), _ptr(part_o), _ptr(part_ml), _stream()))
        return part_o, part_ml

    def flux_attn_combine(self, B, part_o, part_ml, out=None):
        """part_o fp32 [n_sets][B][Hq][D], part_ml fp32 [n_sets][B][Hq][2] -> out bf16 [B][Hq][D]."""
        n_sets = int(part_o.shape[0])
        if out is None:
            out = torch.empty((B, self.cfg.n_q_heads, 128), dtype=torch.bfloat16, device=self.device)
        _check(load().flux_attn_combine(self._h, B, n_sets, _ptr(part_o), _ptr(part_ml), _ptr(out), _stream()))
        return out

    def flux_attn_decode_partial_push(self, layer, B, q, k_caches, v_caches, ctx_len, key_begin, key_end, rank, gather_o, gather_ml, flags, seq):
        """This rank's piece stored straight into slot `rank` of every rank's gather buffer; gather_o / gather_ml / flags:
        one tensor per rank (fp32 [world][B][Hq][D], fp32 [world][B][Hq][2], int32 or uint32 [world]), addressable from this GPU."""
        ps = PeerSet()
        ps.world, ps.rank = len(gather_o), rank
        for p in range(ps.world):
            ps.gather_o[p], ps.gather_ml[p], ps.flags[p] = _ptr(gather_o[p]), _ptr(gather_ml[p]), _ptr(flags[p])
        _check(load().flux_attn_decode_partial_push(self._h, layer, B, _ptr(q), _ptr(k_caches), _ptr(v_caches), _ptr(ctx_len),
                                                    _ptr(key_begin), _ptr(key_end), ctypes.byref(ps), seq, _stream()))

    def flux_attn_combine_wait(self, B, gather_o, gather_ml, flags, seq, out=None, wait_cycles=0):
        """Waits (bounded) until every rank's flag equals seq, then merges this rank's gather buffer -> out bf16 [B][Hq][D]."""
        if out is None:
            out = torch.empty((B, self.cfg.n_q_heads, 128), dtype=torch.bfloat16, device=self.device)
        _check(load().flux_attn_combine_wait(self._h, B, int(gather_o.shape[0]), _ptr(gather_o), _ptr(gather_ml), _ptr(flags), seq,
                                             wait_cycles, _ptr(out), _stream()))
        return out

    def flux_attn_decode_heads(self, B, q, k_caches, v_caches, ctx_len, head_mask, out=None):
        """head_mask: uint8 device tensor [B][Hkv], 1 = dense head group, 0 = sink + window."""
        if out is None:
            out = torch.empty_like(q)
        _check(load().flux_attn_decode_heads(self._h, B, _ptr(q), _ptr(k_caches), _ptr(v_caches),
                                             _ptr(ctx_len), _ptr(head_mask), _ptr(out), _stream()))
        return out

    def flux_attn_decode_step(self, layer, B, q, k_new, v_new, k_caches, v_caches, ctx_len, out=None):
        if out is None:
            out = torch.empty_like(q)
        _check(load().flux_attn_decode_step(self._h, layer, B, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_caches),
                                            _ptr(v_caches), _ptr(ctx_len), _ptr(out), _stream()))
        return out

    def flux_attn_decode_host(self, layer, B, q_host, k_new_host, v_new_host, k_caches, v_caches,
                              pos, ctx_len, out_host):
        _check(load().flux_attn_decode_host(self._h, layer, B, _ptr(q_host), _ptr(k_new_host),
                                            _ptr(v_new_host), _ptr(k_caches), _ptr(v_caches),
                                            _ptr(pos), _ptr(ctx_len), _ptr(out_host), _stream()))
        return out_host

    def flux_attn_prefill_packed(self, layer, q, k, v, q_rows, k_rows=None, out=None):
        """Several requests' prompts (or chunks) in one launch.  q [rows][Hq][128], k / v [rows][Hkv][128], bf16, rows may be
        strided; q_rows / k_rows: HOST int32 [B + 1] (numpy or any sequence) row bounds of every request, k_rows = q_rows when
        omitted.  Rows of out outside the bounds are left as they are."""
        hq, hkv, dev = self.cfg.n_q_heads, self.cfg.n_kv_heads, self._index
        q_rows = _bounds(q_rows, "q_rows")
        k_rows = q_rows if k_rows is None else _bounds(k_rows, "k_rows")
        if q_rows.ndim != 1 or q_rows.shape != k_rows.shape or q_rows.shape[0] < 2:
            raise ValueError("q_rows and k_rows: expected two host arrays of batch + 1 row bounds")
        if q_rows[-1] > q.shape[0] or k_rows[-1] > k.shape[0] or k_rows[-1] > v.shape[0]:
            raise ValueError("row bounds end at %d / %d, q, k, v have %d, %d, %d rows"
                             % (q_rows[-1], k_rows[-1], q.shape[0], k.shape[0], v.shape[0]))
        if out is None:
            out = torch.empty_like(q) if q.is_contiguous() else self._bf16.new_empty(q.shape)
        _check(load().flux_attn_prefill_packed(self._h, layer, q_rows.shape[0] - 1, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                               _rows(q, hq, "q", dev), _rows(k, hkv, "k", dev), _rows(v, hkv, "v", dev),
                                               q_rows.tobytes(), k_rows.tobytes(), _flat_rows(out, q_rows[-1], hq, "out", dev), self._stream()))
        return out

    def flux_kvq_store(self, layer, fmt, k, v, row_start, pos, k_caches, v_caches):
        """Rows of k, v (bf16 [total_rows][Hkv][128], rows may be strided) into the requests' 8-bit caches: request b gets rows
        row_start[b] .. row_start[b + 1] - 1 (device int32 [B + 1]) as positions pos[b] .. (device int32 [B])."""
        B, hkv, dev = int(pos.shape[0]), self.cfg.n_kv_heads, self._index
        ks, vs = _rows(k, hkv, "k", dev), _rows(v, hkv, "v", dev)
        if v.shape[0] != k.shape[0]:
            raise ValueError("k and v have %d and %d rows" % (k.shape[0], v.shape[0]))
        _check(load().flux_kvq_store(self._h, layer, B, fmt, k.data_ptr(), v.data_ptr(), ks, vs, int(k.shape[0]),
                                     _int32(row_start, B + 1, "row_start", dev), _int32(pos, B, "pos", dev),
                                     *self._tables(k_caches, v_caches, B), self._stream()))

    def flux_kvq_load(self, layer, fmt, k_caches, v_caches, ctx_len, row_start, pos, total_rows, k_out=None, v_out=None):
        """The values that positions pos[b] .. of 8-bit caches of ctx_len[b] tokens stand for -> bf16 [total_rows][Hkv][128] each."""
        B, hkv, dev = int(pos.shape[0]), self.cfg.n_kv_heads, self._index
        if k_out is None:
            k_out = self._bf16.new_empty(total_rows, hkv, 128)
            kp = k_out.data_ptr()
        else:
            kp = _flat_rows(k_out, total_rows, hkv, "k_out", dev)
        if v_out is None:
            v_out = self._bf16.new_empty(total_rows, hkv, 128)
            vp = v_out.data_ptr()
        else:
            vp = _flat_rows(v_out, total_rows, hkv, "v_out", dev)
        _check(load().flux_kvq_load(self._h, layer, B, fmt, *self._tables(k_caches, v_caches, B),
                                    _int32(ctx_len, B, "ctx_len", dev), total_rows, _int32(row_start, B + 1, "row_start", dev),
                                    _int32(pos, B, "pos", dev), kp, vp, self._stream()))
        return k_out, v_out

    def flux_attn_decode_kvq(self, layer, B, fmt, q, k_caches, v_caches, ctx_len, out=None):
        """flux_attn_decode over 8-bit caches (fmt: FLUX_KVQ_E4M3 or FLUX_KVQ_INT8)."""
        hq, dev = self.cfg.n_q_heads, self._index
        qp = _flat_rows(q, B, hq, "q", dev)
        if out is None:
            out = torch.empty_like(q)
            op = out.data_ptr()
        else:
            op = _flat_rows(out, B, hq, "out", dev)
        _check(load().flux_attn_decode_kvq(self._h, layer, B, fmt, qp, *self._tables(k_caches, v_caches, B),
                                           _int32(ctx_len, B, "ctx_len", dev), op, self._stream()))
        return out

    def flux_attn_decode_step_kvq(self, layer, B, fmt, q, k_new, v_new, k_caches, v_caches, ctx_len, out=None):
        """Store of one token per request at position ctx_len - 1, then flux_attn_decode_kvq."""
        hq, hkv, dev = self.cfg.n_q_heads, self.cfg.n_kv_heads, self._index
        qp = _flat_rows(q, B, hq, "q", dev)
        if out is None:
            out = torch.empty_like(q)
            op = out.data_ptr()
        else:
            op = _flat_rows(out, B, hq, "out", dev)
        _check(load().flux_attn_decode_step_kvq(self._h, layer, B, fmt, qp, _flat_rows(k_new, B, hkv, "k_new", dev),
                                                _flat_rows(v_new, B, hkv, "v_new", dev), *self._tables(k_caches, v_caches, B),
                                                _int32(ctx_len, B, "ctx_len", dev), op, self._stream()))
        return out

    def flux_plan_status(self, raise_on_flag=True) -> int:
        bits = ctypes.c_uint32()
        rc = load().flux_plan_status(self._h, ctypes.byref(bits), _stream())
        if rc != FLUX_OK and (raise_on_flag or rc not in (FLUX_E_DEVICE_FLAG, FLUX_E_DEVICE_TIMEOUT)):
            _check(rc)
        return bits.value

    def flux_debug_dispatch(self, max_records=None) -> np.ndarray:
        """Records ``[n][8]``: mode, layer, request, n, a_begin, a_end, b_begin, b_end."""
        if max_records is None:
            max_records = self.cfg.max_batch
        rec = np.zeros((max_records, 8), dtype=np.int32)
        n = ctypes.c_int32()
        _check(load().flux_debug_dispatch(self._h, rec.ctypes.data, max_records, ctypes.byref(n), _stream()))
        return rec[: n.value].copy()

    def flux_debug_touched(self, bitmap=None) -> None:
        """bitmap: int32/uint32 device tensor [max_batch][words] (zeroed by the caller) or None (off)."""
        words = 0 if bitmap is None else int(bitmap.shape[1])
        _check(load().flux_debug_touched(self._h, _ptr(bitmap), words))
        self._touch = bitmap          # keep it alive while the plan points at it

    def flux_debug_wait_probe(self, limit_cycles: int) -> None:
        _check(load().flux_debug_wait_probe(self._h, limit_cycles, _stream()))

    def flux_plan_set_launch_overlap(self, on: bool) -> None:
        _check(load().flux_plan_set_launch_overlap(self._h, 1 if on else 0))

    def flux_debug_decode_kernel(self, which: int) -> None:
        _check(load().flux_debug_decode_kernel(self._h, which))

    def flux_profile_enable(self, max_records: int) -> None:
        _check(load().flux_profile_enable(self._h, max_records))

    def flux_profile_read(self, kind: int):
        """(total milliseconds, launches) of the recorded dominant-kernel launches of ``kind``."""
        ms = ctypes.c_double()
        n = ctypes.c_int64()
        _check(load().flux_profile_read(self._h, kind, ctypes.byref(ms), ctypes.byref(n), _stream()))
        return ms.value, n.value

    def flux_launch_count(self) -> int:
        return load().flux_launch_count(self._h)


def flux_attn_decode_noalloc(cfg: FluxConfig, layer, B, mask, q, k_caches, v_caches, ctx_len, out=None,
                             status_out=None):
    """Decode step for callers that cannot allocate device memory: needs no plan and no workspace.

    The split-K scratch is a fixed array inside the library (B <= 64, at most 8 query heads per KV
    head, at most 16 KV heads).  Calls on one device share that array, so calls that could overlap
    on the GPU must be serialised by the caller.  ``out`` is the caller's tensor (allocated here
    with torch only when omitted, as a convenience of this wrapper)."""
    if out is None:
        out = torch.empty_like(q)
    _check(load().flux_attn_decode_noalloc(ctypes.byref(cfg), layer, B, _ptr(mask), _ptr(q), _ptr(k_caches),
                                           _ptr(v_caches), _ptr(ctx_len), _ptr(out), _ptr(status_out),
                                           _stream()))
    return out


def pointer_table(tensors, device) -> torch.Tensor:
    """Device array of the tensors' addresses (the ``k_caches`` / ``v_caches`` argument)."""
    return torch.tensor([t.data_ptr() for t in tensors], dtype=torch.int64, device=device)
