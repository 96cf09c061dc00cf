"""ctypes binding over liblarosa.so: argument marshalling only.

Every function mirrors the C entry point of the same name (include/larosa.h).  Tensors are
torch CUDA tensors used purely as device buffers: 16-bit data as torch.float16 /
torch.bfloat16 (or uint16/int16 bit patterns), indices as torch.int32.  Work is enqueued on
torch's current stream.  A missing library is an error; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblarosa.so")

F16, BF16, F32 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP = 0, -1, -2, -3, -4

_lib = None


class LarosaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _Layer(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int), ("d_q", ctypes.c_int), ("d_kv", ctypes.c_int), ("d_ff", ctypes.c_int),
        ("head_dim", ctypes.c_int),
        ("K1", ctypes.c_int), ("K2", ctypes.c_int), ("K3", ctypes.c_int), ("K4", ctypes.c_int),
        ("Wqkv", ctypes.c_void_p), ("Wo", ctypes.c_void_p), ("Wgu", ctypes.c_void_p), ("Wdown", ctypes.c_void_p),
        ("Q_attn", ctypes.c_void_p), ("Q_mlp", ctypes.c_void_p), ("adapter", ctypes.c_void_p),
        ("rms_attn", ctypes.c_void_p), ("rms_mlp", ctypes.c_void_p),
        ("rms_eps", ctypes.c_float), ("attn_mode", ctypes.c_int), ("dtype", ctypes.c_int),
        ("shortcut_attn", ctypes.c_void_p), ("shortcut_mlp", ctypes.c_void_p),
    ]


TRACE_FIELDS = ("h1", "qkv", "h2", "o", "x1", "h3", "gu", "h4", "down", "x2", "idx1", "idx2", "idx3", "idx4",
                "s1", "s2")


class _Trace(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in TRACE_FIELDS] + [("stage_events", ctypes.c_void_p * 8)]


class _KvCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_layers", "n_pages", "page_tokens", "n_slots", "max_pages", "n_kv_heads", "head_dim",
                                            "dtype")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("data", "refs", "table", "length")]


class _KvBatch(ctypes.Structure):
    _fields_ = [("slots", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("n_seq", ctypes.c_int), ("n_rows", ctypes.c_int),
                ("max_new", ctypes.c_int)]


class _Rotary(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("n_positions", ctypes.c_int), ("rot_dim", ctypes.c_int),
                ("interleaved", ctypes.c_int), ("positions", ctypes.c_void_p), ("n_axes", ctypes.c_int),
                ("axis_pairs", ctypes.c_int * 4)]


def lib() -> ctypes.CDLL:
    """Load liblarosa.so (built in-tree by paper_2507_01299_amd.build); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2507_01299_amd.build` "
                               "(or __graft_entry__.build()) first; there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.larosa_status_string.restype = ctypes.c_char_p
        L.larosa_status_string.argtypes = [i]
        L.larosa_version.restype = i
        L.larosa_workspace_bytes.restype = sz
        L.larosa_workspace_bytes.argtypes = [i, i, i, i]
        L.larosa_workspace_init.argtypes = [vp, sz, vp]
        L.larosa_rotate.argtypes = [vp, vp, vp, i, i, i, vp, sz, vp]
        L.larosa_dense_gemv.argtypes = [vp, vp, vp, i, i, i, i, vp, sz, vp]
        L.larosa_topk.argtypes = [vp, i, i, i, vp, vp, i, vp, sz, vp]
        L.larosa_sparse_gemv.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
        L.larosa_sparse_gemv_static.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp]
        L.larosa_layer_workspace_bytes.restype = sz
        L.larosa_layer_workspace_bytes.argtypes = [ctypes.POINTER(_Layer), i]
        L.larosa_layer_forward.argtypes = [ctypes.POINTER(_Layer), vp, vp, i, ctypes.POINTER(_Trace), vp, sz, vp]
        L.larosa_layer_qkv.argtypes = [ctypes.POINTER(_Layer), vp, vp, vp, i, ctypes.POINTER(_Trace), vp, sz, vp]
        L.larosa_layer_after_attention.argtypes = [ctypes.POINTER(_Layer), vp, vp, vp, i, ctypes.POINTER(_Trace), vp,
                                                   sz, vp]
        L.larosa_set_tuning.argtypes = [i, i]
        L.larosa_quantize_w4.argtypes = [vp, i, i, i, vp, vp, vp]
        L.larosa_sparse_gemv_w4.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
        L.larosa_threshold_select.argtypes = [vp, i, i, ctypes.c_float, i, vp, vp, vp]
        L.larosa_offline_workspace_bytes.restype = sz
        L.larosa_offline_workspace_bytes.argtypes = [i, i]
        L.larosa_second_moment.argtypes = [vp, i, i, i, vp, i, vp]
        L.larosa_fold_input.argtypes = [vp, vp, i, i, i, vp, vp, sz, vp]
        L.larosa_fold_output.argtypes = [vp, vp, i, i, i, vp, vp, sz, vp]
        L.larosa_residual_adapter.argtypes = [vp, vp, i, i, vp, vp, sz, vp]
        cache, batch, rotary = ctypes.POINTER(_KvCache), ctypes.POINTER(_KvBatch), ctypes.POINTER(_Rotary)
        L.larosa_kv4_page_bytes.restype = L.larosa_kv4_data_bytes.restype = sz
        L.larosa_kv4_page_bytes.argtypes = [i, i, i]
        L.larosa_kv4_data_bytes.argtypes = [cache]
        L.larosa_kv4_clear.argtypes = [cache, vp]
        L.larosa_kv4_append.argtypes = [cache, i, batch, vp, i, i, rotary, vp, i, vp]
        L.larosa_kv4_attention_workspace_bytes.restype = sz
        L.larosa_kv4_attention_workspace_bytes.argtypes = [cache, batch, i, i]
        L.larosa_kv4_attention.argtypes = [cache, i, batch, vp, i, i, ctypes.c_float, i, i, vp, i, vp, sz, vp]
        L.larosa_kv4_attention_plan.argtypes = [cache, batch, i, i, i, ctypes.POINTER(i)]
        L.larosa_kv4_pages_workspace_bytes.restype = sz
        L.larosa_kv4_pages_workspace_bytes.argtypes = [cache]
        L.larosa_kv4_grow.argtypes = [cache, vp, vp, i, vp, vp, sz, vp]
        L.larosa_kv4_fork.argtypes = [cache, vp, vp, i, vp, vp]
        L.larosa_kv4_trim.argtypes = [cache, vp, vp, i, vp]
        L.larosa_kv4_compact.argtypes = [cache, vp, vp, sz, vp]
        L.larosa_kv4_copy_pages.argtypes = [cache, vp, vp, i, vp]
        L.larosa_layer_kv4_workspace_bytes.restype = sz
        L.larosa_layer_kv4_workspace_bytes.argtypes = [ctypes.POINTER(_Layer), cache, batch, i]
        L.larosa_layer_forward_kv4.argtypes = [ctypes.POINTER(_Layer), cache, i, batch, rotary, ctypes.c_float, i, i, vp, vp,
                                               ctypes.POINTER(_Trace), vp, sz, vp]
        f32 = ctypes.c_float
        L.larosa_quantize_w8.argtypes = [vp, i, i, i, vp, vp, vp]
        L.larosa_quantize_rows8.argtypes = [vp, i, i, i, vp, f32, i, vp, vp, vp]
        for name, sizes in (("product8", 3), ("dense_w8", 3), ("logprobs", 4), ("score_w8", 4)):
            query = getattr(L, f"larosa_{name}_workspace_bytes")
            query.restype, query.argtypes = sz, [i] * sizes
        L.larosa_product8.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
        L.larosa_dense_w8.argtypes = [vp, vp, vp, i, vp, f32, vp, i, i, i, i, i, vp, sz, vp]
        L.larosa_logprobs.argtypes = [vp, i, i, i, i, f32, vp, i, vp, vp, i, vp, vp, vp, sz, vp]
        L.larosa_score_w8.argtypes = [vp, vp, vp, i, vp, f32, i, i, i, i, f32, vp, i, vp, vp, i, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().larosa_status_string(int(status)).decode()


def version() -> int:
    return lib().larosa_version()


_DTYPE_CODES = {F16: F16, "f16": F16, torch.float16: F16, BF16: BF16, "bf16": BF16, torch.bfloat16: BF16}


def dtype_code(t) -> int:
    try:
        return _DTYPE_CODES[t]
    except (KeyError, TypeError):        # not found by hash: a 0-d array or tensor equal to a code is one too
        if t in (F16, "f16", torch.float16):
            return F16
        if t in (BF16, "bf16", torch.bfloat16):
            return BF16
        raise ValueError(f"unsupported dtype {t}") from None


def torch_dtype(code) -> torch.dtype:
    return torch.float16 if dtype_code(code) == F16 else torch.bfloat16


# A call on one small projection takes 4 - 9 us on the GPU, so what happens on the host before it counts: addresses go to
# ctypes as plain integers (the declared argument types convert them) and the current stream's handle is read without
# building a torch.cuda.Stream (Top-K and projection of 512 x 1024: 14.9 us a pass before, 10.1 now).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(rc: int, where: str):
    if rc != OK:
        raise LarosaError(rc, where)


class Workspace:
    """A caller-owned device buffer passed once through larosa_workspace_init."""

    def __init__(self, nbytes: int, device="cuda:0"):
        self.nbytes = int(nbytes)
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.ptr = self.buf.data_ptr() + off
        _check(lib().larosa_workspace_init(self.ptr, self.nbytes, _stream()), "larosa_workspace_init")


def workspace_bytes(B: int, d_in_max: int, d_out_max: int, K_max: int) -> int:
    return lib().larosa_workspace_bytes(B, d_in_max, d_out_max, K_max)


def workspace(B: int, d_in_max: int, d_out_max: int, K_max: int, device="cuda:0") -> Workspace:
    return Workspace(workspace_bytes(B, d_in_max, d_out_max, K_max), device)


def set_tuning(key: int, value: int):
    _check(lib().larosa_set_tuning(key, value), "larosa_set_tuning")


def rotate(x, Q, h, dtype, ws: Workspace):
    B, d = x.shape
    _check(lib().larosa_rotate(_ptr(x), _ptr(Q), _ptr(h), B, d, dtype_code(dtype),
                               ws.ptr, ws.nbytes, _stream()), "larosa_rotate")
    return h


def dense_gemv(Wp, x, y, dtype, ws: Workspace):
    B, d_in = x.shape
    d_out = Wp.shape[1]
    _check(lib().larosa_dense_gemv(_ptr(Wp), _ptr(x), _ptr(y), B, d_in, d_out, dtype_code(dtype),
                                   ws.ptr, ws.nbytes, _stream()), "larosa_dense_gemv")
    return y


def topk(h, K: int, idx, dtype, vals=None, ws: Workspace | None = None):
    B, d = h.shape
    _check(lib().larosa_topk(_ptr(h), B, d, K, _ptr(idx), _ptr(vals), dtype_code(dtype),
                             ws.ptr if ws else None, ws.nbytes if ws else 0, _stream()),
           "larosa_topk")
    return idx


def sparse_gemv(Wp, h, idx, y, dtype, ws: Workspace):
    B, d_in = h.shape
    d_out = Wp.shape[1]
    K = idx.shape[1]
    _check(lib().larosa_sparse_gemv(_ptr(Wp), _ptr(h), _ptr(idx), _ptr(y), B, d_in, d_out, K, dtype_code(dtype),
                                    ws.ptr, ws.nbytes, _stream()), "larosa_sparse_gemv")
    return y


def sparse_gemv_static(Wp, h, idx, y, dtype):
    """larosa_sparse_gemv without a workspace: the scratch is a fixed device array inside the library."""
    B, d_in = h.shape
    d_out = Wp.shape[1]
    K = idx.shape[1]
    _check(lib().larosa_sparse_gemv_static(_ptr(Wp), _ptr(h), _ptr(idx), _ptr(y), B, d_in, d_out, K,
                                           dtype_code(dtype), _stream()), "larosa_sparse_gemv_static")
    return y


def quantize_w4(W, dtype):
    """Round-to-nearest 4-bit codes (int32 [d_in, d_out/8], eight nibbles per dword) and 16-bit scales
    [d_in, ceil(d_out/128)] of W [d_in, d_out]."""
    d_in, d_out = W.shape
    Wq = torch.empty(d_in, d_out // 8, dtype=torch.int32, device=W.device)
    scales = torch.empty(d_in, (d_out + 127) // 128, dtype=W.dtype, device=W.device)
    _check(lib().larosa_quantize_w4(_ptr(W), d_in, d_out, dtype_code(dtype), _ptr(Wq), _ptr(scales), _stream()),
           "larosa_quantize_w4")
    return Wq, scales


def sparse_gemv_w4(Wq, scales, h, idx, y, dtype, ws: Workspace):
    B, d_in = h.shape
    d_out = Wq.shape[1] * 8
    K = d_in if idx is None else idx.shape[1]
    _check(lib().larosa_sparse_gemv_w4(_ptr(Wq), _ptr(scales), _ptr(h), _ptr(idx), _ptr(y), B, d_in, d_out, K,
                                       dtype_code(dtype), ws.ptr, ws.nbytes, _stream()),
           "larosa_sparse_gemv_w4")
    return y


def threshold_select(h, eps: float, idx, count, dtype):
    """idx [B, d] int32, count [B] int32: per token the ascending channels with |h| > eps."""
    B, d = h.shape
    _check(lib().larosa_threshold_select(_ptr(h), B, d, float(eps), dtype_code(dtype), _ptr(idx), _ptr(count),
                                         _stream()), "larosa_threshold_select")
    return idx, count


class OfflineScratch:
    """Device scratch for the folding calls (16-bit terms of the fp32 rotations)."""

    def __init__(self, d: int, dtype, device="cuda:0"):
        self.nbytes = int(lib().larosa_offline_workspace_bytes(d, dtype_code(dtype)))
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        self.ptr = self.buf.data_ptr() + (-self.buf.data_ptr()) % 256


def second_moment(X, C, dtype, accumulate: bool = False):
    """C [d,d] fp32 (+)= X^T X for X [n,d] 16-bit."""
    n, d = X.shape
    _check(lib().larosa_second_moment(_ptr(X), n, d, dtype_code(dtype), _ptr(C), int(accumulate), _stream()),
           "larosa_second_moment")
    return C


def fold_input(Q, W, W_out, dtype, scratch: OfflineScratch):
    """W_out [d,d_out] = Q^T W with Q [d,d] fp32."""
    d, d_out = W.shape
    _check(lib().larosa_fold_input(_ptr(Q), _ptr(W), d, d_out, dtype_code(dtype), _ptr(W_out),
                                   scratch.ptr, scratch.nbytes, _stream()), "larosa_fold_input")
    return W_out


def fold_output(W, Q, W_out, dtype, scratch: OfflineScratch):
    """W_out [d_in,d] = W Q with Q [d,d] fp32."""
    d_in, d = W.shape
    _check(lib().larosa_fold_output(_ptr(W), _ptr(Q), d_in, d, dtype_code(dtype), _ptr(W_out),
                                    scratch.ptr, scratch.nbytes, _stream()), "larosa_fold_output")
    return W_out


def residual_adapter(Q_l, Q_next, A_out, dtype, scratch: OfflineScratch):
    """A_out [d,d] = Q_l^T Q_next, both fp32."""
    d = Q_l.shape[0]
    _check(lib().larosa_residual_adapter(_ptr(Q_l), _ptr(Q_next), d, dtype_code(dtype), _ptr(A_out),
                                         scratch.ptr, scratch.nbytes, _stream()),
           "larosa_residual_adapter")
    return A_out


class Layer:
    """Holds the device tensors of one decoder layer and the matching C struct."""

    def __init__(self, d, d_q, d_kv, d_ff, head_dim, K1, K2, K3, K4, Wqkv, Wo, Wgu, Wdown, dtype,
                 Q_attn=None, Q_mlp=None, adapter=None, rms_attn=None, rms_mlp=None, rms_eps=-1.0, attn_mode=0,
                 shortcut_attn=None, shortcut_mlp=None):
        self.tensors = dict(Wqkv=Wqkv, Wo=Wo, Wgu=Wgu, Wdown=Wdown, Q_attn=Q_attn, Q_mlp=Q_mlp,
                            adapter=adapter, rms_attn=rms_attn, rms_mlp=rms_mlp, shortcut_attn=shortcut_attn,
                            shortcut_mlp=shortcut_mlp)   # keep alive
        self.dtype = dtype_code(dtype)
        self.c = _Layer(d, d_q, d_kv, d_ff, head_dim, K1, K2, K3, K4,
                        *[None if t is None else t.data_ptr() for t in
                          (Wqkv, Wo, Wgu, Wdown, Q_attn, Q_mlp, adapter, rms_attn, rms_mlp)],
                        float(rms_eps), int(attn_mode), self.dtype,
                        None if shortcut_attn is None else shortcut_attn.data_ptr(),
                        None if shortcut_mlp is None else shortcut_mlp.data_ptr())

    def workspace_bytes(self, B: int) -> int:
        return lib().larosa_layer_workspace_bytes(ctypes.byref(self.c), B)

    def trace_buffers(self, B: int, device="cuda:0") -> dict:
        c, td = self.c, torch_dtype(self.dtype)
        w = dict(h1=c.d, qkv=c.d_q + 2 * c.d_kv, h2=c.d_q, o=c.d, x1=c.d, h3=c.d, gu=2 * c.d_ff, h4=c.d_ff,
                 down=c.d, x2=c.d)
        if c.shortcut_attn:
            w["s1"] = c.d
        if c.shortcut_mlp:
            w["s2"] = c.d
        out = {k: torch.zeros(B, v, dtype=td, device=device) for k, v in w.items()}
        for k, K in (("idx1", c.K1), ("idx2", c.K2), ("idx3", c.K3), ("idx4", c.K4)):
            out[k] = torch.full((B, K), -1, dtype=torch.int32, device=device)
        return out


def _trace_struct(trace: dict | None, stage_events=None):
    if trace is None and stage_events is None:
        return None
    trace = trace or {}
    tr = _Trace(*[None if trace.get(n) is None else trace[n].data_ptr() for n in TRACE_FIELDS])
    if stage_events is not None:
        for i, ev in enumerate(stage_events[:8]):
            tr.stage_events[i] = None if ev is None else ev.cuda_event
    return tr


def layer_forward(layer: Layer, x, x_out, ws: Workspace, trace: dict | None = None, stage_events=None):
    """stage_events: optional list of up to 8 torch.cuda.Event(enable_timing=True) that have been
    recorded once already (so their handles exist); the library records them at stage boundaries."""
    B = x.shape[0]
    tr = _trace_struct(trace, stage_events)
    _check(lib().larosa_layer_forward(ctypes.byref(layer.c), _ptr(x), _ptr(x_out), B,
                                      ctypes.byref(tr) if tr is not None else None,
                                      ws.ptr, ws.nbytes, _stream()), "larosa_layer_forward")
    return x_out


def layer_qkv(layer: Layer, x, qkv, s1, ws: Workspace, trace: dict | None = None):
    """First half of the layer for a caller with its own attention core: writes q|k|v and, if the
    layer has shortcut_attn, the shortcut value s1 (else pass None)."""
    tr = _trace_struct(trace)
    _check(lib().larosa_layer_qkv(ctypes.byref(layer.c), _ptr(x), _ptr(qkv), _ptr(s1), x.shape[0],
                                  ctypes.byref(tr) if tr is not None else None,
                                  ws.ptr, ws.nbytes, _stream()), "larosa_layer_qkv")
    return qkv


def layer_after_attention(layer: Layer, residual, attn, x_out, ws: Workspace, trace: dict | None = None):
    """Rest of the layer from the attention core's output attn [B, d_q]; residual is the layer input x,
    or the s1 written by layer_qkv when the layer has shortcut_attn."""
    tr = _trace_struct(trace)
    _check(lib().larosa_layer_after_attention(ctypes.byref(layer.c), _ptr(residual), _ptr(attn), _ptr(x_out),
                                              residual.shape[0], ctypes.byref(tr) if tr is not None else None,
                                              ws.ptr, ws.nbytes, _stream()),
           "larosa_layer_after_attention")
    return x_out


_INT32 = torch.int32        # (a name of this module: each look into torch's costs a call 40 ns, and a list is checked by four)


def _list(t, n, device):
    """Address of a list for the 4-bit cache (None: none): anything but n int32 in a row on the cache's device would be misread there."""
    if t is None:
        return None
    if t.dtype is not _INT32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"a list of {n} contiguous int32 on the cache's device")
    return t.data_ptr()


def _first_list(t, device):
    """A call's first list, which says how long the others are: its length and address."""
    if t.dtype is not _INT32 or not t.is_contiguous() or t.get_device() != device:
        raise ValueError("a list of contiguous int32 on the cache's device")
    return t.numel(), t.data_ptr()


def _word(t, device):
    """Address of the one int32 that a call reports to."""
    if t is None:
        return None
    if t.dtype is not _INT32 or t.numel() < 1 or t.get_device() != device:
        raise ValueError("an int32 on the cache's device")
    return t.data_ptr()


class KvCache:
    """Device tensors of a 4-bit key/value cache and the matching C struct.  Tensors that are not given are allocated, and the
    cache is then made empty; given ones are taken as they are (all of refs, table and length, or none).  Calls on a cache are made with
    its device as the current one, and with lists and rows on it."""

    def __init__(self, n_layers, n_pages, page_tokens, n_slots, max_pages, n_kv_heads, head_dim, dtype, data=None, refs=None,
                 table=None, length=None, device="cuda:0"):
        self.dtype, self.torch_dtype = dtype_code(dtype), torch_dtype(dtype)
        self.c = _KvCache(n_layers, n_pages, page_tokens, n_slots, max_pages, n_kv_heads, head_dim, self.dtype)
        nbytes = lib().larosa_kv4_data_bytes(ctypes.byref(self.c))
        if nbytes == 0:
            raise LarosaError(EINVAL, "larosa_kv4_data_bytes")
        state = (refs, table, length)
        if any(t is None for t in state) and any(t is not None for t in state):
            raise ValueError("refs, table and length are given together")
        fresh = refs is None
        if fresh:
            refs = torch.empty(n_pages, dtype=torch.int32, device=device)
            table = torch.empty(n_slots, max_pages, dtype=torch.int32, device=device)
            length = torch.empty(n_slots, dtype=torch.int32, device=device)
        if data is None:
            data = torch.empty(nbytes, dtype=torch.uint8, device=device)
        sizes = (refs.numel(), table.numel(), length.numel())
        if sizes != (n_pages, n_slots * max_pages, n_slots) or data.numel() * data.element_size() < nbytes:
            raise ValueError("refs [n_pages], table [n_slots, max_pages], length [n_slots], data of larosa_kv4_data_bytes")
        if any(t.dtype != torch.int32 for t in (refs, table, length)) or not all(t.is_contiguous() for t in (data, refs, table, length)):
            raise ValueError("refs, table and length are contiguous int32 tensors, data is contiguous")
        self.device = refs.get_device()      # (as a number: all of a call's tensors are compared with it)
        if any(t.get_device() != self.device for t in (data, table, length)):
            raise ValueError("refs, table, length and data lie on one device")
        self.data, self.refs, self.table, self.length = data, refs, table, length
        self.c.data, self.c.refs, self.c.table, self.c.length = (t.data_ptr() for t in (data, refs, table, length))
        self.ref = ctypes.byref(self.c)
        if fresh:
            kv4_clear(self)


class KvBatch:
    """Which of n_rows rows are the newest tokens of which sequence: slots [n_seq] int32, starts [n_seq + 1] int32 or None (one
    row for each sequence), max_new the most of one sequence."""

    def __init__(self, slots, n_rows: int, starts=None, max_new: int = 1):
        self.device = slots.get_device()
        n_seq, listed = _first_list(slots, self.device)
        self.tensors = (slots, starts)       # keep alive
        self.n_rows = n_rows
        self.c = _KvBatch(listed, _list(starts, n_seq + 1, self.device), n_seq, n_rows, max_new)
        self.ref = ctypes.byref(self.c)


class Rotary:
    """Rotary positions: table [n_positions, rot_dim] fp32 (cosines, then sines); positions [n_axes, n_rows] int32 or None (a
    token's place in its sequence); axis_pairs: the frequencies of each axis where there are several."""

    def __init__(self, table, positions=None, axis_pairs=None, interleaved: bool = False):
        self.tensors = (table, positions)    # keep alive
        n_axes = len(axis_pairs) if axis_pairs else 1
        if n_axes > 4 or (positions is not None and positions.shape[0] != n_axes):
            raise ValueError("one to four axes, a row of positions and a number of frequencies for each")
        if table.dtype != torch.float32 or not table.is_contiguous() or (
                positions is not None and (positions.dtype != torch.int32 or not positions.is_contiguous())):
            raise ValueError("table [n_positions, rot_dim] is contiguous float32, positions [n_axes, n_rows] contiguous int32")
        self.device, self.n_rows = table.get_device(), None if positions is None else positions.shape[1]
        if positions is not None and positions.get_device() != self.device:
            raise ValueError("table and positions lie on one device")
        self.c = _Rotary(_ptr(table), table.shape[0], table.shape[1], int(interleaved), _ptr(positions), n_axes)
        for k, n in enumerate(axis_pairs or ()):
            self.c.axis_pairs[k] = n
        self.ref = ctypes.byref(self.c)


def _rows(t, n_rows: int, cache) -> int:
    """Distance between the rows of a tensor of the cache's type; anything else would be misread on the device."""
    if t.dtype is not cache.torch_dtype or t.get_device() != cache.device:
        raise ValueError("rows are of the cache's type and on its device")
    ld, one = t.stride()
    if one != 1 or t.shape[0] < n_rows:
        raise ValueError(f"a tensor of at least {n_rows} rows, whose values lie next to one another")
    return ld


def _cache_stream(cache):
    """The current stream; its device has to be the cache's."""
    device = torch._C._cuda_getDevice()      # (the cache's tensors are there, so the runtime is up)
    if device != cache.device:
        raise ValueError("the cache's device is not the current one")
    return torch._C._cuda_getCurrentRawStream(device)


def _check_batch(cache, batch, rotary=None):
    if batch.device != cache.device or (rotary is not None and rotary.device != cache.device):
        raise ValueError("batch and rotary positions lie on the cache's device")
    if rotary is not None and rotary.n_rows is not None and rotary.n_rows != batch.n_rows:
        raise ValueError("positions have a column for every row of the batch")


def kv4_clear(cache: KvCache):
    _check(lib().larosa_kv4_clear(cache.ref, _cache_stream(cache)), "larosa_kv4_clear")


def kv4_append(cache: KvCache, layer: int, batch: KvBatch, qkv, n_heads: int, out=None, rotary: Rotary | None = None):
    """The rows' new keys and values into the cache; out (may be qkv) receives q as turned and k, v as stored."""
    _check_batch(cache, batch, rotary)
    ld_qkv = _rows(qkv, batch.n_rows, cache)
    ld_out = 0 if out is None else _rows(out, batch.n_rows, cache)
    _check(lib().larosa_kv4_append(cache.ref, layer, batch.ref, _ptr(qkv), ld_qkv, n_heads,
                                   rotary.ref if rotary is not None else None, _ptr(out), ld_out,
                                   _cache_stream(cache)), "larosa_kv4_append")
    return out


def kv4_attention_workspace(cache: KvCache, batch: KvBatch, n_heads: int, max_len: int = 0, device="cuda:0") -> Workspace:
    nbytes = lib().larosa_kv4_attention_workspace_bytes(cache.ref, batch.ref, n_heads, max_len)
    if nbytes == 0:
        raise LarosaError(EINVAL, "larosa_kv4_attention_workspace_bytes")
    return Workspace(nbytes, device)


def kv4_attention(cache: KvCache, layer: int, batch: KvBatch, q, n_heads: int, out, ws: Workspace, scale: float | None = None,
                  window: int = 0, max_len: int = 0):
    """out[row] = attention of the row's query heads (the first n_heads heads of q's row) over the cache; scale defaults to
    1 / sqrt(head_dim)."""
    if scale is None:
        scale = cache.c.head_dim ** -0.5
    _check_batch(cache, batch)
    ld_q, ld_out = _rows(q, batch.n_rows, cache), _rows(out, batch.n_rows, cache)
    _check(lib().larosa_kv4_attention(cache.ref, layer, batch.ref, _ptr(q), ld_q, n_heads, scale,
                                      window, max_len, _ptr(out), ld_out, ws.ptr, ws.nbytes, _cache_stream(cache)),
           "larosa_kv4_attention")
    return out


def kv4_attention_plan(cache: KvCache, batch: KvBatch, n_heads: int, window: int = 0, max_len: int = 0) -> dict:
    """How kv4_attention would divide the call (for tests and experiments; not part of the stable interface)."""
    plan = (ctypes.c_int * 5)()
    _check(lib().larosa_kv4_attention_plan(cache.ref, batch.ref, n_heads, window, max_len, plan), "larosa_kv4_attention_plan")
    return dict(zip(("tile_rows", "row_tiles", "chunk", "splits", "sums"), plan))


def kv4_pages_workspace(cache: KvCache, device="cuda:0") -> Workspace:
    return Workspace(lib().larosa_kv4_pages_workspace_bytes(cache.ref), device)


def kv4_grow(cache: KvCache, slots, status, ws: Workspace, counts=None):
    """Room for counts (default one) more tokens in every listed slot; status [1] int32: 0, pages missing, or -1."""
    dev = cache.device
    n, listed = _first_list(slots, dev)
    _check(lib().larosa_kv4_grow(cache.ref, listed, _list(counts, n, dev), n, _word(status, dev), ws.ptr, ws.nbytes,
                                 _cache_stream(cache)), "larosa_kv4_grow")
    return status


def kv4_fork(cache: KvCache, src, dst, status):
    """The sequences of src into the free slots dst, all pages shared; status [1] int32: 0 or -1."""
    dev = cache.device
    n, listed = _first_list(src, dev)
    _check(lib().larosa_kv4_fork(cache.ref, listed, _list(dst, n, dev), n, _word(status, dev), _cache_stream(cache)),
           "larosa_kv4_fork")
    return status


def kv4_trim(cache: KvCache, slots, keep=None):
    """Listed slots keep their first keep tokens (default none)."""
    dev = cache.device
    n, listed = _first_list(slots, dev)
    _check(lib().larosa_kv4_trim(cache.ref, listed, _list(keep, n, dev), n, _cache_stream(cache)), "larosa_kv4_trim")


def kv4_compact(cache: KvCache, live, ws: Workspace):
    """Pages in use to the lowest ids; live [1] int32 (or None) receives their number."""
    _check(lib().larosa_kv4_compact(cache.ref, _word(live, cache.device), ws.ptr, ws.nbytes, _cache_stream(cache)), "larosa_kv4_compact")
    return live


def kv4_copy_pages(cache: KvCache, src, dst):
    """Pages src of every layer into pages dst."""
    dev = cache.device
    n, listed = _first_list(src, dev)
    _check(lib().larosa_kv4_copy_pages(cache.ref, listed, _list(dst, n, dev), n, _cache_stream(cache)), "larosa_kv4_copy_pages")


def layer_kv4_workspace(layer: Layer, cache: KvCache, batch: KvBatch, max_len: int = 0, device="cuda:0") -> Workspace:
    nbytes = lib().larosa_layer_kv4_workspace_bytes(ctypes.byref(layer.c), cache.ref, batch.ref, max_len)
    if nbytes == 0:
        raise LarosaError(EINVAL, "larosa_layer_kv4_workspace_bytes")
    return Workspace(nbytes, device)


def layer_forward_kv4(layer: Layer, cache: KvCache, index: int, batch: KvBatch, x, x_out, ws: Workspace, rotary: Rotary | None = None,
                      scale: float | None = None, window: int = 0, max_len: int = 0, trace: dict | None = None):
    """A decoder layer whose attention runs over layer `index` of the cache; the rows' tokens are counted in the lengths."""
    _check_batch(cache, batch, rotary)
    for t in (x, x_out):
        _rows(t, batch.n_rows, cache)
        if tuple(t.shape) != (batch.n_rows, layer.c.d) or not t.is_contiguous():
            raise ValueError("x and x_out [n_rows of the batch, d of the layer] are contiguous")
    if scale is None:
        scale = cache.c.head_dim ** -0.5
    tr = _trace_struct(trace)
    _check(lib().larosa_layer_forward_kv4(ctypes.byref(layer.c), cache.ref, index, batch.ref,
                                          rotary.ref if rotary is not None else None, scale, window, max_len, _ptr(x),
                                          _ptr(x_out), ctypes.byref(tr) if tr is not None else None, ws.ptr, ws.nbytes, _cache_stream(cache)),
           "larosa_layer_forward_kv4")
    return x_out


# ---- weights in 8-bit floating point, products over them, log probabilities -------------------------------

def codes_pitch8(d: int) -> int:
    """Bytes between the rows of the codes of d channels."""
    return -(-d // 16) * 16


def scales_pitch8(d: int) -> int:
    """Bytes between the rows of their scales."""
    return -(-d // 512) * 4


_CODES = (torch.float8_e4m3fn, torch.uint8)
_LOGITS = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}


def _held8(codes, scales, d_in: int, rows_of_block: int, device: int):
    """Addresses of codes and scales; other shapes or types would be misread on the device."""
    n = codes.shape[0]
    if codes.dtype not in _CODES or scales.dtype is not torch.uint8 or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("codes are contiguous float8_e4m3fn (or uint8), scales contiguous uint8")
    if codes.shape != (n, codes_pitch8(d_in)) or scales.shape != (-(-n // rows_of_block), scales_pitch8(d_in)):
        raise ValueError(f"codes [n, {codes_pitch8(d_in)}] and scales [n / {rows_of_block} up, {scales_pitch8(d_in)}] of {d_in} channels")
    if codes.get_device() != device or scales.get_device() != device:
        raise ValueError("codes and scales lie on the current device")
    return codes.data_ptr(), scales.data_ptr()


def _device_stream(*tensors):
    """The current device and its stream; every tensor has to lie there."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("every tensor lies on the current device")
    return device, torch._C._cuda_getCurrentRawStream(device)


# The library's sizes and distances are 32-bit: a larger one would arrive as its low 32 bits, another matrix.
_SIZE = 1 << 31


def _matrix16(t, code: int) -> int:
    """Distance between the rows of a matrix of the type `code`."""
    stride = t.stride()
    if t.dtype is not torch_dtype(code) or len(stride) != 2:
        raise ValueError("rows are a matrix of the call's type")
    ld, one = stride
    rows, width = t.shape
    if one != 1 and width != 1:
        raise ValueError("the values of a row lie next to one another")
    if rows == 1:        # whatever its tensor says of the distance to a next one, one that the library takes
        ld = max(min(ld // 8 * 8, 1 << 20), -(-width // 8) * 8)
    if ld >= _SIZE or rows >= _SIZE:
        raise ValueError("sizes and distances between rows are below 2^31")
    return ld


def _logits(t):
    """Distance between the rows of logits, and their type."""
    stride = t.stride()
    if t.dtype not in _LOGITS or len(stride) != 2:
        raise ValueError("logits are a matrix of float16, bfloat16 or float32")
    ld, one = stride
    rows, width = t.shape
    if one != 1 and width != 1:
        raise ValueError("the logits of a row lie next to one another")
    if rows == 1:
        ld = width
    if ld >= _SIZE or rows >= _SIZE or width >= _SIZE:
        raise ValueError("sizes and distances between rows are below 2^31")
    return ld, _LOGITS[t.dtype]


def _norm8(rms, d: int, code: int, rms_eps: float = 0.0):
    if rms is not None and not rms_eps >= 0:
        raise ValueError("rms is the scale of a norm: rms_eps is at least 0 with it")
    if rms is not None and (rms.dtype is not torch_dtype(code) or rms.shape != (d,) or not rms.is_contiguous()):
        raise ValueError("rms is a contiguous vector of the call's type, a value for each channel")
    return _ptr(rms)


def quantize_w8(W, dtype):
    """e4m3 codes (float8_e4m3fn [d_out, d_in up to 16]) and scale bytes (uint8 [d_out / 128 up, d_in / 128 up, up to 4]) of
    W [d_in, d_out], d_out a multiple of 8.  An output head of n_vocab tokens, any number: of W filled up with columns of zeros,
    (codes[:n_vocab], scales)."""
    code = dtype_code(dtype)
    _, stream = _device_stream(W)
    _matrix16(W, code)
    d_in, d_out = W.shape
    if not W.is_contiguous():
        raise ValueError("W is a contiguous matrix of the call's type")
    codes = torch.empty(d_out, codes_pitch8(d_in), dtype=torch.float8_e4m3fn, device=W.device)
    scales = torch.empty(-(-d_out // 128), scales_pitch8(d_in), dtype=torch.uint8, device=W.device)
    _check(lib().larosa_quantize_w8(_ptr(W), d_in, d_out, code, _ptr(codes), _ptr(scales), stream), "larosa_quantize_w8")
    return codes, scales


def quantize_rows8(x, dtype, rms=None, rms_eps: float = -1.0):
    """Codes [n, d up to 16] and scale bytes [n, d / 128 up, up to 4] of x [n, d]; rms_eps >= 0: behind a norm (rms: its scale,
    None = 1); without a norm there is no rms."""
    code = dtype_code(dtype)
    _, stream = _device_stream(x, rms)
    ld = _matrix16(x, code)
    n, d = x.shape
    codes = torch.empty(n, codes_pitch8(d), dtype=torch.float8_e4m3fn, device=x.device)
    scales = torch.empty(n, scales_pitch8(d), dtype=torch.uint8, device=x.device)
    _check(lib().larosa_quantize_rows8(_ptr(x), ld, n, d, _norm8(rms, d, code, rms_eps), rms_eps, code, _ptr(codes), _ptr(scales), stream),
           "larosa_quantize_rows8")
    return codes, scales


def _sized(nbytes: int, where: str, device) -> Workspace:
    if nbytes == 0:
        raise LarosaError(EINVAL, where)
    return Workspace(nbytes, device)


def product8_workspace(n_rows: int, d_in: int, d_out: int, device="cuda:0") -> Workspace:
    return _sized(lib().larosa_product8_workspace_bytes(n_rows, d_in, d_out), "larosa_product8_workspace_bytes", device)


def product8(w_codes, w_scales, x_codes, x_scales, d_in: int, y, dtype, ws: Workspace):
    """y [n, d_out] = the product of rows and weight, both in 8 bits."""
    code = dtype_code(dtype)
    device, stream = _device_stream(y, ws.buf)
    wc, wsc = _held8(w_codes, w_scales, d_in, 128, device)
    xc, xsc = _held8(x_codes, x_scales, d_in, 1, device)
    ld_y = _matrix16(y, code)
    n, d_out = y.shape
    if w_codes.shape[0] != d_out or x_codes.shape[0] != n:
        raise ValueError("y has a row for each row of x and a column for each output channel")
    _check(lib().larosa_product8(wc, wsc, xc, xsc, _ptr(y), ld_y, n, d_in, d_out, code, ws.ptr, ws.nbytes, stream), "larosa_product8")
    return y


def dense_w8_workspace(n_rows: int, d_in: int, d_out: int, device="cuda:0") -> Workspace:
    return _sized(lib().larosa_dense_w8_workspace_bytes(n_rows, d_in, d_out), "larosa_dense_w8_workspace_bytes", device)


def dense_w8(w_codes, w_scales, x, y, dtype, ws: Workspace, rms=None, rms_eps: float = -1.0):
    """y [n, d_out] = x [n, d_in] (behind a norm if rms_eps >= 0), brought to 8 bits, times the weight."""
    code = dtype_code(dtype)
    device, stream = _device_stream(x, y, rms, ws.buf)
    n, d_in = x.shape
    wc, wsc = _held8(w_codes, w_scales, d_in, 128, device)
    ld_x, ld_y = _matrix16(x, code), _matrix16(y, code)
    if y.shape != (n, w_codes.shape[0]):
        raise ValueError("y has a row for each row of x and a column for each output channel")
    _check(lib().larosa_dense_w8(wc, wsc, _ptr(x), ld_x, _norm8(rms, d_in, code, rms_eps), rms_eps, _ptr(y), ld_y, n, d_in, y.shape[1], code,
                                 ws.ptr, ws.nbytes, stream), "larosa_dense_w8")
    return y


def _outputs8(n: int, given, logp, entropy, top_id, top_logp):
    """Numbers of given and of top tokens."""
    n_given = 0 if given is None else given.shape[1]
    n_top = 0 if top_id is None else top_id.shape[1]
    for t, width, kind in ((given, n_given, torch.int32), (logp, n_given, torch.float32), (top_id, n_top, torch.int32),
                           (top_logp, n_top, torch.float32)):
        if t is not None and (t.dtype is not kind or t.shape != (n, width) or not t.is_contiguous()):
            raise ValueError("given and top_id are contiguous int32, logp and top_logp contiguous float32 of their shapes")
    if entropy is not None and (entropy.dtype is not torch.float32 or entropy.shape != (n,) or not entropy.is_contiguous()):
        raise ValueError("entropy is a contiguous float32 vector, a value for each row")
    if (logp is None) != (given is None) and n_given:
        raise ValueError("given tokens and logp come together")
    if n_given >> 31:
        raise ValueError("fewer than 2^31 given tokens of a row")
    return n_given, n_top


def logprobs_workspace(n_rows: int, n_vocab: int, n_top: int = 0, dtype="bf16", device="cuda:0") -> Workspace:
    """For n_rows rows or fewer; logits of every type take the same room."""
    code = F32 if dtype in (F32, "f32", torch.float32) else dtype_code(dtype)
    return _sized(lib().larosa_logprobs_workspace_bytes(n_rows, n_vocab, n_top, code), "larosa_logprobs_workspace_bytes", device)


def logprobs(logits, given, logp, ws: Workspace, entropy=None, top_id=None, top_logp=None, scale: float = 1.0):
    """Log probabilities of the given tokens [n, n_given] under softmax(scale * logits [n, n_vocab]), the rows' entropy [n] and the most
    probable tokens top_id [n, n_top] with theirs, top_logp."""
    device, stream = _device_stream(logits, given, logp, entropy, top_id, top_logp, ws.buf)
    ld, kind = _logits(logits)
    n, V = logits.shape
    n_given, n_top = _outputs8(n, given, logp, entropy, top_id, top_logp)
    _check(lib().larosa_logprobs(_ptr(logits), ld, n, V, kind, scale, _ptr(given), n_given,
                                 _ptr(logp), _ptr(entropy), n_top, _ptr(top_id), _ptr(top_logp), ws.ptr, ws.nbytes, stream),
           "larosa_logprobs")
    return logp


def score_w8_workspace(n_rows: int, d_in: int, n_vocab: int, n_top: int = 0, device="cuda:0") -> Workspace:
    return _sized(lib().larosa_score_w8_workspace_bytes(n_rows, d_in, n_vocab, n_top), "larosa_score_w8_workspace_bytes", device)


def score_w8(w_codes, w_scales, x, given, logp, dtype, ws: Workspace, entropy=None, top_id=None, top_logp=None, scale: float = 1.0,
             rms=None, rms_eps: float = -1.0):
    """logprobs of the output head's logits of x [n, d_in] (behind the final norm if rms_eps >= 0); the head in 8 bits."""
    code = dtype_code(dtype)
    device, stream = _device_stream(x, given, logp, entropy, top_id, top_logp, rms, ws.buf)
    n, d_in = x.shape
    wc, wsc = _held8(w_codes, w_scales, d_in, 128, device)
    ld_x = _matrix16(x, code)
    n_given, n_top = _outputs8(n, given, logp, entropy, top_id, top_logp)
    _check(lib().larosa_score_w8(wc, wsc, _ptr(x), ld_x, _norm8(rms, d_in, code, rms_eps), rms_eps, n, d_in, w_codes.shape[0], code, scale,
                                 _ptr(given), n_given, _ptr(logp), _ptr(entropy), n_top, _ptr(top_id), _ptr(top_logp), ws.ptr,
                                 ws.nbytes, stream), "larosa_score_w8")
    return logp
