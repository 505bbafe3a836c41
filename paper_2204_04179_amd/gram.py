"""Thin ctypes binding of libgram (include/gram.h).

Argument marshalling only: every step of the path runs in the HIP kernels of
the library.  PyTorch supplies device memory and the current stream.  There is
no fallback: if the shared library is missing or fails to load, `load()`
raises.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libgram.so")

F32, BF16 = 0, 1
OK, ERR_ARG, ERR_CAPACITY, ERR_SEQUENCE, ERR_RANGE, ERR_HIP, ERR_UNIMPLEMENTED = 0, -1, -2, -3, -4, -5, -6
STATUS_NAMES = {OK: "GRAM_OK", ERR_ARG: "GRAM_ERR_ARG", ERR_CAPACITY: "GRAM_ERR_CAPACITY",
                ERR_SEQUENCE: "GRAM_ERR_SEQUENCE", ERR_RANGE: "GRAM_ERR_RANGE", ERR_HIP: "GRAM_ERR_HIP",
                ERR_UNIMPLEMENTED: "GRAM_ERR_UNIMPLEMENTED"}

EXPORTS = ("gram_workspace_bytes", "gram_create", "gram_destroy", "gram_unique", "gram_encode_gather",
           "gram_grad_accumulate", "gram_pseudo_target", "gram_gather", "gram_encoder_wgrad",
           "gram_encoder_wgrad_chunk", "gram_pseudo_loss_grad", "gram_flush",
           "gram_flush64", "gram_window_end", "gram_window_import", "gram_mlp_encode_gather", "gram_mlp_batch_bytes",
           "gram_mlp_backward", "gram_unique_static",
           "gram_layer_norm", "gram_layer_norm_backward", "gram_layer_norm_work_bytes", "gram_distance_bucket",
           "gram_attention", "gram_attention_backward", "gram_attention_backward_bytes", "gram_attention_step",
           "gram_attention_step_bytes",
           "gram_check", "gram_last_error",
           "gram_kernel_count", "gram_kernel_name", "gram_light_max", "gram_profile_enable",
           "gram_profile_read")


class GramConfig(C.Structure):
    _fields_ = [("vocab_n", C.c_int32), ("d_in", C.c_int32), ("d", C.c_int32),
                ("max_positions", C.c_int64), ("k_steps", C.c_int32), ("pad_id", C.c_int32),
                ("u_total_cap", C.c_int64), ("xw_dtype", C.c_int32), ("buffer_layout", C.c_int32),
                ("d_hidden", C.c_int32), ("h_dtype", C.c_int32)]


class GramAttentionConfig(C.Structure):
    _fields_ = [("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_float), ("cap", C.c_float), ("causal", C.c_int32), ("buckets", C.c_int32),
                ("max_distance", C.c_int32), ("two_sided", C.c_int32)]


class GramRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("row_stride", C.c_int64),
                ("head_stride", C.c_int64)]


class GramError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None


def load():
    """Open libgram.so (built by `python -m paper_2204_04179_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2204_04179_amd.build`")
    # PyTorch ships a HIP runtime of its own.  It has to be in the process before this library is
    # opened, so that the library binds to the same runtime as the tensors it is handed; opened
    # the other way round, PyTorch finds no device afterwards.
    import torch  # noqa: F401
    L = C.CDLL(LIB_PATH)
    vp, i32p = C.c_void_p, C.POINTER(C.c_int32)
    L.gram_workspace_bytes.restype = C.c_int64
    L.gram_workspace_bytes.argtypes = [C.POINTER(GramConfig)]
    L.gram_create.restype = C.c_int
    L.gram_create.argtypes = [C.POINTER(vp), C.POINTER(GramConfig)]
    L.gram_destroy.restype = C.c_int
    L.gram_destroy.argtypes = [vp]
    L.gram_unique.restype = C.c_int
    L.gram_unique.argtypes = [vp, vp, C.c_int64, vp, vp, vp, vp, i32p, vp]
    L.gram_encode_gather.restype = C.c_int
    L.gram_encode_gather.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int64, vp, vp, vp]
    L.gram_grad_accumulate.restype = C.c_int
    L.gram_grad_accumulate.argtypes = [vp, vp, C.c_int64, C.c_int32, vp]
    L.gram_encoder_wgrad_chunk.restype = C.c_int
    L.gram_encoder_wgrad_chunk.argtypes = [vp, vp, vp, C.c_int64, C.c_int64, C.c_int32, vp]
    L.gram_pseudo_loss_grad.restype = C.c_int
    L.gram_pseudo_loss_grad.argtypes = [vp, vp, vp, vp, vp, C.c_int64, vp, vp, C.c_int32, vp, vp]
    L.gram_pseudo_target.restype = C.c_int
    L.gram_pseudo_target.argtypes = [vp, vp, vp, vp, vp]
    L.gram_gather.restype = C.c_int
    L.gram_gather.argtypes = [vp, vp, vp, C.c_int64, vp, vp]
    L.gram_encoder_wgrad.restype = C.c_int
    L.gram_encoder_wgrad.argtypes = [vp, vp, vp, vp]
    L.gram_flush.restype = C.c_int
    L.gram_flush.argtypes = [vp, vp, vp, vp, vp, i32p, vp]
    L.gram_window_end.restype = C.c_int
    L.gram_window_end.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32p, vp]
    L.gram_mlp_encode_gather.restype = C.c_int
    L.gram_mlp_encode_gather.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_int64, vp, vp, vp, vp]
    L.gram_mlp_batch_bytes.restype = C.c_int64
    L.gram_mlp_batch_bytes.argtypes = [vp, C.c_int64]
    L.gram_mlp_backward.restype = C.c_int
    L.gram_mlp_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_int64, vp, vp, vp, C.c_int32, vp, vp]
    L.gram_flush64.restype = C.c_int
    L.gram_flush64.argtypes = [vp, vp, vp, vp, vp, i32p, vp]
    L.gram_window_import.restype = C.c_int
    L.gram_window_import.argtypes = [vp, vp, vp, vp, C.c_int64, vp]
    L.gram_unique_static.restype = C.c_int
    L.gram_unique_static.argtypes = [vp, C.c_int64, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp]
    i32, i64, f32 = C.c_int32, C.c_int64, C.c_float
    acp, rp = C.POINTER(GramAttentionConfig), vp      # rp: the address of a GramRows
    L.gram_layer_norm.restype = C.c_int
    L.gram_layer_norm.argtypes = [vp, i32, vp, vp, vp, i64, i32, f32, vp, i32, vp, vp]
    L.gram_layer_norm_work_bytes.restype = i64
    L.gram_layer_norm_work_bytes.argtypes = [i64, i32]
    L.gram_layer_norm_backward.restype = C.c_int
    L.gram_layer_norm_backward.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, i64, i32, vp, vp, vp, vp, vp]
    L.gram_distance_bucket.restype = i32
    L.gram_distance_bucket.argtypes = [acp, i32]
    L.gram_attention.restype = C.c_int
    L.gram_attention.argtypes = [acp, i32, i32, rp, rp, rp, rp, vp, vp, vp, vp, vp]
    L.gram_attention_backward_bytes.restype = i64
    L.gram_attention_backward_bytes.argtypes = [acp, i32, i32]
    L.gram_attention_backward.restype = C.c_int
    L.gram_attention_backward.argtypes = [acp, i32, i32, rp, rp, rp, rp, vp, rp, rp, rp, rp, vp, vp, vp, vp, vp, vp]
    L.gram_attention_step_bytes.restype = i64
    L.gram_attention_step_bytes.argtypes = [acp, i32, i32]
    L.gram_attention_step.restype = C.c_int
    L.gram_attention_step.argtypes = [acp, i32, i32, rp, rp, rp, rp, rp, vp, vp, vp, rp, vp, vp]
    L.gram_check.restype = C.c_int
    L.gram_check.argtypes = [vp, vp]
    L.gram_last_error.restype = C.c_char_p
    L.gram_last_error.argtypes = [vp]
    L.gram_kernel_count.restype = C.c_int
    L.gram_kernel_count.argtypes = []
    L.gram_light_max.restype = C.c_int
    L.gram_light_max.argtypes = []
    L.gram_kernel_name.restype = C.c_char_p
    L.gram_kernel_name.argtypes = [C.c_int]
    L.gram_profile_enable.restype = C.c_int
    L.gram_profile_enable.argtypes = [vp, C.c_uint64, C.c_int32]
    L.gram_profile_read.restype = C.c_int
    L.gram_profile_read.argtypes = [vp, C.c_int, C.POINTER(C.c_int64), C.POINTER(C.c_double)]
    _lib = L
    return L


def make_config(vocab_n, d_in, d, max_positions, k_steps=1, pad_id=0, u_total_cap=0, xw_dtype=BF16,
                buffer_layout=0, d_hidden=0, h_dtype=F32):
    return GramConfig(int(vocab_n), int(d_in), int(d), int(max_positions), int(k_steps), int(pad_id),
                      int(u_total_cap), int(xw_dtype), int(buffer_layout), int(d_hidden), int(h_dtype))


def workspace_bytes(cfg: GramConfig) -> int:
    return load().gram_workspace_bytes(C.byref(cfg))


def _ptr(t):
    """Device (or NULL) pointer of a torch tensor / raw int."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _current_stream():
    """Handle of PyTorch's current stream on the current device.

    `torch.cuda.current_stream()` builds a Stream object, 2.8 us of a call that takes 5 to 8 us
    altogether (a small step makes five calls and is bound by the host); the handle itself takes 0.3 us.
    It comes from two functions of torch._C; a release without them gets the object.
    """
    import torch
    try:
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        pass
    return torch.cuda.current_stream().cuda_stream


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


UNIQUE_STATIC_MAX_POSITIONS = 262144


def unique_static(ids, vocab_n, pad_id, uniq, inverse, counts, u_dev, err_dev=None, m=None, stream=None):
    """gram_unique_static: the dedup step without a context and without any allocation."""
    L = load()
    rc = L.gram_unique_static(_ptr(ids), int(ids.numel() if m is None else m), int(vocab_n), int(pad_id),
                              _ptr(uniq), _ptr(inverse), _ptr(counts), _ptr(u_dev), _ptr(err_dev),
                              _stream(stream))
    if rc != OK:
        raise GramError(rc, (L.gram_last_error(None) or b"").decode())


# ---- the collaborative filter's layer: calls without a context --------------------------------------------
#
# A small batch is bound by the host here, so the checks below are kept short: a call takes 5 to 10 us.


def _ck_call(rc):
    if rc != OK:
        raise GramError(rc, (load().gram_last_error(None) or b"").decode())


def _refuse(message):
    raise GramError(ERR_ARG, message)


_INT_MAX = (1 << 31) - 1


def _int(v, what):
    """v as the library's 32-bit integers hold it: ctypes would wrap what does not fit."""
    v = int(v)
    if not -_INT_MAX <= v <= _INT_MAX:
        _refuse(f"{what}: {v} does not fit 32 bits")
    return v


def _size(v):
    """A size in a question about work buffers, -1 (which has none) where 32 bits do not hold it."""
    v = int(v)
    return v if v <= _INT_MAX else -1


def _device():
    """The current device's index, and -1 where there is none (host tensors are then refused like any other's)."""
    import torch
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -1


def _elements(t, what):
    import torch
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    _refuse(f"{what}: float32 or bfloat16 expected, got {t.dtype}")


def _flat(t, what, dtype, numel, dev):
    """Pointer of a contiguous tensor of that type and number of elements on device `dev` (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous():
        _refuse(f"{what}: a contiguous {dtype} tensor of {numel} elements expected, got {t.dtype} {tuple(t.shape)}")
    if not t.is_cuda or t.get_device() != dev:
        _refuse(f"{what}: not on the current device")
    return t.data_ptr()


def _work(t, what, size, dev):
    if t is None or t.numel() * t.element_size() < size or not t.is_contiguous():
        _refuse(f"{what}: a contiguous work buffer of at least {size} bytes expected")
    if not t.is_cuda or t.get_device() != dev:
        _refuse(f"{what}: not on the current device")
    return t.data_ptr()


def layer_norm_work_bytes(m, d):
    return int(load().gram_layer_norm_work_bytes(int(m), _size(d)))


def _norm_rows(x, y, what, dev):
    if x.dim() < 1 or y.shape != x.shape or not x.is_contiguous() or not y.is_contiguous():
        _refuse(f"{what}: two contiguous tensors of one shape expected, got {tuple(x.shape)} and {tuple(y.shape)}")
    if not x.is_cuda or x.get_device() != dev or not y.is_cuda or y.get_device() != dev:
        _refuse(f"{what}: not on the current device")
    d = x.shape[-1]
    if d > _INT_MAX:
        _refuse(f"{what}: a width that fits 32 bits expected, got {d}")
    return (x.numel() // d if d else 0), d


def layer_norm(x, weight, bias, y, stats=None, segments=None, eps=1e-5, stream=None):
    """gram_layer_norm: y = (x - mean) * rstd * weight + bias over the last dimension of x.  x and y are float32 or
    bfloat16, independently; stats ([rows, 2], float32) keeps mean and rstd for the backward pass; rows whose segment is
    negative are padding and become zero."""
    import torch
    L, dev, f32 = load(), _device(), torch.float32
    m, d = _norm_rows(x, y, "layer_norm: x and y", dev)
    _ck_call(L.gram_layer_norm(x.data_ptr(), _elements(x, "layer_norm: x"), _flat(weight, "layer_norm: weight", f32, d, dev),
                               _flat(bias, "layer_norm: bias", f32, d, dev),
                               _flat(segments, "layer_norm: segments", torch.int32, m, dev), m, d, eps, y.data_ptr(),
                               _elements(y, "layer_norm: y"), _flat(stats, "layer_norm: stats", f32, 2 * m, dev),
                               _stream(stream)))


def layer_norm_backward(x, weight, stats, dy, dx, dweight, dbias, work, segments=None, add=None, stream=None):
    """gram_layer_norm_backward: dx (float32, plus `add` where given), dweight and dbias of layer_norm; work:
    layer_norm_work_bytes(rows, d) bytes."""
    import torch
    what, L, dev, f32 = "layer_norm_backward: ", load(), _device(), torch.float32
    m, d = _norm_rows(x, dy, what + "x and dy", dev)
    _ck_call(L.gram_layer_norm_backward(
        x.data_ptr(), _elements(x, what + "x"), _flat(weight, what + "weight", f32, d, dev),
        _flat(stats, what + "stats", f32, 2 * m, dev), dy.data_ptr(), _elements(dy, what + "dy"),
        _flat(segments, what + "segments", torch.int32, m, dev), _flat(add, what + "add", f32, m * d, dev), m, d,
        _flat(dx, what + "dx", f32, m * d, dev), _flat(dweight, what + "dweight", f32, d, dev),
        _flat(dbias, what + "dbias", f32, d, dev), _work(work, what + "work", L.gram_layer_norm_work_bytes(m, d), dev),
        _stream(stream)))


class HistoryAttention:
    """Multi-head attention over item histories (gram_attention and its backward, gram_attention_step): the settings of
    a layer, which holds no device memory and may be used by any number of calls at once.

    q, o and their gradients are [batch, length, heads, head_dim] tensors, k and v [batch, length, kv_heads, head_dim],
    with any strides but a contiguous last dimension (views of a packed projection, a cache)."""

    def __init__(self, heads, kv_heads, head_dim, dtype=BF16, scale=None, cap=0.0, causal=True, buckets=0, max_distance=0,
                 two_sided=False):
        import torch
        self._lib = load()
        what = "gram_attention: settings"
        self.heads, self.kv_heads, self.head_dim, self.buckets = (_int(v, what) for v in (heads, kv_heads, head_dim, buckets))
        self.dtype = torch.bfloat16 if dtype == BF16 else torch.float32
        self.cfg = GramAttentionConfig(self.heads, self.kv_heads, self.head_dim, _int(dtype, what),
                                       max(float(head_dim), 1.0) ** -0.5 if scale is None else float(scale), float(cap),
                                       1 if causal else 0, self.buckets, _int(max_distance, what), 1 if two_sided else 0)
        self._cfg = C.byref(self.cfg)
        _ck_call(self._lib.gram_attention(self._cfg, 0, 0, None, None, None, None, None, None, None, None, None))

    def bucket(self, distance):
        """The bucket of the distance query position minus key position (-1 without a bias)."""
        return int(self._lib.gram_distance_bucket(self._cfg, max(-_INT_MAX, min(_INT_MAX, int(distance)))))

    def _operands(self, call, dev, *named):
        """gram_rows of the (name, tensor, shape) given, one after another; shapes of three dimensions have no rows."""
        out = []
        for name, t, shape in named:
            if t.shape != shape or t.dtype is not self.dtype:
                _refuse(f"{call}: {name}: {self.dtype} {list(shape)} expected, got {t.dtype} {list(t.shape)}")
            st = t.stride()
            if st[-1] != 1 and shape[-1] != 1:
                _refuse(f"{call}: {name}: a contiguous last dimension expected, got strides {st}")
            if not t.is_cuda or t.get_device() != dev:
                _refuse(f"{call}: {name}: not on the current device")
            out += (t.data_ptr(), st[0], st[1], st[2]) if len(st) == 4 else (t.data_ptr(), st[0], 0, st[1])
        return array("q", out)

    def _table(self, t, what, dev):
        import torch
        if (t is None) != (self.buckets == 0):
            _refuse(f"{what}: given exactly when the layer has buckets")
        return _flat(t, what, torch.float32, self.heads * self.buckets, dev)

    def forward(self, q, k, v, o, lse=None, segments=None, prefix=None, table=None, stream=None):
        """o = attention of q over k, v.  lse ([batch, heads, length], float32) is kept for the backward pass; segments
        (int32 [batch, length], negative: padding) and prefix (int32 [batch]) mask; table ([heads, buckets], float32)."""
        import torch
        if q.dim() != 4:
            _refuse("forward: q: [batch, length, heads, head_dim] expected")
        B, L, dev = q.shape[0], q.shape[1], _device()
        if B > _INT_MAX or L > _INT_MAX:
            _refuse("forward: batch and length that fit 32 bits expected")
        wide, shared = (B, L, self.heads, self.head_dim), (B, L, self.kv_heads, self.head_dim)
        rows = self._operands("forward", dev, ("q", q, wide), ("k", k, shared), ("v", v, shared), ("o", o, wide))
        at = rows.buffer_info()[0]
        _ck_call(self._lib.gram_attention(
            self._cfg, B, L, at, at + 32, at + 64, at + 96, _flat(segments, "forward: segments", torch.int32, B * L, dev),
            _flat(prefix, "forward: prefix", torch.int32, B, dev), self._table(table, "forward: table", dev),
            _flat(lse, "forward: lse", torch.float32, B * self.heads * L, dev), _stream(stream)))

    def backward_bytes(self, batch, length):
        return int(self._lib.gram_attention_backward_bytes(self._cfg, _size(batch), _size(length)))

    def backward(self, q, k, v, o, lse, do, dq, dk, dv, work, segments=None, prefix=None, table=None, dtable=None,
                 stream=None):
        """dq, dk, dv and, where given, dtable from the gradient `do` of o, at the operands and outputs of forward; work:
        backward_bytes(batch, length) bytes."""
        import torch
        if q.dim() != 4:
            _refuse("backward: q: [batch, length, heads, head_dim] expected")
        if dtable is not None and self.buckets == 0:
            _refuse("backward: dtable without buckets")
        B, L, dev, H, i32, f32 = q.shape[0], q.shape[1], _device(), self.heads, torch.int32, torch.float32
        if B > _INT_MAX or L > _INT_MAX:
            _refuse("backward: batch and length that fit 32 bits expected")
        wide, shared = (B, L, H, self.head_dim), (B, L, self.kv_heads, self.head_dim)
        rows = self._operands("backward", dev, ("q", q, wide), ("k", k, shared), ("v", v, shared), ("o", o, wide),
                              ("do", do, wide), ("dq", dq, wide), ("dk", dk, shared), ("dv", dv, shared))
        at = rows.buffer_info()[0]
        _ck_call(self._lib.gram_attention_backward(
            self._cfg, B, L, at, at + 32, at + 64, at + 96, _flat(lse, "backward: lse", f32, B * H * L, dev), at + 128, at + 160,
            at + 192, at + 224, _flat(segments, "backward: segments", i32, B * L, dev),
            _flat(prefix, "backward: prefix", i32, B, dev), self._table(table, "backward: table", dev),
            _flat(dtable, "backward: dtable", f32, H * self.buckets, dev),
            _work(work, "backward: work", self._lib.gram_attention_backward_bytes(self._cfg, B, L), dev), _stream(stream)))

    def step_bytes(self, batch, capacity):
        return int(self._lib.gram_attention_step_bytes(self._cfg, _size(batch), _size(capacity)))

    def step(self, q, k_new, v_new, k_cache, v_cache, lengths, o, work, first=None, table=None, stream=None):
        """One new item per history: k_new, v_new ([batch, kv_heads, head_dim]) are written to row lengths[b] of the
        caches ([batch, capacity, kv_heads, head_dim]) and q ([batch, heads, head_dim]) attends to rows first[b] to
        lengths[b]; work: step_bytes(batch, capacity) bytes."""
        import torch
        if q.dim() != 3 or k_cache.dim() != 4:
            _refuse("step: q [batch, heads, head_dim] and caches [batch, capacity, kv_heads, head_dim] expected")
        B, rows_max, dev, KV, D = q.shape[0], k_cache.shape[1], _device(), self.kv_heads, self.head_dim
        if B > _INT_MAX or rows_max > _INT_MAX:
            _refuse("step: batch and capacity that fit 32 bits expected")
        wide, new, cache = (B, self.heads, D), (B, KV, D), (B, rows_max, KV, D)
        rows = self._operands("step", dev, ("q", q, wide), ("k_new", k_new, new), ("v_new", v_new, new),
                              ("k_cache", k_cache, cache), ("v_cache", v_cache, cache), ("o", o, wide))
        at = rows.buffer_info()[0]
        _ck_call(self._lib.gram_attention_step(
            self._cfg, B, rows_max, at, at + 32, at + 64, at + 96, at + 128, _flat(lengths, "step: lengths", torch.int32, B, dev),
            _flat(first, "step: first", torch.int32, B, dev), self._table(table, "step: table", dev), at + 160,
            _work(work, "step: work", self._lib.gram_attention_step_bytes(self._cfg, B, rows_max), dev), _stream(stream)))


class Gram:
    """A context of the library.  Tensor arguments are CUDA(HIP) torch tensors,
    contiguous, of the dtypes include/gram.h states; they are passed by pointer."""

    def __init__(self, cfg: GramConfig):
        self._lib = load()
        self.cfg = cfg
        self._h = C.c_void_p()
        rc = self._lib.gram_create(C.byref(self._h), C.byref(cfg))
        if rc != OK:
            raise GramError(rc, (self._lib.gram_last_error(None) or b"").decode())

    def _ck(self, rc):
        if rc != OK:
            raise GramError(rc, (self._lib.gram_last_error(self._h) or b"").decode())

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.gram_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def unique(self, ids, uniq, inverse, counts, u_dev=None, want_host_u=False, stream=None):
        m = ids.numel() if not isinstance(ids, int) else None
        u_host = C.c_int32(-1)
        self._ck(self._lib.gram_unique(self._h, _ptr(ids), m, _ptr(uniq), _ptr(inverse), _ptr(counts),
                                       _ptr(u_dev), C.byref(u_host) if want_host_u else None,
                                       _stream(stream)))
        return u_host.value if want_host_u else None

    def encode_gather(self, X, W, uniq, inverse, u_dev, m, E, H, stream=None):
        self._ck(self._lib.gram_encode_gather(self._h, _ptr(X), _ptr(W), _ptr(uniq), _ptr(inverse),
                                              _ptr(u_dev), int(m), _ptr(E), _ptr(H), _stream(stream)))

    def grad_accumulate(self, dH, m, step_k, stream=None):
        self._ck(self._lib.gram_grad_accumulate(self._h, _ptr(dH), int(m), int(step_k), _stream(stream)))

    def pseudo_target(self, E, Ht=None, loss_dev=None, stream=None):
        self._ck(self._lib.gram_pseudo_target(self._h, _ptr(E), _ptr(Ht), _ptr(loss_dev), _stream(stream)))

    def gather(self, src, inverse, m, H, stream=None):
        self._ck(self._lib.gram_gather(self._h, _ptr(src), _ptr(inverse), int(m), _ptr(H), _stream(stream)))

    def encoder_wgrad(self, X, dW, stream=None):
        self._ck(self._lib.gram_encoder_wgrad(self._h, _ptr(X), _ptr(dW), _stream(stream)))

    def encoder_wgrad_chunk(self, X, dW, first_row, n_rows, accumulate, stream=None):
        self._ck(self._lib.gram_encoder_wgrad_chunk(self._h, _ptr(X), _ptr(dW), int(first_row), int(n_rows),
                                                    1 if accumulate else 0, _stream(stream)))

    def pseudo_loss_grad(self, X, W, ids, Ht, n, R, dW, accumulate=False, loss_dev=None, stream=None):
        self._ck(self._lib.gram_pseudo_loss_grad(self._h, _ptr(X), _ptr(W), _ptr(ids), _ptr(Ht), int(n),
                                                 _ptr(R), _ptr(dW), 1 if accumulate else 0,
                                                 _ptr(loss_dev), _stream(stream)))

    def flush(self, uniq_total=None, counts_total=None, G_total=None, u_total_dev=None,
              want_host_u=False, stream=None):
        u_host = C.c_int32(-1)
        self._ck(self._lib.gram_flush(self._h, _ptr(uniq_total), _ptr(counts_total), _ptr(G_total),
                                      _ptr(u_total_dev), C.byref(u_host) if want_host_u else None,
                                      _stream(stream)))
        return u_host.value if want_host_u else None

    def window_end(self, X, dW, uniq_total=None, counts_total=None, G_total=None, u_total_dev=None,
                   want_host_u=False, stream=None):
        u_host = C.c_int32(-1)
        self._ck(self._lib.gram_window_end(self._h, _ptr(X), _ptr(dW), _ptr(uniq_total), _ptr(counts_total),
                                           _ptr(G_total), _ptr(u_total_dev),
                                           C.byref(u_host) if want_host_u else None, _stream(stream)))
        return u_host.value if want_host_u else None

    def mlp_encode_gather(self, X, W1, W2, uniq, inverse, u_dev, m, A1, E, H, stream=None):
        self._ck(self._lib.gram_mlp_encode_gather(self._h, _ptr(X), _ptr(W1), _ptr(W2), _ptr(uniq), _ptr(inverse),
                                                  _ptr(u_dev), int(m), _ptr(A1), _ptr(E), _ptr(H),
                                                  _stream(stream)))

    def mlp_batch_bytes(self, n):
        return int(self._lib.gram_mlp_batch_bytes(self._h, int(n)))

    def mlp_backward(self, X, W1, W2, ids, G_rows, Ht, n, work, dW1, dW2, accumulate=False, loss_dev=None,
                     stream=None):
        self._ck(self._lib.gram_mlp_backward(self._h, _ptr(X), _ptr(W1), _ptr(W2), _ptr(ids), _ptr(G_rows),
                                             _ptr(Ht), int(n), _ptr(work), _ptr(dW1), _ptr(dW2),
                                             1 if accumulate else 0, _ptr(loss_dev), _stream(stream)))

    def flush64(self, uniq_total=None, counts_total=None, G_total=None, u_total_dev=None,
                want_host_u=False, stream=None):
        u_host = C.c_int32(-1)
        self._ck(self._lib.gram_flush64(self._h, _ptr(uniq_total), _ptr(counts_total), _ptr(G_total),
                                        _ptr(u_total_dev), C.byref(u_host) if want_host_u else None,
                                        _stream(stream)))
        return u_host.value if want_host_u else None

    def window_import(self, ids, counts, G_rows, n, stream=None):
        self._ck(self._lib.gram_window_import(self._h, _ptr(ids), _ptr(counts), _ptr(G_rows), int(n),
                                              _stream(stream)))

    def light_max(self):
        return int(self._lib.gram_light_max())

    def kernel_names(self):
        return [self._lib.gram_kernel_name(k).decode() for k in range(self._lib.gram_kernel_count())]

    def profile_enable(self, kernels=None, max_launches=8192):
        """Time the named kernels (all if None, none if empty) with HIP events."""
        names = self.kernel_names()
        mask = 0
        for k, nm in enumerate(names):
            if kernels is None or nm in kernels:
                mask |= 1 << k
        self._ck(self._lib.gram_profile_enable(self._h, mask, max_launches if mask else 0))

    def profile_read(self):
        """{kernel: (launches, total_ms)} of the timed launches so far."""
        out = {}
        for k, nm in enumerate(self.kernel_names()):
            n, ms = C.c_int64(0), C.c_double(0.0)
            self._ck(self._lib.gram_profile_read(self._h, k, C.byref(n), C.byref(ms)))
            if n.value:
                out[nm] = (n.value, ms.value)
        return out

    def check(self, stream=None):
        self._ck(self._lib.gram_check(self._h, _stream(stream)))
