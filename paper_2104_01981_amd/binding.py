"""Thin ctypes binding of libecrm.so: argument marshalling only.

Every step of the update path runs in the library's HIP kernels; torch is used for device memory
and streams.  The library must have been built (paper_2104_01981_amd/build.py); there is no CPU
fallback, and a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os

ECRM_OK, ECRM_EINVAL, ECRM_ENOTBOUND, ECRM_ESCRATCH, ECRM_EBATCH, ECRM_EKEYRANGE, ECRM_EHIP = 0, -1, -2, -3, -4, -5, -6
ECRM_EBUFFER, ECRM_ESTATE = -7, -8
ECRM_PHASES = 3

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("ECRM_LIBRARY") or os.path.join(_HERE, "libecrm.so")
_lib = None

SYMBOLS = ["ecrm_create", "ecrm_destroy", "ecrm_data_bytes", "ecrm_parity_bytes", "ecrm_scratch_bytes", "ecrm_update_scratch_bytes",
           "ecrm_bind", "ecrm_encode", "ecrm_route", "ecrm_update", "ecrm_update_static", "ecrm_status", "ecrm_clear_status",
           "ecrm_tune", "ecrm_probe_row_traffic", "ecrm_profile", "ecrm_profile_read", "ecrm_batch_stats", "ecrm_host_placement", "ecrm_strerror",
           "ecrm_fail_server", "ecrm_recover_server", "ecrm_degraded_read",
           "ecrm_recovery_begin", "ecrm_recovery_lock", "ecrm_recovery_decode", "ecrm_recovery_unlock",
           "ecrm_recovery_state", "ecrm_recovery_read",
           "ecrm_embed", "ecrm_embed_grad", "ecrm_embed_grad_dense",
           "ecrm_dropout", "ecrm_embed_dropout", "ecrm_embed_grad_dropout", "ecrm_embed_grad_dense_dropout",
           "ecrm_ffn_create", "ecrm_ffn_destroy", "ecrm_ffn_bytes", "ecrm_ffn_bind", "ecrm_ffn_forward", "ecrm_ffn_backward",
           "ecrm_grads_create", "ecrm_grads_destroy", "ecrm_grads_bytes", "ecrm_grads_bind", "ecrm_grads_norm", "ecrm_grads_clip"]


class EcrmConfig(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("dim", C.c_uint32), ("k", C.c_uint32), ("servers", C.c_uint32),
                ("optimizer", C.c_uint32), ("lr", C.c_float), ("eps", C.c_float), ("max_batch", C.c_uint64),
                ("momentum", C.c_float), ("combine", C.c_uint32), ("propagation", C.c_uint32)]


class EcrmTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("elements", C.c_uint64), ("rows", C.c_void_p), ("row_elements", C.c_uint32),
                ("type", C.c_uint32)]


class EcrmMask(C.Structure):
    _fields_ = [("state", C.c_void_p), ("offset", C.c_uint64), ("p", C.c_double)]


class EcrmFfnConfig(C.Structure):
    _fields_ = [("dim", C.c_uint32), ("hidden", C.c_uint32), ("type", C.c_uint32), ("activation", C.c_uint32),
                ("max_rows", C.c_uint64), ("training", C.c_uint32)]


class EcrmError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {strerror(code)} ({code})")


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libecrm.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python paper_2104_01981_amd/build.py`")
        lib = C.CDLL(_LIB_PATH)
        vp, u64p, u32p, f32p = C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p
        lib.ecrm_create.argtypes = [C.POINTER(EcrmConfig), C.POINTER(C.c_void_p)]
        lib.ecrm_destroy.argtypes = [vp]
        lib.ecrm_destroy.restype = None
        for name in ("ecrm_data_bytes", "ecrm_parity_bytes", "ecrm_scratch_bytes", "ecrm_update_scratch_bytes"):
            getattr(lib, name).argtypes = [vp]
            getattr(lib, name).restype = C.c_size_t
        lib.ecrm_bind.argtypes = [vp, f32p, f32p, f32p, f32p, u64p, u64p, vp, C.c_size_t]
        lib.ecrm_encode.argtypes = [vp, vp]
        lib.ecrm_route.argtypes = [vp, u64p, C.c_uint64, u64p, u32p, u32p, u32p, vp]
        lib.ecrm_update.argtypes = [vp, u64p, f32p, C.c_uint64, vp]
        lib.ecrm_update_static.argtypes = [vp, f32p, f32p, f32p, f32p, u64p, u64p, u64p, f32p, C.c_uint64, u32p, vp]
        lib.ecrm_fail_server.argtypes = [vp, C.c_uint32, vp]
        lib.ecrm_recover_server.argtypes = [vp, C.c_uint32, vp]
        lib.ecrm_degraded_read.argtypes = [vp, u64p, C.c_uint64, C.c_uint32, f32p, f32p, vp]
        lib.ecrm_recovery_begin.argtypes = [vp, C.c_uint32, C.c_uint32, u64p, f32p, C.c_uint64, vp]
        lib.ecrm_recovery_read.argtypes = [vp, u64p, C.c_uint64, f32p, f32p, vp]
        lib.ecrm_recovery_lock.argtypes = [vp]
        lib.ecrm_recovery_decode.argtypes = [vp, vp]
        lib.ecrm_recovery_unlock.argtypes = [vp, vp]
        lib.ecrm_recovery_state.argtypes = [vp, vp, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32),
                                            C.POINTER(C.c_uint32), C.POINTER(C.c_uint64)]
        lib.ecrm_status.argtypes = [vp, vp]
        lib.ecrm_clear_status.argtypes = [vp, vp]
        lib.ecrm_tune.argtypes = [vp, C.c_int, C.c_uint64]
        lib.ecrm_probe_row_traffic.argtypes = [vp, vp, C.c_uint64, vp, C.c_uint64, C.c_int, vp, vp]
        lib.ecrm_profile.argtypes = [vp, C.c_int]
        lib.ecrm_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_uint64)]
        lib.ecrm_batch_stats.argtypes = [vp, vp, C.POINTER(C.c_uint64)]
        lib.ecrm_host_placement.argtypes = [vp, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint32,
                                            C.POINTER(C.c_uint32)]
        u64, u32, f32 = C.c_uint64, C.c_uint32, C.c_float
        lib.ecrm_embed.argtypes = [vp, u64p, u64, u64, f32, u32, vp, u32, u64, vp]
        lib.ecrm_embed_grad.argtypes = [vp, u64p, vp, u32, u64, u64, u64, f32, u64p, f32p, u64p, vp]
        lib.ecrm_embed_grad_dense.argtypes = [vp, u64p, vp, u32, u64, u64, u64, f32, f32p, C.c_int, vp]
        lib.ecrm_grads_create.argtypes = [C.POINTER(EcrmTensor), u32, C.POINTER(C.c_void_p)]
        lib.ecrm_grads_destroy.argtypes = [vp]
        lib.ecrm_grads_destroy.restype = None
        lib.ecrm_grads_bytes.argtypes = [vp]
        lib.ecrm_grads_bytes.restype = C.c_size_t
        lib.ecrm_grads_bind.argtypes = [vp, vp, C.c_size_t, vp]
        lib.ecrm_grads_norm.argtypes = [vp, f32p, vp]
        lib.ecrm_grads_clip.argtypes = [vp, vp, f32p, f32, vp]
        mask = C.POINTER(EcrmMask)
        lib.ecrm_dropout.argtypes = [mask, vp, u64, vp, u64, vp, u64, u32, u64, u32, vp]
        lib.ecrm_embed_dropout.argtypes = [vp, u64p, u64, u64, f32, u32, mask, vp, u32, u64, vp]
        lib.ecrm_embed_grad_dropout.argtypes = [vp, u64p, vp, u32, u64, u64, u64, f32, mask, u64p, f32p, u64p, vp]
        lib.ecrm_embed_grad_dense_dropout.argtypes = [vp, u64p, vp, u32, u64, u64, u64, f32, mask, f32p, C.c_int, vp]
        lib.ecrm_ffn_create.argtypes = [C.POINTER(EcrmFfnConfig), C.POINTER(C.c_void_p)]
        lib.ecrm_ffn_destroy.argtypes = [vp]
        lib.ecrm_ffn_destroy.restype = None
        lib.ecrm_ffn_bytes.argtypes = [vp]
        lib.ecrm_ffn_bytes.restype = C.c_size_t
        lib.ecrm_ffn_bind.argtypes = [vp, vp, u64, vp, u64, vp, u64, vp, C.c_size_t]
        lib.ecrm_ffn_forward.argtypes = [vp, vp, u64, u64, vp, u64, mask, vp, u64, vp, vp]
        lib.ecrm_ffn_backward.argtypes = [vp, vp, u64, vp, vp, u64, u64, mask, vp, u64, vp, u64, vp, vp, vp, u32, C.c_int, vp]
        lib.ecrm_strerror.argtypes = [C.c_int]
        lib.ecrm_strerror.restype = C.c_char_p
        _lib = lib
    return _lib


def strerror(code: int) -> str:
    return load_library().ecrm_strerror(code).decode()


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


_raw_stream = _raw_device = None


def _stream(stream):
    """Address of a stream, by default the current device's current one.  (As a torch.cuda.Stream object, the current one takes
    2.7 us to get, a third of a short call; its address alone 0.1.)"""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch
        of, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if of and device:
            _raw_stream = lambda: of(device())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return _raw_stream()


def _current_device():
    """Index of the current device (of torch.cuda.current_device, without its checks)."""
    global _raw_device
    if _raw_device is None:
        import torch
        _raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _raw_device()


def _stream_object(stream):
    """The torch stream of a call: the one given, which may be any object with an address, or the current one."""
    import torch
    if stream is None:
        return torch.cuda.current_stream()
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)


def probe_row_traffic(table_a, table_b, table_rows, rows, write, sink, stream=None):
    """ecrm_probe_row_traffic (measurement aid): rows of 128 floats at rows[i], alternately from the two tables."""
    rc = load_library().ecrm_probe_row_traffic(_ptr(table_a), _ptr(table_b), C.c_uint64(table_rows), _ptr(rows),
                                               C.c_uint64(rows.numel()), C.c_int(1 if write else 0), _ptr(sink),
                                               _stream(stream))
    if rc != ECRM_OK:
        raise EcrmError(rc, "ecrm_probe_row_traffic")


_NO_PADDING = 1 << 63
_types, _words = {}, set()


def _type(t):
    """ECRM_F32, ECRM_BF16 or ECRM_F16 of a tensor."""
    if not _types:
        import torch
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    return _types[t.dtype]


def _is_words(t):
    """Contiguous 64-bit integers in device memory?"""
    if not _words:
        import torch
        _words.update({torch.int64, torch.uint64})
    return t.is_cuda and t.dtype in _words and t.is_contiguous()


def _key(padding):
    """A padding token as the library takes it: negative ones as the unsigned value with the same bits."""
    return _NO_PADDING if padding is None else padding & 0xFFFFFFFFFFFFFFFF


def _row(t):
    """Elements from one row to the next; of a single row torch may say anything."""
    return t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 4) * 4


class Grads:
    """A list of gradient tensors: their global norm, and clipping (ecrm_grads_<name>).  An item is a contiguous tensor, or a
    pair (rows of a gradient [n, D], device tensor with the number of rows that count).  The tensors are kept alive, and
    have to stay where they are; make a new list when they move.  The list is written on `stream`: order its use on other streams
    behind that.  It may be dropped while calls are still to run, on whatever streams; a graph that uses it needs it kept."""

    def __init__(self, tensors, stream=None):
        import torch
        self._lib = load_library()
        self._grads = C.c_void_p(0)
        items = [t if isinstance(t, (tuple, list)) else (t, None) for t in tensors]
        assert items, "a list of at least one tensor"
        table = (EcrmTensor * len(items))()
        for to, (t, rows) in zip(table, items):
            assert t.is_cuda and t.is_contiguous()
            to.data, to.elements, to.type = t.data_ptr(), t.numel(), _type(t)
            if rows is not None:
                assert _is_words(rows) and rows.numel() == 1 and t.dim() == 2
                to.rows, to.row_elements = rows.data_ptr(), t.shape[1]
        rc = self._lib.ecrm_grads_create(table, C.c_uint32(len(items)), C.byref(self._grads))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_grads_create")
        size = self._lib.ecrm_grads_bytes(self._grads)
        with torch.cuda.stream(_stream_object(stream)):  # memory that stream has done with
            self._keep = (items, torch.empty(size, dtype=torch.uint8, device=items[0][0].device))
        self._streams = set()
        rc = self._lib.ecrm_grads_bind(self._grads, _ptr(self._keep[1]), C.c_size_t(size), self._on(stream))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_grads_bind")

    def _on(self, stream):
        """Address of a call's stream.  The allocator learns that the list's memory is used there: who drops the list may hold
        nothing else of it, and the memory has to wait for what that stream has still to run."""
        address = _stream(stream)
        if address not in self._streams:
            self._streams.add(address)
            use = _stream_object(stream)
            items, table = self._keep
            for t in [table] + [t for item in items for t in item if t is not None]:
                t.record_stream(use)
        return address

    def destroy(self):
        if self._grads:
            self._lib.ecrm_grads_destroy(self._grads)
            self._grads = C.c_void_p(0)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def norm(self, norm, stream=None, check=True):
        """norm: device tensor of one fp32 value."""
        assert norm.is_cuda and _type(norm) == 0 and norm.numel() == 1
        rc = self._lib.ecrm_grads_norm(self._grads, norm.data_ptr(), self._on(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_grads_norm")
        return rc

    def clip(self, norm, max_norm, out=None, stream=None, check=True):
        """In place, or into the tensors of `out`, another list."""
        assert norm.is_cuda and _type(norm) == 0 and norm.numel() == 1
        if out is not None and not out._grads:           # destroyed: NULL would be "in place"
            rc = ECRM_EINVAL
        else:
            if out is not None:
                out._on(stream)
            rc = self._lib.ecrm_grads_clip(self._grads, out._grads if out is not None else None, norm.data_ptr(), max_norm, self._on(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_grads_clip")
        return rc


class Dropout:
    """The masks of one place of a model (ecrm_mask): probability, device tensor of two 64-bit integers -- a seed and the number of masks
    drawn before, which the program adds to, once a step -- and the place's offset among those of a step.  The state is kept alive; it and
    the object may be dropped while calls are still to run, on whatever streams; a graph that draws from it needs it kept."""

    def __init__(self, p, state, offset=0):
        assert _is_words(state) and state.numel() == 2
        self._lib = load_library()
        self.state, self._device = state, state.get_device()
        self.mask = EcrmMask(state.data_ptr(), offset & 0xFFFFFFFFFFFFFFFF, p)
        self._streams = set()

    def _on(self, address, stream):
        """The mask, for a call on that stream: the allocator learns that the state is read there."""
        if address not in self._streams:
            self._streams.add(address)
            self.state.record_stream(_stream_object(stream))
        return self.mask

    def apply(self, x, out, residual=None, stream=None, check=True):
        """out = residual + dropout(x); the gradient of x is apply(gradient of out).  x, out, residual: [rows, cols] of fp32, bf16 or
        fp16, rows at any multiple of 4 elements from each other; out may be x or residual."""
        shape, t = x.shape, x.dtype
        device = self._device
        assert len(shape) == 2 and out.shape == shape and out.dtype == t
        assert x.get_device() == out.get_device() == device == _current_device(), "all on the current device"
        rows, cols = shape
        assert rows == 0 or cols < 2 or (x.stride(1) == 1 and out.stride(1) == 1)
        assert residual is None or _is_rows(residual, rows, cols, t, device)
        address = _stream(stream)
        if address not in self._streams:                 # as _on, without a call
            self._on(address, stream)
        rc = self._lib.ecrm_dropout(self.mask, x.data_ptr(), _row(x), *_optional(residual), out.data_ptr(), _row(out), _type(x),
                                    rows, cols, address)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_dropout")
        return rc


def _is_rows(t, rows, cols, dtype, device):
    """A matrix in that device's memory whose rows have their elements side by side?"""
    return (t.get_device() == device and t.dim() == 2 and t.shape[0] == rows and t.shape[1] == cols and t.dtype == dtype
            and (rows == 0 or cols < 2 or t.stride(1) == 1))


def _optional(t):
    """Address and distance of the rows of a matrix that need not be there."""
    return (None, 0) if t is None else (t.data_ptr(), _row(t))


class FeedForward:
    """A gated feed-forward block (ecrm_ffn_<name>) with the weights gate, up [hidden, dim] and down [dim, hidden], which are kept alive
    and have to stay where they are.  activation: "silu", "gelu" or "relu".  Its workspace, for calls of up to max_rows rows and, with
    training, the backward pass, may be another block's (workspace=other.workspace) if no two calls on them overlap in time; one of the same
    type that is no smaller in dim, hidden and max_rows, and trains if this one does, has a workspace that is large enough.  The block
    may be dropped while calls are still to run, on whatever streams; a graph that uses it needs it kept."""

    ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}

    def __init__(self, gate, up, down, max_rows, activation="silu", training=False, workspace=None, stream=None):
        import torch
        self._lib = load_library()
        self._ffn = C.c_void_p(0)
        self.hidden, self.dim = gate.shape
        self.dtype, self.max_rows = gate.dtype, max_rows
        self._device = device = torch.cuda.current_device()
        assert _is_rows(gate, self.hidden, self.dim, self.dtype, device) and _is_rows(up, self.hidden, self.dim, self.dtype, device)
        assert _is_rows(down, self.dim, self.hidden, self.dtype, device)
        cfg = EcrmFfnConfig(self.dim, self.hidden, _type(gate), self.ACTIVATIONS[activation], max_rows, 1 if training else 0)
        rc = self._lib.ecrm_ffn_create(C.byref(cfg), C.byref(self._ffn))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_ffn_create")
        if workspace is None:
            with torch.cuda.stream(_stream_object(stream)):  # memory that stream has done with
                workspace = torch.empty(self.workspace_bytes(), dtype=torch.uint8, device=gate.device)
        assert workspace.is_cuda and workspace.is_contiguous() and workspace.device == gate.device
        self.workspace = workspace
        self._keep, self._streams = (gate, up, down, workspace), set()
        rc = self._lib.ecrm_ffn_bind(self._ffn, gate.data_ptr(), _row(gate), up.data_ptr(), _row(up), down.data_ptr(), _row(down),
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size())
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_ffn_bind")

    def workspace_bytes(self):
        return self._lib.ecrm_ffn_bytes(self._ffn)

    def _on(self, stream):
        """Address of a call's stream; the allocator learns that weights and workspace are used there."""
        address = _stream(stream)
        assert _current_device() == self._device, "the block's device has to be the current one"
        if address not in self._streams:
            self._streams.add(address)
            use = _stream_object(stream)
            for t in self._keep:
                t.record_stream(use)
        return address

    def destroy(self):
        if self._ffn:
            self._lib.ecrm_ffn_destroy(self._ffn)
            self._ffn = C.c_void_p(0)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def forward(self, x, out, residual=None, dropout=None, saved=None, stream=None, check=True):
        """out = residual + dropout(block(x)); x, out, residual: [n, dim], rows at any multiple of 4 elements from each other; out may be
        x or residual.  saved [n, 2 * hidden]: what the backward pass needs."""
        n, t, device = x.shape[0], self.dtype, self._device
        assert _is_rows(x, n, self.dim, t, device) and _is_rows(out, n, self.dim, t, device)
        assert residual is None or _is_rows(residual, n, self.dim, t, device)
        assert saved is None or (_is_rows(saved, n, 2 * self.hidden, t, device) and saved.is_contiguous())
        assert dropout is None or dropout._device == device
        address = self._on(stream)
        rc = self._lib.ecrm_ffn_forward(self._ffn, x.data_ptr(), _row(x), n, *_optional(residual),
                                        dropout._on(address, stream) if dropout else None, out.data_ptr(), _row(out),
                                        saved.data_ptr() if saved is not None else None, address)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_ffn_forward")
        return rc

    def backward(self, x, saved, d_out, d_x=None, d_gate=None, d_up=None, d_down=None, add=None, dropout=None, accumulate=False,
                 stream=None, check=True):
        """x, saved, dropout: the forward call's.  d_x = add + gradient of x (add: d_out where the residual was x); d_x may be add or d_out.
        d_gate, d_up, d_down: contiguous, of the block's type or fp32, all or none; accumulate: added to."""
        n, t, device = x.shape[0], self.dtype, self._device
        assert _is_rows(x, n, self.dim, t, device) and _is_rows(d_out, n, self.dim, t, device)
        assert _is_rows(saved, n, 2 * self.hidden, t, device) and saved.is_contiguous()
        assert d_x is None or _is_rows(d_x, n, self.dim, t, device)
        assert add is None or _is_rows(add, n, self.dim, t, device)
        weights = [w for w in (d_gate, d_up, d_down) if w is not None]
        assert all(w.get_device() == device and w.is_contiguous() and w.dtype == weights[0].dtype for w in weights)
        assert d_gate is None or tuple(d_gate.shape) == (self.hidden, self.dim)
        assert d_up is None or tuple(d_up.shape) == (self.hidden, self.dim)
        assert d_down is None or tuple(d_down.shape) == (self.dim, self.hidden)
        assert dropout is None or dropout._device == device
        address = self._on(stream)
        rc = self._lib.ecrm_ffn_backward(self._ffn, x.data_ptr(), _row(x), saved.data_ptr(), d_out.data_ptr(), _row(d_out), n,
                                         dropout._on(address, stream) if dropout else None, *_optional(add), *_optional(d_x),
                                         *[w.data_ptr() if w is not None else None for w in (d_gate, d_up, d_down)],
                                         _type(weights[0]) if weights else 0, 1 if accumulate else 0, address)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_ffn_backward")
        return rc


class Ecrm:
    """One context of the library.  Method names mirror the C entry points (ecrm_<name>)."""

    def __init__(self, rows, dim=128, k=4, servers=5, lr=0.01, eps=1e-8, max_batch=1 << 20, optimizer=0,
                 momentum=0.0, combine=0, propagation=0):
        self._lib = load_library()
        self.cfg = EcrmConfig(rows, dim, k, servers, optimizer, lr, eps, max_batch, momentum, combine, propagation)
        self._ctx = C.c_void_p(0)
        rc = self._lib.ecrm_create(C.byref(self.cfg), C.byref(self._ctx))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_create")
        self._keep = None

    def destroy(self):
        if self._ctx:
            self._lib.ecrm_destroy(self._ctx)
            self._ctx = C.c_void_p(0)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def data_bytes(self):
        return self._lib.ecrm_data_bytes(self._ctx)

    def parity_bytes(self):
        return self._lib.ecrm_parity_bytes(self._ctx)

    def scratch_bytes(self):
        return self._lib.ecrm_scratch_bytes(self._ctx)

    def update_scratch_bytes(self):
        """What is enough for a context whose gradient calls (embed_grad, embed_grad_dense) are not used."""
        return self._lib.ecrm_update_scratch_bytes(self._ctx)

    def bind_raw(self, E, A, PE, PA, load_data, load_parity, scratch, scratch_bytes):
        """ecrm_bind with raw integer addresses (for error-path tests)."""
        return self._lib.ecrm_bind(self._ctx, C.c_void_p(E), C.c_void_p(A), C.c_void_p(PE), C.c_void_p(PA),
                                   C.c_void_p(load_data), C.c_void_p(load_parity), C.c_void_p(scratch),
                                   C.c_size_t(scratch_bytes))

    def bind(self, E, A, PE, PA, load_data, load_parity, scratch):
        import torch
        R, D, k, S = self.cfg.rows, self.cfg.dim, self.cfg.k, self.cfg.servers
        for t, shape in ((E, (R, D)), (A, (R, D)), (PE, (R // k, D)), (PA, (R // k, D))):
            assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == shape
        for t in (load_data, load_parity):
            assert t.is_cuda and t.dtype in (torch.int64, torch.uint64) and t.numel() == S and t.is_contiguous()
        assert scratch.is_cuda and scratch.dtype == torch.uint8 and scratch.is_contiguous()
        rc = self._lib.ecrm_bind(self._ctx, _ptr(E), _ptr(A), _ptr(PE), _ptr(PA), _ptr(load_data),
                                 _ptr(load_parity), _ptr(scratch), C.c_size_t(scratch.numel()))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_bind")
        self._keep = (E, A, PE, PA, load_data, load_parity, scratch)

    def drop_buffers(self):
        """Python side only: stop keeping the bound tensors alive (bind again before any further call)."""
        self._keep = None

    def encode(self, stream=None):
        rc = self._lib.ecrm_encode(self._ctx, _stream(stream))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_encode")

    def route(self, keys, stripe=None, member=None, data_srv=None, parity_srv=None, stream=None):
        rc = self._lib.ecrm_route(self._ctx, _ptr(keys), C.c_uint64(keys.numel()), _ptr(stripe), _ptr(member),
                                  _ptr(data_srv), _ptr(parity_srv), _stream(stream))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_route")

    def update(self, keys, grads, n=None, stream=None, check=True):
        n = keys.numel() if n is None else n
        rc = self._lib.ecrm_update(self._ctx, _ptr(keys), _ptr(grads), C.c_uint64(n), _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_update")
        return rc

    def update_static(self, E, A, PE, PA, load_data, load_parity, keys, grads, n=None, rejected=None, stream=None,
                      check=True):
        """ecrm_update_static: the library's own fixed scratch array, tables passed per call."""
        n = keys.numel() if n is None else n
        rc = self._lib.ecrm_update_static(self._ctx, _ptr(E), _ptr(A), _ptr(PE), _ptr(PA), _ptr(load_data),
                                          _ptr(load_parity), _ptr(keys), _ptr(grads), C.c_uint64(n), _ptr(rejected),
                                          _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_update_static")
        return rc

    def fail_server(self, server, stream=None):
        rc = self._lib.ecrm_fail_server(self._ctx, C.c_uint32(server), _stream(stream))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_fail_server")

    def recover_server(self, server, stream=None):
        rc = self._lib.ecrm_recover_server(self._ctx, C.c_uint32(server), _stream(stream))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recover_server")

    def degraded_read(self, keys, lost_server, out_E, out_A=None, stream=None, check=True):
        lost = 0xFFFFFFFF if lost_server is None else lost_server
        rc = self._lib.ecrm_degraded_read(self._ctx, _ptr(keys), C.c_uint64(keys.numel()), C.c_uint32(lost),
                                          _ptr(out_E), _ptr(out_A), _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_degraded_read")
        return rc

    def recovery_read(self, keys, out_E, out_A=None, stream=None, check=True):
        rc = self._lib.ecrm_recovery_read(self._ctx, _ptr(keys), C.c_uint64(keys.numel()), _ptr(out_E), _ptr(out_A),
                                          _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recovery_read")
        return rc

    def recovery_begin(self, server, chunks, buf_keys, buf_grads, capacity, stream=None, check=True):
        rc = self._lib.ecrm_recovery_begin(self._ctx, C.c_uint32(server), C.c_uint32(chunks), _ptr(buf_keys),
                                           _ptr(buf_grads), C.c_uint64(capacity), _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recovery_begin")
        self._keep_rec = (buf_keys, buf_grads)
        return rc

    def recovery_lock(self, check=True):
        rc = self._lib.ecrm_recovery_lock(self._ctx)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recovery_lock")
        return rc

    def recovery_decode(self, stream=None, check=True):
        rc = self._lib.ecrm_recovery_decode(self._ctx, _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recovery_decode")
        return rc

    def recovery_unlock(self, stream=None, check=True):
        rc = self._lib.ecrm_recovery_unlock(self._ctx, _stream(stream))
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recovery_unlock")
        return rc

    def recovery_state(self, stream=None):
        a, nx, ch, bf = C.c_uint32(0), C.c_uint32(0), C.c_uint32(0), C.c_uint64(0)
        rc = self._lib.ecrm_recovery_state(self._ctx, _stream(stream), C.byref(a), C.byref(nx), C.byref(ch), C.byref(bf))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_recovery_state")
        return dict(active=bool(a.value), next_chunk=int(nx.value), chunks=int(ch.value), buffered=int(bf.value))

    def embed(self, keys, out, scale=1.0, padding=None, lost_server=None, stream=None, check=True, dropout=None):
        """out: [n, D] of fp32, bf16 or fp16, rows at any multiple of 4 elements from each other."""
        n = keys.numel()
        assert _is_words(keys)
        assert out.is_cuda and out.dim() == 2 and out.shape[0] == n and out.shape[1] == self.cfg.dim and (n == 0 or out.stride(1) == 1)
        lost = 0xFFFFFFFF if lost_server is None else lost_server
        if dropout is None:
            rc = self._lib.ecrm_embed(self._ctx, keys.data_ptr(), n, _key(padding), scale, lost, out.data_ptr(), _type(out), _row(out),
                                      _stream(stream))
        else:
            assert dropout._device == out.get_device()
            address = _stream(stream)
            rc = self._lib.ecrm_embed_dropout(self._ctx, keys.data_ptr(), n, _key(padding), scale, lost, dropout._on(address, stream),
                                              out.data_ptr(), _type(out), _row(out), address)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_embed" if dropout is None else "ecrm_embed_dropout")
        return rc

    def _check_grad(self, keys, d_out):
        n = keys.numel()
        assert _is_words(keys)
        assert d_out.is_cuda and d_out.dim() == 2 and d_out.shape[0] == n and d_out.shape[1] == self.cfg.dim
        assert n == 0 or d_out.stride(1) == 1
        return n

    def embed_grad(self, keys, d_out, out_keys, out_grads, count, scale=1.0, padding=None, stream=None, check=True, dropout=None):
        """d_out: [n, D] of fp32, bf16 or fp16; out_keys [n] and out_grads [n, D] have room for as many distinct keys.  dropout: the
        lookup's."""
        import torch
        n = self._check_grad(keys, d_out)
        assert _is_words(out_keys) and out_keys.numel() >= n
        assert out_grads.is_cuda and out_grads.dtype == torch.float32 and out_grads.is_contiguous()
        assert out_grads.numel() >= n * self.cfg.dim and _is_words(count) and count.numel() == 1
        batch = (self._ctx, keys.data_ptr(), d_out.data_ptr(), _type(d_out), _row(d_out), n, _key(padding), scale)
        address = _stream(stream)
        out = (out_keys.data_ptr(), out_grads.data_ptr(), count.data_ptr(), address)
        if dropout is None:
            rc = self._lib.ecrm_embed_grad(*batch, *out)
        else:
            assert dropout._device == d_out.get_device()
            rc = self._lib.ecrm_embed_grad_dropout(*batch, dropout._on(address, stream), *out)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_embed_grad" if dropout is None else "ecrm_embed_grad_dropout")
        return rc

    def embed_grad_dense(self, keys, d_out, out, scale=1.0, padding=None, accumulate=False, stream=None, check=True, dropout=None):
        """out: [R, D] fp32.  dropout: the lookup's."""
        import torch
        n = self._check_grad(keys, d_out)
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == (self.cfg.rows, self.cfg.dim)
        batch = (self._ctx, keys.data_ptr(), d_out.data_ptr(), _type(d_out), _row(d_out), n, _key(padding), scale)
        address = _stream(stream)
        to = (out.data_ptr(), 1 if accumulate else 0, address)
        if dropout is None:
            rc = self._lib.ecrm_embed_grad_dense(*batch, *to)
        else:
            assert dropout._device == d_out.get_device()
            rc = self._lib.ecrm_embed_grad_dense_dropout(*batch, dropout._on(address, stream), *to)
        if check and rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_embed_grad_dense" if dropout is None else "ecrm_embed_grad_dense_dropout")
        return rc

    def status(self, stream=None):
        return self._lib.ecrm_status(self._ctx, _stream(stream))

    def clear_status(self, stream=None):
        rc = self._lib.ecrm_clear_status(self._ctx, _stream(stream))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_clear_status")

    def profile(self, enable=True):
        rc = self._lib.ecrm_profile(self._ctx, 1 if enable else 0)
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_profile")

    def profile_read(self):
        ms = (C.c_double * ECRM_PHASES)()
        calls = C.c_uint64(0)
        rc = self._lib.ecrm_profile_read(self._ctx, ms, C.byref(calls))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_profile_read")
        return list(ms), int(calls.value)

    def host_placement(self, key, failed_server, chunks, next_chunk, locked):
        out = (C.c_uint32 * 6)()
        rc = self._lib.ecrm_host_placement(self._ctx, C.c_uint64(key), C.c_uint32(failed_server), C.c_uint32(chunks),
                                           C.c_uint32(next_chunk), C.c_uint32(1 if locked else 0), out)
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_host_placement")
        return [int(v) for v in out]

    def batch_stats(self, stream=None):
        out = (C.c_uint64 * 5)()
        rc = self._lib.ecrm_batch_stats(self._ctx, _stream(stream), out)
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_batch_stats")
        return dict(long_rows=int(out[0]), pieces=int(out[1]), long_items=int(out[2]), rejected=int(out[3]),
                    one_workgroup_rows=int(out[4]))

    def tune(self, what, value):
        rc = self._lib.ecrm_tune(self._ctx, C.c_int(what), C.c_uint64(value))
        if rc != ECRM_OK:
            raise EcrmError(rc, "ecrm_tune")
