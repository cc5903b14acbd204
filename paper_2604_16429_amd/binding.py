"""ctypes binding of libmosaic_bsa.so: argument marshalling only.

Every function here has the name and the argument order of the C entry point
it forwards to (include/mosaic_bsa.h).  Tensors are torch tensors that own
device memory; torch supplies the current HIP stream.  Nothing is computed in
Python and there is no fallback: if the library has not been built, loading
fails with an error.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(PKG_DIR, "libmosaic_bsa.so")
_lib = None

F32, BF16 = 0, 1
OP_SELECT, OP_FWD, OP_BWD = 0, 1, 2


ROTATE_HALVES, ROTATE_PAIRS = 0, 1
SCALE_NONE, SCALE_LINEAR, SCALE_BASE, SCALE_RAMP = 0, 1, 2, 3
MAX_PAIRS = 64


class BsaError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"mosaic_bsa error {code}: {text}")
        self.code = code


class _CParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("block_h", ctypes.c_int32), ("block_w", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("n_select", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("kv_heads", ctypes.c_int32)]


@dataclasses.dataclass
class Params:
    """Mirror of the C struct mosaic_bsa_params."""
    batch: int
    heads: int
    grid_h: int
    grid_w: int
    block_h: int
    block_w: int
    head_dim: int
    n_select: int
    dtype: int = BF16
    softmax_scale: float = 0.0
    kv_heads: int = 0

    def c_struct(self) -> _CParams:
        return _CParams(self.batch, self.heads, self.grid_h, self.grid_w,
                        self.block_h, self.block_w, self.head_dim,
                        self.n_select, self.dtype, self.softmax_scale, self.kv_heads)

    @property
    def n_tokens(self) -> int:
        return self.grid_h * self.grid_w

    @property
    def block_tokens(self) -> int:
        return self.block_h * self.block_w

    @property
    def n_blocks(self) -> int:
        return self.n_tokens // self.block_tokens


class _CStrides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("head", ctypes.c_int64), ("token", ctypes.c_int64)]


class _CRotation(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("turns", ctypes.c_uint64 * MAX_PAIRS)]


class _CHeadsParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in
                 ("batch", "tokens", "heads", "kv_heads", "head_dim", "dtype", "cache_tokens",
                  "position_batch")] + [("norm_eps", ctypes.c_float)] +
                [(n, _CStrides) for n in ("q", "k", "v", "q_out", "k_out", "v_out")])


class _CWindowParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in
                 ("batch", "heads", "kv_heads", "q_tokens", "k_tokens", "head_dim", "dtype",
                  "window_left", "window_right", "n_sink", "ring")] +
                [("softmax_scale", ctypes.c_float)] +
                [(n, _CStrides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")])


class _CPagedParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in
                 ("batch", "heads", "kv_heads", "q_tokens", "head_dim", "dtype", "pages",
                  "page_tokens", "table_pages", "prefix_tokens", "window_left", "n_sink",
                  "position_batch")] +
                [("norm_eps", ctypes.c_float), ("softmax_scale", ctypes.c_float)] +
                [(n, _CStrides) for n in ("q", "k", "v", "out", "k_pages", "v_pages")])


class Rotation:
    """A mosaic_bsa_rotation, filled by mosaic_bsa_rotation_init (see there): the frequencies
    of a rotation of heads by their positions, made once and used by every call.  inv_freq:
    frequencies in radians per position that replace theta and the scaling; `c.magnitude`, 1 then, may
    be set to what belongs to them."""

    def __init__(self, rotary_dim: int, axes: int = 1, layout: int = ROTATE_HALVES,
                 theta: float = 10000.0, scaling: int = SCALE_NONE, factor: float = 1.0,
                 original_tokens: float = 0.0, beta_fast: float = 0.0, beta_slow: float = 0.0,
                 inv_freq=None):
        freq = None
        if inv_freq is not None:
            values = [float(x) for x in inv_freq]
            if axes in (1, 2) and len(values) != rotary_dim // axes // 2:
                raise ValueError(f"inv_freq needs {rotary_dim // axes // 2} values")
            freq = (ctypes.c_double * max(1, len(values)))(*values)
        self.c = _CRotation()
        self.axes = axes
        _check(load_library().mosaic_bsa_rotation_init(
            rotary_dim, axes, layout, theta, scaling, factor, original_tokens, beta_fast,
            beta_slow, freq, ctypes.byref(self.c)))
        self.ref = ctypes.byref(self.c)

    def __getstate__(self):
        return self.axes, bytes(self.c)

    def __setstate__(self, state):
        self.axes = state[0]
        self.c = _CRotation.from_buffer_copy(state[1])
        self.ref = ctypes.byref(self.c)


class _StridedParams:
    """Parameters whose C struct also carries the tensors' strides.  A call has a struct of its own for
    the types, shapes and strides of its tensors, which is kept for the entry point's next call if that
    has the same and not written to again: threads can call with one object at the same time (setting
    a field of it meanwhile is another matter).  A copy keeps structs of its own."""

    _C = None
    _SCALARS = ()

    def __setattr__(self, name, value):
        self.__dict__[name] = value
        self.__dict__.update(_struct=None, _ref=None, _kept={})

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k not in ("_struct", "_ref", "_kept")}

    def __setstate__(self, state):
        self.__dict__.update(state, _struct=None, _ref=None, _kept={})

    def _new_struct(self):
        c = self._C()
        for name in self._SCALARS:
            setattr(c, name, getattr(self, name))
        return c

    def _c(self):
        """The struct without strides (contiguous tensors)."""
        c = self._struct
        if c is None:
            c = self._new_struct()
            self.__dict__.update(_struct=c, _ref=ctypes.byref(c))
        return c

    def _call(self, entry, *args, position_batch=None, device=None):
        """(struct, its reference, device pointers) of a call of `entry` on [batch, heads, tokens, head_dim]
        tensors, given as (field of the struct, tensor, heads, tokens) one after the other.  Integers and
        None are taken as they are (contiguous).  device: the GPU that all of them have to be on."""
        looks, pointers = [position_batch], []
        for _, t, heads, tokens in args:
            if t is None or isinstance(t, int):
                looks.append(None)
                pointers.append(t)
            else:
                looks.append((t.shape, t.stride(), t.dtype,
                              t.is_cuda if device is None else t.get_device() == device, heads, tokens))
                pointers.append(t.data_ptr())
        kept = self._kept
        last = kept.get(entry)
        if last is None or last[0] != looks:
            c = self._new_struct()
            if position_batch is not None:
                c.position_batch = position_batch
            for field, t, heads, tokens in args:
                if t is not None and not isinstance(t, int):
                    if device is not None and t.get_device() != device:
                        raise ValueError(f"{field}: on {t.device} instead of the first tensor's GPU")
                    setattr(c, field, self._strides(field, t, heads, tokens))
            last = kept[entry] = looks, c, ctypes.byref(c)
        return last[1], last[2], pointers

    def _entries(self, field):
        """First dimension of a field's tensor."""
        return self.batch

    def _strides(self, field, t, heads, tokens):
        entries = self._entries(field)
        wanted, strides = (entries, heads, tokens, self.head_dim), t.stride()
        if t.shape != wanted:
            raise ValueError(f"{field}: shape {tuple(t.shape)} instead of {wanted}")
        if t.dtype is not _named_dtype(self.dtype) or not t.is_cuda:
            raise ValueError(f"{field}: {t.dtype} on {t.device} instead of the parameters' dtype "
                             "on a GPU")
        if strides[3] != 1:
            raise ValueError(f"{field}: channels must be consecutive")
        if strides[2] == 0 and tokens > 1:
            raise ValueError(f"{field}: tokens share memory")
        # a dimension of one entry may carry any stride: the contiguous one is taken
        token = strides[2] if tokens > 1 else self.head_dim
        head = strides[1] if heads > 1 else token * tokens
        batch = strides[0] if entries > 1 else head * heads
        return _CStrides(batch, head, token)


_TORCH_DTYPES = {}


def _named_dtype(name):
    if not _TORCH_DTYPES:
        import torch
        _TORCH_DTYPES.update({F32: torch.float32, BF16: torch.bfloat16,
                              "float32": torch.float32, "int32": torch.int32})
    return _TORCH_DTYPES.get(name)


def _vector(name, t, size, dtype_name):
    """Pointer of a contiguous device tensor of `size` values of torch dtype `dtype_name`."""
    if t is None or isinstance(t, int):
        return t
    if (t.numel() != size or t.dtype is not _named_dtype(dtype_name) or not t.is_cuda or
            not t.is_contiguous()):
        raise ValueError(f"{name}: {size} contiguous {dtype_name} values on a GPU expected")
    return t.data_ptr()


class _Positions:
    """Positions of [batch, n] tokens."""

    def _positions_of(self, rotation, t, n):
        """Pointer and values from one batch entry's positions to the next's."""
        per = 0
        if t is not None and not isinstance(t, int):
            axes = rotation.axes
            if t.dtype is not _named_dtype("int32") or not t.is_cuda or not t.is_contiguous():
                raise ValueError("positions: contiguous int32 on a GPU expected")
            if t.shape == (self.batch, n, axes) or (axes == 1 and t.shape == (self.batch, n)):
                per = n * axes
            elif t.shape != (n, axes) and not (axes == 1 and t.shape == (n,)):
                raise ValueError(f"positions: shape {tuple(t.shape)}")
            t = t.data_ptr()
        return t, per


@dataclasses.dataclass
class HeadsParams(_Positions, _StridedParams):
    """Mirror of the C struct mosaic_bsa_heads_params (the strides come from the tensors)."""
    batch: int
    tokens: int
    heads: int
    head_dim: int
    dtype: int = BF16
    kv_heads: int = 0
    cache_tokens: int = 0
    norm_eps: float = 1e-6

    _C = _CHeadsParams
    _SCALARS = ("batch", "tokens", "heads", "head_dim", "dtype", "kv_heads", "cache_tokens",
                "norm_eps")

    def _positions(self, rotation, t):
        return self._positions_of(rotation, t, self.tokens)


@dataclasses.dataclass
class WindowParams(_StridedParams):
    """Mirror of the C struct mosaic_bsa_window_params (the strides come from the tensors)."""
    batch: int
    heads: int
    q_tokens: int
    k_tokens: int
    head_dim: int
    dtype: int = BF16
    kv_heads: int = 0
    window_left: int = -1
    window_right: int = 0
    n_sink: int = 0
    ring: int = 0
    softmax_scale: float = 0.0

    _C = _CWindowParams
    _SCALARS = ("batch", "heads", "q_tokens", "k_tokens", "head_dim", "dtype", "kv_heads",
                "window_left", "window_right", "n_sink", "ring", "softmax_scale")


@dataclasses.dataclass
class PagedParams(_Positions, _StridedParams):
    """Mirror of the C struct mosaic_bsa_paged_params (the strides come from the tensors)."""
    batch: int
    heads: int
    q_tokens: int
    head_dim: int
    pages: int
    page_tokens: int
    table_pages: int
    dtype: int = BF16
    kv_heads: int = 0
    prefix_tokens: int = 0
    window_left: int = -1
    n_sink: int = 0
    norm_eps: float = 1e-6
    softmax_scale: float = 0.0

    _C = _CPagedParams
    _SCALARS = ("batch", "heads", "q_tokens", "head_dim", "pages", "page_tokens", "table_pages",
                "dtype", "kv_heads", "prefix_tokens", "window_left", "n_sink", "norm_eps",
                "softmax_scale")

    def _entries(self, field):
        return self.pages if field in ("k_pages", "v_pages") else self.batch


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load the built library; raises if it is missing (no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(
                f"{_LIB_PATH} is not built; run `python -m paper_2604_16429_amd.build`")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        pp = ctypes.POINTER(_CParams)
        lib.mosaic_bsa_workspace_bytes.restype = sz
        lib.mosaic_bsa_workspace_bytes.argtypes = [pp, i32]
        lib.mosaic_bsa_select.restype = i32
        lib.mosaic_bsa_select.argtypes = [pp, vp, vp, vp, vp, sz, vp]
        lib.mosaic_bsa_select_static.restype = i32
        lib.mosaic_bsa_select_static.argtypes = [pp, vp, vp, vp, vp]
        lib.mosaic_bsa_fwd.restype = i32
        lib.mosaic_bsa_fwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.mosaic_bsa_bwd.restype = i32
        lib.mosaic_bsa_bwd.argtypes = [pp] + [vp] * 10 + [vp, sz, vp]
        lib.mosaic_bsa_three_branch_workspace_bytes.restype = sz
        lib.mosaic_bsa_three_branch_workspace_bytes.argtypes = [pp, ctypes.c_int32, ctypes.c_int32]
        lib.mosaic_bsa_fwd_three_branch.restype = i32
        lib.mosaic_bsa_fwd_three_branch.argtypes = (
            [pp, ctypes.c_int32, ctypes.c_int32] + [vp] * 7 + [sz, vp])
        lib.mosaic_bsa_three_branch_bwd_workspace_bytes.restype = sz
        lib.mosaic_bsa_three_branch_bwd_workspace_bytes.argtypes = [
            pp, ctypes.c_int32, ctypes.c_int32]
        lib.mosaic_bsa_bwd_three_branch.restype = i32
        lib.mosaic_bsa_bwd_three_branch.argtypes = (
            [pp, ctypes.c_int32, ctypes.c_int32] + [vp] * 12 + [sz, vp])
        lib.mosaic_bsa_check_selection.restype = i32
        lib.mosaic_bsa_check_selection.argtypes = [pp, vp, ctypes.c_int32, vp, vp]
        lib.mosaic_bsa_probe_mfma.restype = i32
        lib.mosaic_bsa_probe_mfma.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, vp]
        dbl, st = ctypes.c_double, ctypes.POINTER(_CStrides)
        hp, rp = ctypes.POINTER(_CHeadsParams), ctypes.POINTER(_CRotation)
        wp = ctypes.POINTER(_CWindowParams)
        lib.mosaic_bsa_rotation_init.restype = i32
        lib.mosaic_bsa_rotation_init.argtypes = (
            [ctypes.c_int32] * 3 + [dbl, ctypes.c_int32] + [dbl] * 4 + [ctypes.POINTER(dbl), rp])
        lib.mosaic_bsa_rope_fwd.restype = i32
        lib.mosaic_bsa_rope_fwd.argtypes = [hp, rp] + [vp] * 9
        lib.mosaic_bsa_rope_bwd.restype = i32
        lib.mosaic_bsa_rope_bwd.argtypes = [hp, rp] + [vp] * 6
        lib.mosaic_bsa_qk_norm_rope_fwd.restype = i32
        lib.mosaic_bsa_qk_norm_rope_fwd.argtypes = [hp, rp] + [vp] * 11
        lib.mosaic_bsa_qk_norm_rope_workspace_bytes.restype = sz
        lib.mosaic_bsa_qk_norm_rope_workspace_bytes.argtypes = [hp]
        lib.mosaic_bsa_qk_norm_rope_bwd.restype = i32
        lib.mosaic_bsa_qk_norm_rope_bwd.argtypes = [hp, rp] + [vp] * 7 + [st, st] + [vp] * 5 + [sz, vp]
        lib.mosaic_bsa_window_workspace_bytes.restype = sz
        lib.mosaic_bsa_window_workspace_bytes.argtypes = [wp, i32]
        lib.mosaic_bsa_window_fwd.restype = i32
        lib.mosaic_bsa_window_fwd.argtypes = [wp] + [vp] * 8 + [sz, vp]
        lib.mosaic_bsa_window_bwd.restype = i32
        lib.mosaic_bsa_window_bwd.argtypes = [wp] + [vp] * 12 + [sz, vp]
        gp = ctypes.POINTER(_CPagedParams)
        lib.mosaic_bsa_paged_append.restype = i32
        lib.mosaic_bsa_paged_append.argtypes = [gp, rp] + [vp] * 14
        lib.mosaic_bsa_paged_workspace_bytes.restype = sz
        lib.mosaic_bsa_paged_workspace_bytes.argtypes = [gp]
        lib.mosaic_bsa_paged_fwd.restype = i32
        lib.mosaic_bsa_paged_fwd.argtypes = [gp] + [vp] * 11 + [sz, vp]
        lib.mosaic_bsa_strerror.restype = ctypes.c_char_p
        lib.mosaic_bsa_strerror.argtypes = [i32]
        _lib = lib
    return _lib


def _ptr(t):
    """Device (or raw integer) pointer of a tensor-like argument."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _raw():
    """Functions for a device's current stream and for the current device."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_device()                   # (initialises the device on first use)
        _raw_stream = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    return _raw_stream


def _stream(stream):
    if stream is None:
        # the handle of torch.cuda.current_stream() without its Stream object, which
        # took 3.1 us of a call (a forward with its one launch 8.5 us, without 5.6)
        of_device, device = _raw_stream or _raw()
        return of_device(device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_raw_stream = None


def _nbytes(t) -> int:
    return 0 if t is None or isinstance(t, int) else t.numel() * t.element_size()


def _check(code: int) -> None:
    if code != 0:
        raise BsaError(code, mosaic_bsa_strerror(code))


def mosaic_bsa_strerror(code: int) -> str:
    return load_library().mosaic_bsa_strerror(int(code)).decode()


def mosaic_bsa_workspace_bytes(params: Params, op: int) -> int:
    cp = params.c_struct()
    return int(load_library().mosaic_bsa_workspace_bytes(ctypes.byref(cp), int(op)))


def mosaic_bsa_select(params: Params, q, k, sel_idx, workspace, stream=None,
                      workspace_bytes=None) -> None:
    cp = params.c_struct()
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load_library().mosaic_bsa_select(
        ctypes.byref(cp), _ptr(q), _ptr(k), _ptr(sel_idx), _ptr(workspace), wb,
        _stream(stream)))


def mosaic_bsa_select_static(params: Params, q, k, sel_idx, stream=None) -> None:
    cp = params.c_struct()
    _check(load_library().mosaic_bsa_select_static(
        ctypes.byref(cp), _ptr(q), _ptr(k), _ptr(sel_idx), _stream(stream)))


def mosaic_bsa_fwd(params: Params, q, k, v, sel_idx, out, lse=None,
                   workspace=None, stream=None, workspace_bytes=None) -> None:
    cp = params.c_struct()
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load_library().mosaic_bsa_fwd(
        ctypes.byref(cp), _ptr(q), _ptr(k), _ptr(v), _ptr(sel_idx), _ptr(out),
        _ptr(lse), _ptr(workspace), wb, _stream(stream)))


def mosaic_bsa_bwd(params: Params, q, k, v, out, lse, dout, sel_idx, dq, dk, dv,
                   workspace=None, stream=None, workspace_bytes=None) -> None:
    cp = params.c_struct()
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load_library().mosaic_bsa_bwd(
        ctypes.byref(cp), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
        _ptr(dout), _ptr(sel_idx), _ptr(dq), _ptr(dk), _ptr(dv),
        _ptr(workspace), wb, _stream(stream)))


def mosaic_bsa_three_branch_workspace_bytes(params: Params, local_h: int, local_w: int) -> int:
    cp = params.c_struct()
    return int(load_library().mosaic_bsa_three_branch_workspace_bytes(
        ctypes.byref(cp), int(local_h), int(local_w)))


def mosaic_bsa_fwd_three_branch(params: Params, local_h: int, local_w: int, q, k, v, gates,
                                out, sel_idx, workspace, stream=None,
                                workspace_bytes=None) -> None:
    cp = params.c_struct()
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load_library().mosaic_bsa_fwd_three_branch(
        ctypes.byref(cp), int(local_h), int(local_w), _ptr(q), _ptr(k), _ptr(v), _ptr(gates),
        _ptr(out), _ptr(sel_idx), _ptr(workspace), wb, _stream(stream)))


def mosaic_bsa_probe_mfma(sink, workgroups: int, iters: int, stream=None) -> None:
    _check(load_library().mosaic_bsa_probe_mfma(_ptr(sink), int(workgroups), int(iters),
                                                _stream(stream)))


def mosaic_bsa_three_branch_bwd_workspace_bytes(params: Params, local_h: int,
                                                local_w: int) -> int:
    cp = params.c_struct()
    return int(load_library().mosaic_bsa_three_branch_bwd_workspace_bytes(
        ctypes.byref(cp), int(local_h), int(local_w)))


def mosaic_bsa_bwd_three_branch(params: Params, local_h: int, local_w: int, q, k, v, gates,
                                dout, sel_idx, fwd_workspace, dq, dk, dv, dgates, workspace,
                                stream=None, workspace_bytes=None) -> None:
    cp = params.c_struct()
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load_library().mosaic_bsa_bwd_three_branch(
        ctypes.byref(cp), int(local_h), int(local_w), _ptr(q), _ptr(k), _ptr(v), _ptr(gates),
        _ptr(dout), _ptr(sel_idx), _ptr(fwd_workspace), _ptr(dq), _ptr(dk), _ptr(dv),
        _ptr(dgates), _ptr(workspace), wb, _stream(stream)))


def mosaic_bsa_check_selection(params: Params, sel_idx, own_block_allowed: bool, n_bad,
                               stream=None) -> None:
    cp = params.c_struct()
    _check(load_library().mosaic_bsa_check_selection(
        ctypes.byref(cp), _ptr(sel_idx), 1 if own_block_allowed else 0, _ptr(n_bad),
        _stream(stream)))


# ---- rotation, head norms and windowed attention: tensors of shape [batch, heads, tokens,
# head_dim] with any strides of the first three dimensions

def mosaic_bsa_rotation_init(rotary_dim: int, axes: int = 1, layout: int = ROTATE_HALVES,
                             **kw) -> Rotation:
    """The C entry point's name for Rotation(...)."""
    return Rotation(rotary_dim, axes, layout, **kw)


def _heads_forward(params, rotation, positions, q, k, q_out, k_out, v, v_out, rows):
    h, kv, n = params.heads, params.kv_heads or params.heads, params.tokens
    m = n if rows is None else params.cache_tokens
    pos, per = params._positions(rotation, positions)
    rows = None if rows is None else _vector("rows", rows, params.batch * n, "int32")
    if v is None and v_out is None:
        _, ref, (q, k, q_out, k_out) = params._call(
            "fwd", ("q", q, h, n), ("k", k, kv, n), ("q_out", q_out, h, n), ("k_out", k_out, kv, m),
            position_batch=per)
    else:
        _, ref, (q, k, q_out, k_out, v, v_out) = params._call(
            "cached", ("q", q, h, n), ("k", k, kv, n), ("q_out", q_out, h, n), ("k_out", k_out, kv, m),
            ("v", v, kv, n), ("v_out", v_out, kv, m), position_batch=per)
    return ref, pos, q, k, v, rows, q_out, k_out, v_out


def mosaic_bsa_rope_fwd(params: HeadsParams, rotation: Rotation, positions, q, k, q_out, k_out,
                        v=None, v_out=None, rows=None, stream=None) -> None:
    ref, pos, q, k, v, rows, q_out, k_out, v_out = _heads_forward(
        params, rotation, positions, q, k, q_out, k_out, v, v_out, rows)
    _check(load_library().mosaic_bsa_rope_fwd(ref, rotation.ref, pos, q, k, v, rows, q_out, k_out, v_out,
                                              _stream(stream)))


def mosaic_bsa_rope_bwd(params: HeadsParams, rotation: Rotation, positions, dq_out, dk_out, dq, dk,
                        stream=None) -> None:
    h, kv, n = params.heads, params.kv_heads or params.heads, params.tokens
    pos, per = params._positions(rotation, positions)
    _, ref, (dq_out, dk_out, dq, dk) = params._call(
        "rope_bwd", ("q_out", dq_out, h, n), ("k_out", dk_out, kv, n), ("q", dq, h, n), ("k", dk, kv, n),
        position_batch=per)
    _check(load_library().mosaic_bsa_rope_bwd(ref, rotation.ref, pos, dq_out, dk_out, dq, dk,
                                              _stream(stream)))


def mosaic_bsa_qk_norm_rope_fwd(params: HeadsParams, rotation: Rotation, positions, q, k, q_weight,
                                k_weight, q_out, k_out, v=None, v_out=None, rows=None,
                                stream=None) -> None:
    ref, pos, q, k, v, rows, q_out, k_out, v_out = _heads_forward(
        params, rotation, positions, q, k, q_out, k_out, v, v_out, rows)
    d = params.head_dim
    _check(load_library().mosaic_bsa_qk_norm_rope_fwd(
        ref, rotation.ref, pos, q, k, v, _vector("q_weight", q_weight, d, "float32"),
        _vector("k_weight", k_weight, d, "float32"), rows, q_out, k_out, v_out, _stream(stream)))


def mosaic_bsa_qk_norm_rope_workspace_bytes(params: HeadsParams) -> int:
    return int(load_library().mosaic_bsa_qk_norm_rope_workspace_bytes(ctypes.byref(params._c())))


def mosaic_bsa_qk_norm_rope_bwd(params: HeadsParams, rotation: Rotation, positions, q, k, q_weight,
                                k_weight, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace,
                                stream=None, workspace_bytes=None) -> None:
    h, kv, n, d = params.heads, params.kv_heads or params.heads, params.tokens, params.head_dim
    pos, per = params._positions(rotation, positions)
    # the strides of dq and dk are arguments of their own: the fields of v and v_out hold them
    c, ref, (q, k, dq_out, dk_out, dq, dk) = params._call(
        "norm_bwd", ("q", q, h, n), ("k", k, kv, n), ("q_out", dq_out, h, n), ("k_out", dk_out, kv, n),
        ("v", dq, h, n), ("v_out", dk, kv, n), position_batch=per)
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(load_library().mosaic_bsa_qk_norm_rope_bwd(
        ref, rotation.ref, pos, q, k, _vector("q_weight", q_weight, d, "float32"),
        _vector("k_weight", k_weight, d, "float32"), dq_out, dk_out, ctypes.byref(c.v),
        ctypes.byref(c.v_out), dq, dk, _vector("dq_weight", dq_weight, d, "float32"),
        _vector("dk_weight", dk_weight, d, "float32"), _ptr(workspace), wb, _stream(stream)))


def mosaic_bsa_window_workspace_bytes(params: WindowParams, op: int) -> int:
    return int(load_library().mosaic_bsa_window_workspace_bytes(ctypes.byref(params._c()), int(op)))


def mosaic_bsa_window_fwd(params: WindowParams, q, k, v, out, lse=None, q_lens=None, k_lens=None,
                          workspace=None, stream=None, workspace_bytes=None) -> None:
    h, kv, nq, nk = params.heads, params.kv_heads or params.heads, params.q_tokens, params.k_tokens
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _, ref, (q, k, v, out) = params._call("fwd", ("q", q, h, nq), ("k", k, kv, nk), ("v", v, kv, nk),
                                          ("out", out, h, nq))
    _check(load_library().mosaic_bsa_window_fwd(
        ref, q, k, v, _vector("q_lens", q_lens, params.batch, "int32"),
        _vector("k_lens", k_lens, params.batch, "int32"), out,
        _vector("lse", lse, params.batch * h * nq, "float32"), _ptr(workspace), wb,
        _stream(stream)))


def mosaic_bsa_window_bwd(params: WindowParams, q, k, v, out, lse, dout, dq, dk, dv,
                          workspace=None, q_lens=None, k_lens=None, stream=None,
                          workspace_bytes=None) -> None:
    h, kv, nq, nk = params.heads, params.kv_heads or params.heads, params.q_tokens, params.k_tokens
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _, ref, (q, k, v, out, dout, dq, dk, dv) = params._call(
        "bwd", ("q", q, h, nq), ("k", k, kv, nk), ("v", v, kv, nk), ("out", out, h, nq),
        ("dout", dout, h, nq), ("dq", dq, h, nq), ("dk", dk, kv, nk), ("dv", dv, kv, nk))
    _check(load_library().mosaic_bsa_window_bwd(
        ref, q, k, v, out, _vector("lse", lse, params.batch * h * nq, "float32"), dout,
        _vector("q_lens", q_lens, params.batch, "int32"),
        _vector("k_lens", k_lens, params.batch, "int32"), dq, dk, dv, _ptr(workspace), wb,
        _stream(stream)))


# ---- a cache in pages: k_pages and v_pages of shape [pages, kv_heads, page_tokens, head_dim] with any
# strides of the first three dimensions

def _device_of(name, t):
    """The GPU of a tensor; None for an address."""
    if t is None or isinstance(t, int):
        return None
    device = t.get_device()
    if device < 0:
        raise ValueError(f"{name}: on {t.device} instead of a GPU")
    return device


def _vector_on(device, name, t, size, dtype):
    """_vector on one GPU, of a torch dtype."""
    if t is None or isinstance(t, int):
        return t
    if (t.numel() != size or t.dtype is not dtype or not t.is_contiguous() or
            (t.get_device() != device if device is not None else not t.is_cuda)):
        raise ValueError(f"{name}: {size} contiguous {dtype} values on the tensors' GPU expected")
    return t.data_ptr()


def _table_on(device, t, params):
    """_vector_on for a page table, [batch, table_pages] or flat."""
    wanted = (params.batch, params.table_pages)
    if t is not None and not isinstance(t, int) and t.shape != wanted and len(t.shape) != 1:
        raise ValueError(f"page_table: shape {tuple(t.shape)} instead of {wanted}")
    return _vector_on(device, "page_table", t, wanted[0] * wanted[1], _named_dtype("int32"))


def _stream_on(device, stream):
    """_stream, which has to belong to the tensors' GPU (a handle of 0 to the current one; of other handles
    that is not known)."""
    handle = _stream(stream)
    if device is not None:
        if not isinstance(stream, int):
            there = _raw_stream[1]() if stream is None else stream.device_index
        else:
            there = device if stream else (_raw_stream or _raw())[1]()
        if there != device:
            raise ValueError(f"tensors on cuda:{device}, stream on cuda:{there}")
    return handle


def mosaic_bsa_paged_append(params: PagedParams, rotation: Rotation, positions, q, k, v, q_weight,
                            k_weight, q_lens, k_lens, page_table, prefix_len, q_out, k_pages, v_pages,
                            stream=None) -> None:
    h, kv, n, d = params.heads, params.kv_heads or params.heads, params.q_tokens, params.head_dim
    b, t, on = params.batch, params.page_tokens, _device_of("q", q)
    i32, f32 = _named_dtype("int32"), _named_dtype("float32")
    pos, per = params._positions_of(rotation, positions, n)
    if pos is not positions and on is not None and positions.get_device() != on:
        raise ValueError("positions: on another GPU")
    _, ref, (q, k, v, q_out, k_pages, v_pages) = params._call(
        "append", ("q", q, h, n), ("k", k, kv, n), ("v", v, kv, n), ("out", q_out, h, n),
        ("k_pages", k_pages, kv, t), ("v_pages", v_pages, kv, t), position_batch=per, device=on)
    _check(load_library().mosaic_bsa_paged_append(
        ref, rotation.ref, pos, q, k, v, _vector_on(on, "q_weight", q_weight, d, f32),
        _vector_on(on, "k_weight", k_weight, d, f32), _vector_on(on, "q_lens", q_lens, b, i32),
        _vector_on(on, "k_lens", k_lens, b, i32),
        _table_on(on, page_table, params),
        _vector_on(on, "prefix_len", prefix_len, 1, i32), q_out, k_pages, v_pages,
        _stream_on(on, stream)))


def mosaic_bsa_paged_workspace_bytes(params: PagedParams) -> int:
    return int(load_library().mosaic_bsa_paged_workspace_bytes(ctypes.byref(params._c())))


def mosaic_bsa_paged_fwd(params: PagedParams, q, k_pages, v_pages, q_lens, k_lens, page_table,
                         prefix_table, prefix_len, out, lse=None, workspace=None, stream=None,
                         workspace_bytes=None) -> None:
    h, kv, n, b = params.heads, params.kv_heads or params.heads, params.q_tokens, params.batch
    t, on = params.page_tokens, _device_of("q", q)
    i32, f32 = _named_dtype("int32"), _named_dtype("float32")
    wb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    if _device_of("workspace", workspace) not in (None, on) and on is not None:
        raise ValueError("workspace: on another device than the tensors")
    _, ref, (q, k_pages, v_pages, out) = params._call(
        "fwd", ("q", q, h, n), ("k_pages", k_pages, kv, t), ("v_pages", v_pages, kv, t),
        ("out", out, h, n), device=on)
    if params.prefix_tokens <= 0:
        prefix_table = None
    _check(load_library().mosaic_bsa_paged_fwd(
        ref, q, k_pages, v_pages, _vector_on(on, "q_lens", q_lens, b, i32),
        _vector_on(on, "k_lens", k_lens, b, i32),
        _table_on(on, page_table, params),
        _vector_on(on, "prefix_table", prefix_table, -(-params.prefix_tokens // max(t, 1)), i32),
        _vector_on(on, "prefix_len", prefix_len, 1, i32), out,
        _vector_on(on, "lse", lse, b * h * n, f32), _ptr(workspace), wb, _stream_on(on, stream)))
