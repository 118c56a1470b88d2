"""Python binding of libattr, the MI355X gradient-attribution hot path.

Thin ctypes marshalling over the C ABI declared in ``include/attr.h``: the
functions below carry the same names as the C entry points, take torch
tensors that already live on the GPU, and pass their device pointers, sizes
and the current HIP stream through unchanged.  Every arithmetic step runs in
the library's HIP kernels; PyTorch only provides device memory and streams.
The library must have been built (``python -m paper_2606_11660_amd.build``);
importing this package without it raises, there is no fallback path.

Every wrapper checks the tensors it is given against the sizes it passes
(shapes, dtypes, devices) and raises ``ValueError`` before calling the
library, which sees only pointers.  The one host step of the method, turning
the accumulated second moment into H^{-1/2}, lives in ``finalize``.
"""
from __future__ import annotations

import ctypes
import os
import threading
import warnings
from typing import Dict, Iterable, List, Optional, Sequence, Tuple

import torch

__all__ = [
    "AttrError", "ATTR_F32", "ATTR_BF16", "ATTR_F16", "PRECOND_NONE", "PRECOND_DIAG",
    "PRECOND_FULL", "Module", "lib", "lib_path", "attr_project", "attr_project_noalloc",
    "attr_project_tokens",
    "attr_precond_accumulate",
    "attr_precond_apply", "attr_score_topk", "attr_project_workspace_size",
    "attr_precond_accumulate_workspace_size", "attr_precond_apply_workspace_size",
    "attr_score_topk_workspace_size", "Workspace", "attr_probe_read", "attr_probe_mfma",
    "ATTR_E4M3", "TokenRows", "attr_token_logp", "attr_policy_loss", "attr_preference_loss",
    "attr_token_logp_workspace_size", "attr_policy_loss_workspace_size",
    "attr_preference_loss_workspace_size", "AdamTensors", "attr_adamw_step",
    "MuonTensors", "attr_muon_step", "attr_muon_step_workspace_size", "ExampleRows", "attr_embed", "attr_embed_backward",
    "attr_embed_backward_workspace_size", "attr_layer_norm", "attr_layer_norm_backward",
    "attr_layer_norm_backward_workspace_size",
]

_PKG = os.path.dirname(os.path.abspath(__file__))
# ATTR_LIBRARY selects another build of the same library (the host-sanitizer
# build of the CPU tests); by default the in-tree libattr.so.
_LIB_PATH = os.environ.get("ATTR_LIBRARY") or os.path.join(_PKG, "libattr.so")

ATTR_F32, ATTR_BF16, ATTR_F16, ATTR_E4M3 = 0, 1, 2, 3
PRECOND_NONE, PRECOND_DIAG, PRECOND_FULL = 0, 1, 2
_STATUS = {0: "ATTR_OK", 1: "ATTR_ERR_INVALID_ARG", 2: "ATTR_ERR_UNSUPPORTED",
           3: "ATTR_ERR_ALIGNMENT", 4: "ATTR_ERR_WORKSPACE", 5: "ATTR_ERR_DEVICE"}
_TORCH_DTYPE = {torch.float32: ATTR_F32, torch.bfloat16: ATTR_BF16, torch.float16: ATTR_F16}


class AttrError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status
        self.message = message


class _CModule(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("g", ctypes.c_void_p), ("R", ctypes.c_void_p),
                ("S", ctypes.c_void_p), ("lda", ctypes.c_int64), ("ldg", ctypes.c_int64),
                ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64), ("out_col", ctypes.c_int64),
                ("v_out", ctypes.c_void_p), ("v_in", ctypes.c_void_p)]


class _CTokenRows(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("dtype", ctypes.c_int), ("n_rows", ctypes.c_int64),
                ("V", ctypes.c_int64), ("ldl", ctypes.c_int64), ("logit_scale", ctypes.c_float),
                ("target", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("n_examples", ctypes.c_int64),
                ("T", ctypes.c_int64), ("row_offset", ctypes.c_void_p), ("length", ctypes.c_void_p)]


class _CAdamTensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("master", ctypes.c_void_p), ("m_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n", ctypes.c_int64), ("lr_scale", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]


class _CMuonMatrix(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p), ("master", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("lr_scale", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]


class _CRows(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int64), ("n_examples", ctypes.c_int64), ("T", ctypes.c_int64),
                ("row_offset", ctypes.c_void_p), ("length", ctypes.c_void_p)]


_lib = None


def lib_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """Load libattr.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2606_11660_amd.build`")
    L = ctypes.CDLL(_LIB_PATH)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    L.attr_last_error.restype = ctypes.c_char_p
    L.attr_status_string.restype = ctypes.c_char_p
    L.attr_status_string.argtypes = [ctypes.c_int]
    L.attr_abi_version.restype = ctypes.c_int
    L.attr_project_workspace_size.restype = sz
    L.attr_project_workspace_size.argtypes = [ctypes.POINTER(_CModule), i32, ctypes.c_int, i64, i64, i32]
    L.attr_project.restype = ctypes.c_int
    L.attr_project.argtypes = [ctypes.POINTER(_CModule), i32, ctypes.c_int, i32, i64, i64, vp, vp,
                               vp, i64, vp, sz, vp]
    L.attr_project_tokens.restype = ctypes.c_int
    L.attr_project_tokens.argtypes = [ctypes.POINTER(_CModule), i32, ctypes.c_int, i32, i64, i64, vp,
                                      vp, vp, i64, i64, vp, sz, vp]
    L.attr_project_noalloc.restype = ctypes.c_int
    L.attr_project_noalloc.argtypes = [ctypes.POINTER(_CModule), i32, ctypes.c_int, i32, i64, i64,
                                       vp, vp, vp, i64, vp]
    L.attr_precond_accumulate_workspace_size.restype = sz
    L.attr_precond_accumulate_workspace_size.argtypes = [i64, i64, ctypes.c_int, ctypes.c_int]
    L.attr_precond_accumulate.restype = ctypes.c_int
    L.attr_precond_accumulate.argtypes = [vp, ctypes.c_int, i64, i64, i64, ctypes.c_int, vp, vp, sz, vp]
    L.attr_precond_apply_workspace_size.restype = sz
    L.attr_precond_apply_workspace_size.argtypes = [i64, i64, ctypes.c_int]
    L.attr_precond_apply.restype = ctypes.c_int
    L.attr_precond_apply.argtypes = [vp, ctypes.c_int, i64, i64, i64, ctypes.c_int, vp, i32, vp,
                                     ctypes.c_int, i64, vp, sz, vp]
    L.attr_probe_read.restype = ctypes.c_int
    L.attr_probe_read.argtypes = [vp, sz, vp, vp]
    L.attr_probe_mfma.restype = ctypes.c_int
    L.attr_probe_mfma.argtypes = [i64, vp, vp]
    L.attr_score_topk_workspace_size.restype = sz
    L.attr_score_topk_workspace_size.argtypes = [i64, i64, i64, i32]
    L.attr_score_topk.restype = ctypes.c_int
    L.attr_score_topk.argtypes = [vp, i64, i64, vp, i64, i64, ctypes.c_int, i64, i32, i64, i32, vp,
                                  vp, vp, sz, vp]
    f32, f64, rows = ctypes.c_float, ctypes.c_double, ctypes.POINTER(_CTokenRows)
    for name in ("attr_token_logp", "attr_policy_loss", "attr_preference_loss"):
        query = getattr(L, name + "_workspace_size")
        query.restype, query.argtypes = sz, [rows]
    L.attr_token_logp.restype = ctypes.c_int
    L.attr_token_logp.argtypes = [rows, vp, vp, sz, vp]
    L.attr_policy_loss.restype = ctypes.c_int
    L.attr_policy_loss.argtypes = [rows, vp, i32, vp, vp, f32, f32, f32, vp, vp, vp, i64, vp, sz, vp]
    L.attr_preference_loss.restype = ctypes.c_int
    L.attr_preference_loss.argtypes = [rows, vp, vp, f32, f32, f32, vp, vp, vp, vp, i64, vp, sz, vp]
    L.attr_adamw_step.restype = ctypes.c_int
    L.attr_adamw_step.argtypes = [ctypes.POINTER(_CAdamTensor), i32, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                  i64, f64, f64, f64, f64, f64, vp, vp]
    mats, code, batch = ctypes.POINTER(_CMuonMatrix), ctypes.c_int, ctypes.POINTER(_CRows)
    L.attr_muon_step_workspace_size.restype = sz
    L.attr_muon_step_workspace_size.argtypes = [mats, i32, i32]
    L.attr_muon_step.restype = code
    L.attr_muon_step.argtypes = [mats, i32, code, code, f64, f64, i32, i32, i32, vp, vp, sz, vp]
    L.attr_embed.restype = code
    L.attr_embed.argtypes = [batch, vp, vp, code, i64, i64, i64, f32, vp, code, i64, vp]
    L.attr_embed_backward_workspace_size.restype = sz
    L.attr_embed_backward_workspace_size.argtypes = [batch, i64, i64]
    L.attr_embed_backward.restype = code
    L.attr_embed_backward.argtypes = [batch, vp, vp, code, i64, i64, i64, f32, vp, code, i64, i32, vp, sz, vp]
    L.attr_layer_norm.restype = code
    L.attr_layer_norm.argtypes = [batch, vp, code, i64, i64, vp, vp, code, f32, vp, code, i64, vp, vp, vp]
    L.attr_layer_norm_backward_workspace_size.restype = sz
    L.attr_layer_norm_backward_workspace_size.argtypes = [batch, i64, i32]
    L.attr_layer_norm_backward.restype = code
    L.attr_layer_norm_backward.argtypes = [batch, vp, code, i64, vp, code, i64, i64, vp, vp, vp, code, vp, i64, vp, i64,
                                           vp, i64, i32, i32, vp, sz, vp]
    _lib = L
    return L


_native_modules = None
_native_call = None
_native_rows = None
_native_written = None


def _written(tensors: Sequence[torch.Tensor]) -> None:
    """Counts a change in place of tensors that a call wrote through their pointers, so that a
    backward pass that saved their earlier values raises."""
    global _native_written
    if _native_written is None:
        try:
            from ._marshal import written as _native_written
        except ImportError:  # the calls that need it warn
            _native_written = torch.autograd.graph.increment_version
    _native_written(tensors)


def _native_token_call():
    """The native checks and calls of the token losses, loaded once, as _native()."""
    global _native_call
    if _native_call is None:
        try:
            from ._marshal import token_call
        except ImportError as e:
            warnings.warn(f"_marshal is not available ({e}): token calls check their tensors in Python "
                          "(build it with `python -m paper_2606_11660_amd.build`)", RuntimeWarning, stacklevel=2)

            def token_call(*args):
                return None
        _native_call = token_call
    return _native_call


def _native_rows_call():
    """The native checks and calls of embedding and layer norm, loaded once, as _native()."""
    global _native_rows
    if _native_rows is None:
        try:
            from ._marshal import rows_call
        except ImportError as e:
            warnings.warn(f"_marshal is not available ({e}): calls over token rows check their tensors in Python "
                          "(build it with `python -m paper_2606_11660_amd.build`)", RuntimeWarning, stacklevel=2)

            def rows_call(*args):
                return None
        _native_rows = rows_call
    return _native_rows


def _native():
    """The native gatherer of module descriptors (csrc/marshal.cpp), loaded once.
    Where it was not built, or for another torch, the binding's Python checks take
    every call: the same results, more host time per module."""
    global _native_modules
    if _native_modules is None:
        try:
            from ._marshal import modules
        except ImportError as e:
            warnings.warn(f"_marshal is not available ({e}): projection calls check their modules in Python "
                          "(build it with `python -m paper_2606_11660_amd.build`)", RuntimeWarning, stacklevel=2)

            def modules(*args):
                return None
        _native_modules = modules
    return _native_modules


def _check(status: int) -> None:
    if status != 0:
        raise AttrError(status, lib().attr_last_error().decode(errors="replace"))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _call_stream(stream):
    """The call's stream, looked up once."""
    return torch.cuda.current_stream() if stream is None else stream


def _raw_stream(stream) -> int:
    """The call's stream as a handle, without a Stream object (2.8 us) for the current one."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return _stream(stream)


def _dtype(t: torch.Tensor) -> int:
    if t.dtype not in _TORCH_DTYPE:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return _TORCH_DTYPE[t.dtype]


def _rows(t: torch.Tensor) -> Tuple[int, int, int]:
    """(rows, width, row stride) of a tensor whose last dim is contiguous."""
    if t.dim() < 2 or t.stride(-1) != 1:
        raise ValueError("expected a tensor with a contiguous last dimension")
    width, ld = t.shape[-1], t.stride(-2)
    rows = 1
    for d in range(t.dim() - 1):
        rows *= t.shape[d]
    for d in range(t.dim() - 2):
        if t.stride(d) != t.stride(d + 1) * t.shape[d + 1]:
            raise ValueError("leading dimensions must be packed")
    return rows, width, ld


def _same_gpu(*tensors: Optional[torch.Tensor]) -> None:
    """Every given tensor lives on one GPU (the library takes raw pointers)."""
    ts = [t for t in tensors if t is not None]
    if not ts:
        return
    d = ts[0].device
    for t in ts:
        if not t.is_cuda or t.device != d:
            raise ValueError("every tensor must live on the same GPU device")


def _vector(t: Optional[torch.Tensor], n: int, dtype, name: str) -> None:
    """t is None or a contiguous `dtype` tensor with at least n elements."""
    if t is None:
        return
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of at least {n} elements")


def _torch_stream(stream):
    if stream is None:
        return torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream))


class Workspace:
    """Grow-only device scratch buffer handed to the library calls.

    A workspace serves one stream and one host thread at a time: calls that may
    overlap on different streams need workspaces of their own, and so do calls
    that several threads make on one stream, since a call is several launches
    and another thread's may come between them (the default workspace is kept
    per device, stream and thread).  Every stream of use is recorded on the
    buffer (once: torch's allocator keeps a buffer's streams until it is
    freed), so a buffer replaced by a larger one is not handed out again
    before the work queued on those streams has finished.
    """

    def __init__(self, device=None):
        self.device = torch.device(device or "cuda")
        self.buf = None

    @property
    def buf(self) -> Optional[torch.Tensor]:
        return self._buf

    @buf.setter
    def buf(self, buf: Optional[torch.Tensor]) -> None:
        self._buf = buf
        self._streams = set()  # the raw streams recorded on it

    def get(self, nbytes: int, stream=None) -> Tuple[Optional[int], int]:
        if nbytes == 0:
            return None, 0
        if self._buf is None or self._buf.numel() < nbytes:
            self.buf = torch.empty(int(nbytes), dtype=torch.uint8, device=self.device)
        raw = _stream(stream)
        if raw not in self._streams:
            self._buf.record_stream(_torch_stream(stream))
            self._streams.add(raw)
        return self._buf.data_ptr(), self._buf.numel()


_default_ws: Dict[Tuple[torch.device, int, int], Workspace] = {}


def _ws(ws: Optional[Workspace], device, stream=None) -> Workspace:
    if ws is not None:
        return ws
    # a thread that has ended leaves its identity, and so its workspaces, to a later one
    key = (device, _stream(stream), threading.get_ident())
    if key not in _default_ws:
        _default_ws[key] = Workspace(device)
    return _default_ws[key]


# ----------------------------------------------------------------------------
# (1) projection
# ----------------------------------------------------------------------------
class Module:
    """One linear module's inputs for ``attr_project``.

    a: [..., d_in] activations, g: [..., d_out] output gradients (token rows,
    last dim contiguous); R: [d_out, k], S: [d_in, k] contiguous, same dtype
    as a and g; out_col: first column of the module's k*k block in the output
    row.  v_out [d_out] and v_in [d_in] (fp32, optional, both or neither): the
    factored (Adafactor) second moment that normalises the gradient before
    projection.
    """

    def __init__(self, a: torch.Tensor, g: torch.Tensor, R: torch.Tensor, S: torch.Tensor,
                 out_col: int, v_out: Optional[torch.Tensor] = None,
                 v_in: Optional[torch.Tensor] = None):
        self.a, self.g, self.R, self.S, self.out_col = a, g, R, S, int(out_col)
        self.v_out, self.v_in = v_out, v_in

    def tensors(self):
        return (self.a, self.g, self.R, self.S, self.v_out, self.v_in)

    def c(self) -> _CModule:
        _, d_in, lda = _rows(self.a)
        _, d_out, ldg = _rows(self.g)
        if not (self.R.is_contiguous() and self.S.is_contiguous()):
            raise ValueError("R and S must be contiguous")
        for v, n, name in ((self.v_out, d_out, "v_out"), (self.v_in, d_in, "v_in")):
            if v is not None and (v.dtype != torch.float32 or not v.is_contiguous() or v.numel() != n):
                raise ValueError(f"{name} must be a contiguous fp32 vector of {n} elements")
        return _CModule(self.a.data_ptr(), self.g.data_ptr(), self.R.data_ptr(), self.S.data_ptr(),
                        lda, ldg, d_in, d_out, self.out_col, _ptr(self.v_out), _ptr(self.v_in))


def _cmods(mods: Sequence[Module]):
    arr = (_CModule * len(mods))(*[m.c() for m in mods])
    return arr


def _check_modules(mods: Sequence[Module], k: int, n_examples: int, T: int,
                   row_offset: Optional[torch.Tensor], length: Optional[torch.Tensor],
                   out: torch.Tensor, out_rows_needed: int) -> int:
    """Validate a projection call's tensors against its sizes; returns the
    input dtype code."""
    if not mods:
        raise ValueError("need at least one module")
    dt = mods[0].a.dtype
    if dt not in (torch.float32, torch.bfloat16):
        raise ValueError("token rows must be fp32 or bf16")
    if out.dtype != torch.float32 or out.dim() != 2 or out.stride(1) != 1:
        raise ValueError("out must be fp32 [rows, ldo] with contiguous rows")
    if out.shape[0] < out_rows_needed:
        raise ValueError(f"out has {out.shape[0]} rows, the call writes {out_rows_needed}")
    if n_examples < 0 or T < 1:
        raise ValueError("n_examples must be >= 0 and T >= 1")
    _vector(row_offset, n_examples, torch.int64, "row_offset")
    _vector(length, n_examples, torch.int32, "length")
    for j, m in enumerate(mods):
        for name, t in (("a", m.a), ("g", m.g), ("R", m.R), ("S", m.S)):
            if t.dtype != dt:
                raise ValueError(f"module {j}: {name} is {t.dtype}, module 0's a is {dt}")
        na, d_in, _ = _rows(m.a)
        ng, d_out, _ = _rows(m.g)
        if tuple(m.R.shape) != (d_out, k) or tuple(m.S.shape) != (d_in, k):
            raise ValueError(f"module {j}: R must be [{d_out}, {k}] and S [{d_in}, {k}]")
        if m.out_col < 0 or m.out_col + k * k > out.shape[1]:
            raise ValueError(f"module {j}: columns [{m.out_col}, {m.out_col + k * k}) exceed "
                             f"out's width {out.shape[1]}")
        if row_offset is None and min(na, ng) < n_examples * T:
            raise ValueError(f"module {j}: a/g hold {min(na, ng)} rows, {n_examples} examples "
                             f"of {T} tokens need {n_examples * T}")
    _same_gpu(out, row_offset, length, *[t for m in mods for t in m.tensors()])
    return _dtype(mods[0].a)


def _project_args(mods: Sequence[Module], k: int, n_examples: int, T: int,
                  row_offset: Optional[torch.Tensor], length: Optional[torch.Tensor], out: torch.Tensor,
                  out_rows_needed: int):
    """(dtype code, module descriptors) of a checked projection call."""
    got = _native()(mods, Module, k, n_examples, T, row_offset, length, out, out_rows_needed)
    if got is not None:
        return got[0], (_CModule * len(mods)).from_buffer(got[1])
    return _check_modules(mods, k, n_examples, T, row_offset, length, out, out_rows_needed), _cmods(mods)


def attr_project_workspace_size(mods: Sequence[Module], in_dtype: int, n_examples: int, T: int,
                                k: int) -> int:
    return int(lib().attr_project_workspace_size(_cmods(mods), len(mods), in_dtype, n_examples, T, k))


def attr_project(mods: Sequence[Module], k: int, n_examples: int, T: int,
                 out: torch.Tensor, row_offset: Optional[torch.Tensor] = None,
                 length: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None,
                 stream=None) -> torch.Tensor:
    """P_{i,m} = sum_{t < len_i} (R^T g_t)(S^T a_t)^T into out[i, out_col:out_col+k*k].

    Without row_offset, example i's tokens are rows i*T .. i*T + T - 1 of every
    a and g; with it (int64 [n_examples], device) they start at row_offset[i]
    and the caller keeps every valid token inside a and g (device values
    cannot be checked here).  length: int32 [n_examples] on the device,
    clamped to [0, T] by the library."""
    in_dtype, cm = _project_args(mods, k, n_examples, T, row_offset, length, out, n_examples)
    L = lib()
    stream = _call_stream(stream)
    need = L.attr_project_workspace_size(cm, len(mods), in_dtype, n_examples, T, k)
    wsp, wsn = _ws(ws, out.device, stream).get(need, stream)
    _check(L.attr_project(cm, len(mods), in_dtype, k, n_examples, T, _ptr(row_offset), _ptr(length),
                          out.data_ptr(), out.stride(0), wsp, wsn, _stream(stream)))
    return out


def attr_project_noalloc(mods: Sequence[Module], k: int, n_examples: int, T: int,
                         out: torch.Tensor, row_offset: Optional[torch.Tensor] = None,
                         length: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """attr_project without a workspace: the library's static per-GPU scratch
    (ATTR_PROJECT_NOALLOC_SCRATCH bytes) serves as workspace, so this call
    allocates nothing (usable under graph capture).  Calls that overlap on one
    GPU share that scratch and must be ordered by the caller."""
    in_dtype, cm = _project_args(mods, k, n_examples, T, row_offset, length, out, n_examples)
    _check(lib().attr_project_noalloc(cm, len(mods), in_dtype, k, n_examples, T,
                                      _ptr(row_offset), _ptr(length), out.data_ptr(),
                                      out.stride(0), _stream(stream)))
    return out


def attr_project_tokens(mods: Sequence[Module], k: int, n_examples: int, T: int,
                        out: torch.Tensor, row_offset: Optional[torch.Tensor] = None,
                        length: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None,
                        stream=None) -> torch.Tensor:
    """Per-token blocks (R^T g_t)(S^T a_t)^T into out[token row, out_col:out_col+k*k];
    rows at or past out.shape[0] are not written."""
    in_dtype, cm = _project_args(mods, k, n_examples, T, row_offset, length, out, 0)
    L = lib()
    stream = _call_stream(stream)
    need = L.attr_project_workspace_size(cm, len(mods), in_dtype, n_examples, T, k)
    wsp, wsn = _ws(ws, out.device, stream).get(need, stream)
    _check(L.attr_project_tokens(cm, len(mods), in_dtype, k, n_examples, T, _ptr(row_offset),
                                 _ptr(length), out.data_ptr(), out.stride(0), out.shape[0], wsp, wsn,
                                 _stream(stream)))
    return out


# ----------------------------------------------------------------------------
# (2) preconditioning
# ----------------------------------------------------------------------------
def _check_precond_matrix(t: Optional[torch.Tensor], mode: int, D: int, name: str) -> None:
    """DIAG: fp32 [D]; FULL: fp32 [D, D], contiguous."""
    if mode == PRECOND_NONE:
        if t is not None:
            raise ValueError(f"{name} must be None without a preconditioner")
        return
    want = (D,) if mode == PRECOND_DIAG else (D, D) if mode == PRECOND_FULL else None
    if want is None:
        raise ValueError(f"unknown preconditioner mode {mode}")
    if t is None or t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != want:
        raise ValueError(f"{name} must be a contiguous fp32 tensor of shape {list(want)}")


def attr_precond_accumulate_workspace_size(n_rows: int, D: int, x_dtype: int, mode: int) -> int:
    return int(lib().attr_precond_accumulate_workspace_size(n_rows, D, x_dtype, mode))


def attr_precond_accumulate(X: torch.Tensor, mode: int, H: torch.Tensor,
                            ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """H += diag(X^T X) (DIAG, H [D]) or the upper triangle of X^T X (FULL, H [D, D])."""
    n, D, ldx = _rows(X)
    xd = _dtype(X)
    if mode not in (PRECOND_DIAG, PRECOND_FULL):
        raise ValueError("attr_precond_accumulate takes PRECOND_DIAG or PRECOND_FULL")
    _check_precond_matrix(H, mode, D, "H")
    _same_gpu(X, H)
    L = lib()
    stream = _call_stream(stream)
    need = L.attr_precond_accumulate_workspace_size(n, D, xd, mode)
    wsp, wsn = _ws(ws, X.device, stream).get(need, stream)
    _check(L.attr_precond_accumulate(X.data_ptr(), xd, n, D, ldx, mode, H.data_ptr(), wsp, wsn,
                                     _stream(stream)))
    return H


def attr_precond_apply_workspace_size(n_rows: int, D: int, mode: int) -> int:
    return int(lib().attr_precond_apply_workspace_size(n_rows, D, mode))


def attr_precond_apply(X: torch.Tensor, mode: int, M: Optional[torch.Tensor], unit_normalize: bool,
                       Y: torch.Tensor, ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """Y = unit_normalise(precondition(X)) cast to Y's dtype."""
    n, D, ldx = _rows(X)
    ny, Dy, ldy = _rows(Y)
    if (ny, Dy) != (n, D):
        raise ValueError("X and Y shapes differ")
    _check_precond_matrix(M, mode, D, "M")
    _same_gpu(X, Y, M)
    L = lib()
    stream = _call_stream(stream)
    need = L.attr_precond_apply_workspace_size(n, D, mode)
    wsp, wsn = _ws(ws, X.device, stream).get(need, stream)
    _check(L.attr_precond_apply(X.data_ptr(), _dtype(X), n, D, ldx, mode, _ptr(M),
                                1 if unit_normalize else 0, Y.data_ptr(), _dtype(Y), ldy, wsp, wsn,
                                _stream(stream)))
    return Y


# ----------------------------------------------------------------------------
# (3) scoring
# ----------------------------------------------------------------------------
def attr_score_topk_workspace_size(n_q: int, n_g: int, D: int, k: int) -> int:
    return int(lib().attr_score_topk_workspace_size(n_q, n_g, D, k))


def attr_score_topk(Q: torch.Tensor, G: torch.Tensor, k: int, top_score: torch.Tensor,
                    top_index: torch.Tensor, index_base: int = 0, merge: bool = False,
                    ws: Optional[Workspace] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Exact top-k of <Q_q, G_j> per query, merged with top_* when merge is set."""
    nq, D, ldq = _rows(Q)
    ng, Dg, ldg = _rows(G)
    if Dg != D:
        raise ValueError("Q and G widths differ")
    if Q.dtype != G.dtype:
        raise ValueError("Q and G dtypes differ")
    if top_score.dtype != torch.float32 or top_index.dtype != torch.int64:
        raise ValueError("top_score must be fp32 and top_index int64")
    if not (top_score.is_contiguous() and top_index.is_contiguous()):
        raise ValueError("top_score / top_index must be contiguous")
    if tuple(top_score.shape) != (nq, k) or tuple(top_index.shape) != (nq, k):
        raise ValueError(f"top_score and top_index must be [{nq}, {k}]")
    _same_gpu(Q, G, top_score, top_index)
    L = lib()
    stream = _call_stream(stream)
    need = L.attr_score_topk_workspace_size(nq, ng, D, k)
    wsp, wsn = _ws(ws, Q.device, stream).get(need, stream)
    _check(L.attr_score_topk(Q.data_ptr(), nq, ldq, G.data_ptr(), ng, ldg, _dtype(Q), D, k,
                             index_base, 1 if merge else 0, top_score.data_ptr(),
                             top_index.data_ptr(), wsp, wsn, _stream(stream)))
    return top_score, top_index


# ----------------------------------------------------------------------------
# (4) losses over token log-probabilities
# ----------------------------------------------------------------------------
class TokenRows:
    """A batch's rows of logits and the token each row predicts.

    logits: [n_rows, V] (leading dims packed, last dim contiguous; fp32, bf16 or
    fp16); target: int64 [n_rows]; token t of example i is row i*T + t, or
    row_offset[i] + t.  length (int32 [n_examples]), weight (fp32 [n_rows], 0
    masks a token) and targets outside [0, V) say which tokens count;
    logit_scale is one over the sampling temperature.
    """

    def __init__(self, logits: torch.Tensor, target: torch.Tensor, n_examples: int, T: int,
                 row_offset: Optional[torch.Tensor] = None, length: Optional[torch.Tensor] = None,
                 weight: Optional[torch.Tensor] = None, logit_scale: float = 1.0):
        self.logits, self.target, self.weight = logits, target, weight
        self.n_examples, self.T = int(n_examples), int(T)
        self.row_offset, self.length, self.logit_scale = row_offset, length, float(logit_scale)

    def c(self) -> _CTokenRows:
        """The checked descriptor."""
        n, V, ldl = _rows(self.logits)
        if self.n_examples < 0 or self.T < 1:
            raise ValueError("n_examples must be >= 0 and T >= 1")
        if self.row_offset is None and n < self.n_examples * self.T:
            raise ValueError(f"logits hold {n} rows, {self.n_examples} examples of {self.T} tokens need "
                             f"{self.n_examples * self.T}")
        _vector(self.target, n, torch.int64, "target")
        _vector(self.weight, n, torch.float32, "weight")
        _vector(self.row_offset, self.n_examples, torch.int64, "row_offset")
        _vector(self.length, self.n_examples, torch.int32, "length")
        _same_gpu(self.logits, self.target, self.weight, self.row_offset, self.length)
        return _CTokenRows(self.logits.data_ptr(), _dtype(self.logits), n, V, ldl, self.logit_scale,
                           self.target.data_ptr(), _ptr(self.weight), self.n_examples, self.T,
                           _ptr(self.row_offset), _ptr(self.length))


def attr_token_logp_workspace_size(rows: TokenRows) -> int:
    return int(lib().attr_token_logp_workspace_size(rows.c()))


def attr_policy_loss_workspace_size(rows: TokenRows) -> int:
    return int(lib().attr_policy_loss_workspace_size(rows.c()))


def attr_preference_loss_workspace_size(rows: TokenRows) -> int:
    return int(lib().attr_preference_loss_workspace_size(rows.c()))


_LOGP, _POLICY, _POLICY_PER_TOKEN, _PREFERENCE = range(4)
_TOKEN_ENTRY = ("attr_token_logp", "attr_policy_loss", "attr_policy_loss", "attr_preference_loss")
_token_address: Dict[int, int] = {}


def _token_call(op: int, rows: TokenRows, per_row: tuple, per_example: tuple, per_pair: tuple, scalars: tuple,
                dlogits: Optional[torch.Tensor], ws: Optional[Workspace], stream) -> None:
    """One call of a token loss.  The tuples hold its fp32 vectors (or None) by the number of
    elements that each needs, in the order of csrc/marshal.cpp's token_call()."""
    L = lib()
    if not rows.logits.is_cuda:
        rows.c()  # raises
    raw = _raw_stream(stream)
    w = _ws(ws, rows.logits.device, raw)
    buf = w.buf
    if op not in _token_address:
        _token_address[op] = ctypes.cast(getattr(L, _TOKEN_ENTRY[op]), ctypes.c_void_p).value
    ready = buf is not None and raw in w._streams
    status = _native_token_call()(op, _token_address[op], rows, TokenRows, per_row, per_example, per_pair, dlogits,
                                  scalars, buf.data_ptr() if ready else 0, buf.numel() if ready else 0, raw)
    if status == 0:
        return
    if status is not None and status != 4:
        _check(status)
    # the Python checks, or (ATTR_ERR_WORKSPACE) a workspace that has to grow or that
    # this stream has not used yet
    c = rows.c()
    for ts, n, what in ((per_row, c.n_rows, "row"), (per_example, c.n_examples, "example"),
                        (per_pair, c.n_examples // 2, "pair")):
        for t in ts:
            _vector(t, n, torch.float32, f"a vector with one value for each {what}")
    ldd = 0
    if dlogits is not None:
        n, V, ldd = _rows(dlogits)
        if dlogits.dtype != rows.logits.dtype or (n, V) != (c.n_rows, c.V):
            raise ValueError("dlogits must have the logits' shape and type")
    _same_gpu(rows.logits, dlogits, *per_row, *per_example, *per_pair)
    wsp, wsn = w.get(getattr(L, _TOKEN_ENTRY[op] + "_workspace_size")(c), raw)
    if op == _LOGP:
        args = (_ptr(per_row[0]),)
    elif op == _PREFERENCE:
        args = (_ptr(per_row[1]), _ptr(per_pair[1]), *scalars, _ptr(per_pair[0]), _ptr(per_example[0]),
                _ptr(per_row[0]), _ptr(dlogits), ldd)
    else:
        advantage = per_row[3] if op == _POLICY_PER_TOKEN else per_example[1]
        args = (_ptr(advantage), int(op == _POLICY_PER_TOKEN), _ptr(per_row[1]), _ptr(per_row[2]), *scalars,
                _ptr(per_example[0]), _ptr(per_row[0]), _ptr(dlogits), ldd)
    _check(getattr(L, _TOKEN_ENTRY[op])(c, *args, wsp, wsn, raw))
    # what it wrote stands first in each tuple
    _written([t for t in (dlogits, *per_row[:1], *per_example[:1], *per_pair[:1]) if t is not None])


def attr_token_logp(rows: TokenRows, logp: torch.Tensor, ws: Optional[Workspace] = None,
                    stream=None) -> torch.Tensor:
    """Log-probability of every row's target into logp (fp32 [n_rows]; 0 for tokens that do not count)."""
    _token_call(_LOGP, rows, (logp,), (), (), (), None, ws, stream)
    return logp


def attr_policy_loss(rows: TokenRows, advantage: torch.Tensor, loss: torch.Tensor,
                     logp: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                     logp_old: Optional[torch.Tensor] = None, logp_ref: Optional[torch.Tensor] = None,
                     per_token: bool = False, clip_low: float = 0.2, clip_high: float = 0.2,
                     beta: float = 0.0, ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """Clipped policy loss with a KL term per example into loss (fp32 [n_examples]), and its gradient.

    advantage: fp32 [n_examples], or [n_rows] with per_token; logp_old, logp_ref:
    fp32 [n_rows] (logp_old None: on policy, ratio 1).  dlogits (the logits' shape
    and type, may be the logits themselves: a change in place to autograd) takes the
    gradient of loss.sum(); rows' weights carry the mask and the normalisation."""
    if per_token:
        _token_call(_POLICY_PER_TOKEN, rows, (logp, logp_old, logp_ref, advantage), (loss,), (),
                    (clip_low, clip_high, beta), dlogits, ws, stream)
    else:
        _token_call(_POLICY, rows, (logp, logp_old, logp_ref), (loss, advantage), (), (clip_low, clip_high, beta),
                    dlogits, ws, stream)
    return loss


def attr_preference_loss(rows: TokenRows, loss: torch.Tensor, log_ratio: Optional[torch.Tensor] = None,
                         logp: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                         logp_ref: Optional[torch.Tensor] = None, pair_weight: Optional[torch.Tensor] = None,
                         beta: float = 0.1, margin: float = 0.0, label_smoothing: float = 0.0,
                         ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """Preference loss of n_examples / 2 pairs into loss (fp32 [n_pairs]), and its gradient.

    Pair p: example p was chosen, example n_pairs + p rejected.  log_ratio: fp32
    [n_examples], the weighted sums of logp - logp_ref; dlogits takes the gradient
    of loss.sum(); pair_weight (fp32 [n_pairs]) scales each pair's loss."""
    _token_call(_PREFERENCE, rows, (logp, logp_ref), (log_ratio,), (loss, pair_weight),
                (beta, margin, label_smoothing), dlogits, ws, stream)
    return loss


# ----------------------------------------------------------------------------
# (5) AdamW
# ----------------------------------------------------------------------------
def _refuse_overlaps(spans: List[Tuple[int, int, str, int]]) -> None:
    """spans: (from, to, buffer's name, tensor).  Gradients ("g") are only read and may overlap
    each other; every other buffer stands alone."""
    read = written = (0, 0, "", 0)  # of either kind, the span that reaches furthest so far
    for s in sorted(spans):
        other = read if s[2] != "g" and s[0] < read[1] else written
        if s[0] < other[1]:
            raise ValueError(f"tensor {other[3]}'s {other[2]} and tensor {s[3]}'s {s[2]} overlap")
        if s[2] != "g":
            written = s
        elif s[1] > read[1]:
            read = s


class AdamTensors:
    """A model's tensors for ``attr_adamw_step``, checked once.

    p, g, m, v: lists of contiguous tensors, one of each per weight, with the same
    number of elements; p and g fp32, bf16 or fp16, all of one type each; m and v
    fp32, or torch.float8_e4m3fn with m_scale and v_scale (fp32, one element per
    256 of the tensor's; v then holds the second moment's root).  master: fp32
    weights that the step updates, p taking their rounded values.  weight_decay
    and lr_scale: one number, or one for each tensor.

    The object keeps the tensors and their addresses: give their storage new
    contents, not a new place (a step with gradients elsewhere needs a new object,
    2 us of host time a tensor: keep the gradients' storage between steps).
    """

    def __init__(self, p: Sequence[torch.Tensor], g: Sequence[torch.Tensor], m: Sequence[torch.Tensor],
                 v: Sequence[torch.Tensor], master: Optional[Sequence[torch.Tensor]] = None,
                 m_scale: Optional[Sequence[torch.Tensor]] = None,
                 v_scale: Optional[Sequence[torch.Tensor]] = None, weight_decay=0.0, lr_scale=1.0):
        n = len(p)
        if n == 0:
            raise ValueError("need at least one tensor")
        eight = m[0].dtype == torch.float8_e4m3fn if len(m) else False
        if eight != (m_scale is not None) or eight != (v_scale is not None):
            raise ValueError("m_scale and v_scale go with 8-bit states")
        state = torch.float8_e4m3fn if eight else torch.float32
        kinds = {"p": (p, p[0].dtype), "g": (g, g[0].dtype if len(g) else None), "m": (m, state), "v": (v, state),
                 "master": (master, torch.float32), "m_scale": (m_scale, torch.float32),
                 "v_scale": (v_scale, torch.float32)}
        kinds = {k: x for k, x in kinds.items() if x[0] is not None}
        decay, scale = ([float(x)] * n if isinstance(x, (int, float)) else [float(y) for y in x]
                        for x in (weight_decay, lr_scale))
        for name, ts in [(k, x[0]) for k, x in kinds.items()] + [("weight_decay", decay), ("lr_scale", scale)]:
            if len(ts) != n:
                raise ValueError(f"{name} has {len(ts)} entries, p has {n}")
        self.p_dtype, self.g_dtype = _dtype(p[0]), _dtype(g[0])
        self.state_dtype = ATTR_E4M3 if eight else ATTR_F32
        self.tensors = {k: list(x[0]) for k, x in kinds.items()}
        self.weights = self.tensors["p"] + self.tensors.get("master", [])  # what autograd may have saved
        self.device = device = p[0].device
        if device.type != "cuda":
            raise ValueError("every tensor must live on the same GPU device")
        sizes, address, spans = [t.numel() for t in p], {}, []
        for name, (ts, dtype) in kinds.items():
            want = [-(-x // 256) for x in sizes] if name.endswith("_scale") else sizes
            each, address[name] = dtype.itemsize, [t.data_ptr() for t in ts]
            for j, t in enumerate(ts):
                if t.dtype != dtype or not t.is_contiguous() or t.numel() != want[j]:
                    raise ValueError(f"tensor {j}: {name} must be a contiguous {dtype} tensor of {want[j]} elements")
                if t.device != device:
                    raise ValueError("every tensor must live on the same GPU device")
            spans += [(a, a + x * each, name, j) for j, (a, x) in enumerate(zip(address[name], want)) if x]
        none = [None] * n
        self.array = (_CAdamTensor * n)(*zip(*(address.get(k, none) for k in ("p", "g", "m", "v", "master", "m_scale",
                                                                              "v_scale")), sizes, scale, decay))
        _refuse_overlaps(spans)


def attr_adamw_step(tensors: AdamTensors, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
                    eps: float = 1e-8, eps_root: float = 0.0, grad_scale: Optional[torch.Tensor] = None,
                    stream=None) -> None:
    """AdamW step number `step` (from 1) over every tensor: updates p, m, v (and
    master, scales) in place, which autograd counts as a change of p and master.
    grad_scale: fp32 device scalar that multiplies the gradients.  A graph that
    captured the call repeats this step, with its number and its lr."""
    if grad_scale is not None:
        _vector(grad_scale, 1, torch.float32, "grad_scale")
        if grad_scale.device != tensors.device:
            raise ValueError("every tensor must live on the same GPU device")
    _check(lib().attr_adamw_step(tensors.array, len(tensors.array), tensors.p_dtype, tensors.g_dtype,
                                 tensors.state_dtype, step, lr, beta1, beta2, eps, eps_root, _ptr(grad_scale),
                                 _raw_stream(stream)))
    _written(tensors.weights)


# ----------------------------------------------------------------------------
# (5b) Muon
# ----------------------------------------------------------------------------
class MuonTensors:
    """A model's matrices for ``attr_muon_step``, checked once.

    p, g, m: lists of contiguous 2-D tensors, one of each per weight matrix, of the
    same shape; p and g fp32, bf16 or fp16, all of one type each; m (the momentum)
    fp32.  master: fp32 weights that the step updates, p taking their rounded values.
    weight_decay, lr_scale and update_scale: one number, or one for each matrix.
    lr_scale is of the matrix's rate, so of its decay too, as in ``AdamTensors``;
    update_scale (positive) is of the orthogonal update alone:
        w - lr lr_scale (weight_decay w + update_scale X).
    What a published recipe scales by a matrix's shape is the update: sqrt(max(1, rows / cols)), or
    0.2 sqrt(max(rows, cols)), which makes steps as long as AdamW's and goes with its rate and decay.

    The object keeps the tensors and their addresses: give their storage new
    contents, not a new place.
    """

    def __init__(self, p: Sequence[torch.Tensor], g: Sequence[torch.Tensor], m: Sequence[torch.Tensor],
                 master: Optional[Sequence[torch.Tensor]] = None, weight_decay=0.0, lr_scale=1.0, update_scale=1.0):
        n = len(p)
        if n == 0:
            raise ValueError("need at least one matrix")
        kinds = {"p": (p, p[0].dtype), "g": (g, g[0].dtype if len(g) else None), "m": (m, torch.float32),
                 "master": (master, torch.float32)}
        kinds = {k: x for k, x in kinds.items() if x[0] is not None}
        decay, scale, update = ([float(x)] * n if isinstance(x, (int, float)) else [float(y) for y in x]
                                for x in (weight_decay, lr_scale, update_scale))
        for name, ts in [(k, x[0]) for k, x in kinds.items()] + [("weight_decay", decay), ("lr_scale", scale),
                                                                 ("update_scale", update)]:
            if len(ts) != n:
                raise ValueError(f"{name} has {len(ts)} entries, p has {n}")
        if not all(0.0 < x < float("inf") for x in update):
            raise ValueError("update_scale must be positive and finite")
        # the entry point's rate is of the decay too
        decay, scale = [x / u for x, u in zip(decay, update)], [x * u for x, u in zip(scale, update)]
        self.p_dtype, self.g_dtype = _dtype(p[0]), _dtype(g[0])
        self.tensors = {k: list(x[0]) for k, x in kinds.items()}
        self.weights = self.tensors["p"] + self.tensors.get("master", [])  # what autograd may have saved
        self.device = device = p[0].device
        if device.type != "cuda":
            raise ValueError("every tensor must live on the same GPU device")
        address, spans = {}, []
        for name, (ts, dtype) in kinds.items():
            address[name] = [t.data_ptr() for t in ts]
            for j, t in enumerate(ts):
                if t.dim() != 2 or t.dtype != dtype or not t.is_contiguous() or t.shape != p[j].shape:
                    raise ValueError(f"matrix {j}: {name} must be a contiguous {dtype} tensor of shape {list(p[j].shape)}")
                if t.device != device:
                    raise ValueError("every tensor must live on the same GPU device")
                if t.numel():
                    spans.append((address[name][j], address[name][j] + t.numel() * dtype.itemsize, name, j))
        none = [None] * n
        self.array = (_CMuonMatrix * n)(*zip(*(address.get(k, none) for k in ("p", "g", "m", "master")),
                                             [t.shape[0] for t in p], [t.shape[1] for t in p], scale, decay))
        _refuse_overlaps(spans)
        self._need: Dict[int, int] = {}

    def workspace_size(self, pairs: bool) -> int:
        k = int(pairs)
        if k not in self._need:
            self._need[k] = int(lib().attr_muon_step_workspace_size(self.array, len(self.array), k))
        return self._need[k]

    def default_pairs(self) -> bool:
        return self.p_dtype == ATTR_F32 or "master" in self.tensors


def attr_muon_step_workspace_size(tensors: MuonTensors, pairs: Optional[bool] = None) -> int:
    return tensors.workspace_size(tensors.default_pairs() if pairs is None else pairs)


def attr_muon_step(tensors: MuonTensors, lr: float, momentum: float = 0.95, nesterov: bool = True, steps: int = 5,
                   pairs: Optional[bool] = None, grad_scale: Optional[torch.Tensor] = None,
                   ws: Optional[Workspace] = None, stream=None) -> None:
    """One Muon step over every matrix: updates p and m (and master) in place, which autograd
    counts as a change of p and master.

    pairs: whether the orthogonalisation holds its operands as pairs of fp16 (three times the
    products, an update good to 1e-6 to 4e-6 of its norm) or as fp16 (1.2e-3 to 1.5e-3, and up to some 4e-2 where a
    few directions carry nearly all of it).  None: pairs where the step updates 32-bit weights (p or
    masters), fp16 where it updates 16-bit ones.  grad_scale: fp32 device scalar that multiplies the
    gradients.  A graph that captured the call repeats this step with its lr."""
    if grad_scale is not None:
        _vector(grad_scale, 1, torch.float32, "grad_scale")
        if grad_scale.device != tensors.device:
            raise ValueError("every tensor must live on the same GPU device")
    pairs = tensors.default_pairs() if pairs is None else bool(pairs)
    raw = _here(tensors.weights[0], stream)
    wsp, wsn = _ws(ws, tensors.device, raw).get(tensors.workspace_size(pairs), raw)
    _check(lib().attr_muon_step(tensors.array, len(tensors.array), tensors.p_dtype, tensors.g_dtype, lr, momentum,
                                int(bool(nesterov)), steps, int(pairs), _ptr(grad_scale), wsp, wsn, raw))
    _written(tensors.weights)


# ----------------------------------------------------------------------------
# (6) embedding and layer norm over token rows
# ----------------------------------------------------------------------------
class ExampleRows:
    """The rows of a batch: token t of example i is row i*T + t, or row_offset[i] + t (int64
    [n_examples]); tokens from length[i] on (int32 [n_examples]) are padding, never read, and
    written as zeros without row_offset, not at all with it."""

    def __init__(self, n_examples: int, T: int, row_offset: Optional[torch.Tensor] = None,
                 length: Optional[torch.Tensor] = None):
        self.n_examples, self.T = int(n_examples), int(T)
        self.row_offset, self.length = row_offset, length

    def c(self, n_rows: int) -> _CRows:
        """The checked descriptor of a call over tensors of n_rows rows."""
        if self.n_examples < 0 or self.T < 1:
            raise ValueError("n_examples must be >= 0 and T >= 1")
        if self.row_offset is None and n_rows < self.n_examples * self.T:
            raise ValueError(f"{n_rows} rows, {self.n_examples} examples of {self.T} tokens need "
                             f"{self.n_examples * self.T}")
        _vector(self.row_offset, self.n_examples, torch.int64, "row_offset")
        _vector(self.length, self.n_examples, torch.int32, "length")
        return _CRows(n_rows, self.n_examples, self.T, _ptr(self.row_offset), _ptr(self.length))


_ALL_ROWS = ExampleRows(0, 1)


def _batch(rows: Optional[ExampleRows], n_rows: int) -> Tuple[_CRows, ExampleRows]:
    """The call's rows; without `rows` every row is a token of one example."""
    if rows is None:
        return _CRows(n_rows, 1 if n_rows else 0, max(n_rows, 1), None, None), _ALL_ROWS
    return rows.c(n_rows), rows


def _matrix(t: torch.Tensor, rows: Optional[int], width: int, name: str) -> int:
    """Row stride of a tensor of `rows` (None: any number of) rows of `width` elements."""
    n, w, ld = _rows(t)
    if (rows is not None and n != rows) or w != width:
        raise ValueError(f"{name} must have {rows} rows of {width} elements, it has {n} of {w}")
    return ld if n > 1 else max(ld, w)


_EMBED, _EMBED_BACK, _NORM, _NORM_BACK = range(4)
_ROWS_ENTRY = ("attr_embed", "attr_embed_backward", "attr_layer_norm", "attr_layer_norm_backward")
_rows_address: Dict[int, int] = {}


def _rows_call(op: int, rows: Optional[ExampleRows], tensors: tuple, numbers: tuple, raw: int,
               w: Optional[Workspace] = None) -> bool:
    """One call through csrc/marshal.cpp's rows_call(), the tensors in its order.  False: the Python
    checks decide, or (ATTR_ERR_WORKSPACE) the workspace has to grow or this stream has not used it yet."""
    if op not in _rows_address:
        _rows_address[op] = ctypes.cast(getattr(lib(), _ROWS_ENTRY[op]), ctypes.c_void_p).value
    buf = w.buf if w is not None and raw in w._streams else None
    status = _native_rows_call()(op, _rows_address[op], rows, ExampleRows, tensors, numbers,
                                 0 if buf is None else buf.data_ptr(), 0 if buf is None else buf.numel(), raw)
    if status == 0:
        return True
    if status is not None and status != 4:
        _check(status)
    return False


def _here(t: torch.Tensor, stream) -> int:
    """The call's stream as a handle (0 for a CPU tensor, whose checks raise); the call's tensors live
    on the current device, whose stream it is."""
    on = t.get_device()
    if on < 0:
        return 0
    here = torch.cuda.current_device()
    if on != here:
        raise ValueError("the call's tensors must live on the current GPU device")
    return torch._C._cuda_getCurrentRawStream(here) if stream is None else _stream(stream)


def _tokens(token: torch.Tensor, n_rows: int) -> None:
    _vector(token, n_rows, torch.int64, "token")


def attr_embed(table: torch.Tensor, token: torch.Tensor, out: torch.Tensor, scale: float = 1.0,
               rows: Optional[ExampleRows] = None, stream=None) -> torch.Tensor:
    """out[row] = scale * table[token[row]] (table [V, d], token int64 [n_rows], out [n_rows, d], any
    types); rows of tokens outside [0, V) are zeros."""
    raw = _here(out, stream)
    if _rows_call(_EMBED, rows, (table, token, out), (scale,), raw):
        return out
    n, d, ldo = _rows(out)
    V = table.shape[0]
    ldt = _matrix(table, V, d, "table")
    _tokens(token, n)
    batch, where = _batch(rows, n)
    _same_gpu(table, token, out, where.row_offset, where.length)
    _check(lib().attr_embed(batch, token.data_ptr(), table.data_ptr(), _dtype(table), V, d, ldt, scale, out.data_ptr(),
                            _dtype(out), max(ldo, d), raw))
    _written((out,))
    return out


def attr_embed_backward_workspace_size(n_rows: int, V: int, d: int, rows: Optional[ExampleRows] = None) -> int:
    return int(lib().attr_embed_backward_workspace_size(_batch(rows, n_rows)[0], V, d))


def attr_embed_backward(dout: torch.Tensor, token: torch.Tensor, dtable: torch.Tensor, scale: float = 1.0,
                        accumulate: bool = False, rows: Optional[ExampleRows] = None, ws: Optional[Workspace] = None,
                        stream=None) -> torch.Tensor:
    """dtable[v] = scale * sum of dout's rows whose token is v (zeros where there is none), or with
    accumulate added to what dtable holds.  The same bits for the same call: tokens are sorted,
    and their rows added up in order."""
    raw = _here(dout, stream)
    w = _ws(ws, dout.device, raw) if dout.is_cuda else None
    if _rows_call(_EMBED_BACK, rows, (dtable, token, dout), (scale, accumulate), raw, w):
        return dtable
    n, d, ldd = _rows(dout)
    V = dtable.shape[0]
    ldt = _matrix(dtable, V, d, "dtable")
    _tokens(token, n)
    batch, where = _batch(rows, n)
    _same_gpu(dout, token, dtable, where.row_offset, where.length)
    wsp, wsn = w.get(lib().attr_embed_backward_workspace_size(batch, V, d), raw)
    _check(lib().attr_embed_backward(batch, token.data_ptr(), dout.data_ptr(), _dtype(dout), max(ldd, d), V, d, scale,
                                     dtable.data_ptr(), _dtype(dtable), ldt, int(bool(accumulate)), wsp, wsn, raw))
    _written((dtable,))
    return dtable


def _norm_weights(d: int, *weights: Optional[torch.Tensor]) -> int:
    """The one type of a norm's weights (fp32 without any)."""
    kinds = {w.dtype for w in weights if w is not None}
    if len(kinds) > 1:
        raise ValueError("weight and bias must have one type")
    for w in weights:
        if w is not None and (w.dim() != 1 or w.numel() != d or not w.is_contiguous()):
            raise ValueError(f"weight and bias must be contiguous vectors of {d} elements")
    for w in weights:
        if w is not None:
            return _dtype(w)
    return ATTR_F32


def attr_layer_norm(x: torch.Tensor, y: torch.Tensor, weight: Optional[torch.Tensor] = None,
                    bias: Optional[torch.Tensor] = None, eps: float = 1e-5, mean: Optional[torch.Tensor] = None,
                    rstd: Optional[torch.Tensor] = None, rows: Optional[ExampleRows] = None, stream=None) -> torch.Tensor:
    """y = (x - mean) rstd weight + bias over the last dimension (x, y [n_rows, d], any types; weight
    and bias [d] of one type).  mean, rstd: fp32 [n_rows], what the backward pass takes.  y may be x."""
    raw = _here(x, stream)
    if _rows_call(_NORM, rows, (x, y, weight, bias, mean, rstd), (eps,), raw):
        return y
    n, d, ldx = _rows(x)
    ldy = _matrix(y, n, d, "y")
    w_dtype = _norm_weights(d, weight, bias)
    _vector(mean, n, torch.float32, "mean")
    _vector(rstd, n, torch.float32, "rstd")
    batch, where = _batch(rows, n)
    _same_gpu(x, y, weight, bias, mean, rstd, where.row_offset, where.length)
    _check(lib().attr_layer_norm(batch, x.data_ptr(), _dtype(x), d, max(ldx, d), _ptr(weight), _ptr(bias), w_dtype, eps,
                                 y.data_ptr(), _dtype(y), ldy, _ptr(mean), _ptr(rstd), raw))
    _written([t for t in (y, mean, rstd) if t is not None])
    return y


def attr_layer_norm_backward_workspace_size(n_rows: int, d: int, per_example: bool = False,
                                            rows: Optional[ExampleRows] = None) -> int:
    return int(lib().attr_layer_norm_backward_workspace_size(_batch(rows, n_rows)[0], d, int(bool(per_example))))


def attr_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                             weight: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                             dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                             per_example: bool = False, accumulate: bool = False, rows: Optional[ExampleRows] = None,
                             ws: Optional[Workspace] = None, stream=None) -> None:
    """Gradients of attr_layer_norm into those of dx (x's shape and type; may be x or dy), dweight and
    dbias that are given.  dweight, dbias: fp32 [d], or with per_example [n_examples, d] (rows may be
    columns of wider ones): every example's own.  accumulate adds to what they hold."""
    raw = _here(x, stream)
    w = _ws(ws, x.device, raw) if x.is_cuda else None
    if _rows_call(_NORM_BACK, rows, (x, dy, weight, dx, mean, rstd, dweight, dbias), (per_example, accumulate), raw, w):
        return
    n, d, ldx = _rows(x)
    ldy = _matrix(dy, n, d, "dy")
    w_dtype = _norm_weights(d, weight)
    if mean is None or rstd is None:
        raise ValueError("mean and rstd are what the forward pass gave")
    _vector(mean, n, torch.float32, "mean")
    _vector(rstd, n, torch.float32, "rstd")
    batch, where = _batch(rows, n)
    lddx, lds = 0, []
    if dx is not None:
        lddx = _matrix(dx, n, d, "dx")
        if dx.dtype != x.dtype:
            raise ValueError("dx must have x's type")
    for name, t in (("dweight", dweight), ("dbias", dbias)):
        if t is None:
            lds.append(d)
        elif t.dtype != torch.float32:
            raise ValueError(f"{name} must be fp32")
        elif per_example:
            lds.append(_matrix(t, batch.n_examples, d, name))
        else:
            if t.dim() != 1 or t.numel() != d or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous vector of {d} elements")
            lds.append(d)
    _same_gpu(dy, x, mean, rstd, weight, dx, dweight, dbias, where.row_offset, where.length)
    wsp, wsn = w.get(lib().attr_layer_norm_backward_workspace_size(batch, d, int(bool(per_example))), raw)
    _check(lib().attr_layer_norm_backward(batch, dy.data_ptr(), _dtype(dy), ldy, x.data_ptr(), _dtype(x), d, max(ldx, d),
                                          mean.data_ptr(), rstd.data_ptr(), _ptr(weight), w_dtype, _ptr(dx), lddx,
                                          _ptr(dweight), lds[0], _ptr(dbias), lds[1], int(bool(per_example)),
                                          int(bool(accumulate)), wsp, wsn, raw))
    _written([t for t in (dx, dweight, dbias) if t is not None])


# ----------------------------------------------------------------------------
# calibration (measured peaks; not part of the method)
# ----------------------------------------------------------------------------
def attr_probe_read(x: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """One streaming read of every byte of x (HBM read-bandwidth probe)."""
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    _same_gpu(x, sink)
    _check(lib().attr_probe_read(x.data_ptr(), x.numel() * x.element_size(), sink.data_ptr(),
                                 _stream(stream)))


def attr_probe_mfma(n_mfma: int, sink: torch.Tensor, stream=None) -> int:
    """n_mfma fp16 16x16x32 MFMAs per wave on 2048 waves; returns the flops."""
    _same_gpu(sink)
    _check(lib().attr_probe_mfma(n_mfma, sink.data_ptr(), _stream(stream)))
    return 2 * 16 * 16 * 32 * n_mfma * 2048
