"""Thin ctypes binding of libcavs.so (see include/cavs.h).

Argument marshalling only: every step of the schedule, forward and backward
runs in the library's HIP kernels.  PyTorch supplies device memory and the
stream.  The library must be built (``python -m paper_1712_04048_amd.build``);
loading fails loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as ct
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libcavs.so")

OK = 0
ERR_ARG = -1
ERR_RANGE = -2
ERR_MULTIPARENT = -3
ERR_CYCLE = -4
ERR_MISMATCH = -5
ERR_WORKSPACE = -6
ERR_HIP = -7
ERR_UNSUPPORTED = -8
ERR_DUP_PULL = -9

TREE_LSTM = 0
TREE_FC = 1
FP32 = 0
BF16 = 1
LOSS_CE = 0
LOSS_L2 = 1
LOSS_NONE = 2
T_F32 = 0
T_BF16 = 1

_i32 = ct.c_int32
_vp = ct.c_void_p


class cavs_graphs(ct.Structure):
    _fields_ = [("V", _i32), ("N", _i32), ("n_x", _i32), ("n_push", _i32),
                ("child", _vp), ("parent", _vp), ("pull_idx", _vp), ("push_idx", _vp)]


class cavs_sched(ct.Structure):
    _fields_ = [("T", _i32), ("V", _i32), ("N", _i32), ("n_x", _i32), ("n_push", _i32),
                ("n_pull", _i32), ("n_labelled", _i32), ("n_leaf_noinput", _i32),
                ("n_inner_input", _i32),
                ("level", _vp), ("order", _vp), ("pos", _vp), ("child_pos", _vp),
                ("parent_pos", _vp), ("pull_pos", _vp), ("push_pos", _vp), ("pull_list", _vp),
                ("level_offsets", _vp), ("level_offsets_host", _vp), ("dag", _i32),
                ("in_offsets", _vp), ("in_edges", _vp)]


class cavs_params(ct.Structure):
    _fields_ = [("cell", _i32), ("prec", _i32), ("loss", _i32), ("D", _i32), ("H", _i32),
                ("N", _i32), ("C", _i32),
                ("Wx", _vp), ("U", _vp), ("b", _vp), ("Ws", _vp), ("bs", _vp)]


class cavs_inputs(ct.Structure):
    _fields_ = [("X", _vp), ("Y", _vp), ("n_y", _i32), ("dH_ext", _vp)]


class cavs_grads(ct.Structure):
    _fields_ = [("dWx", _vp), ("dU", _vp), ("db", _vp), ("dWs", _vp), ("dbs", _vp), ("dX", _vp)]


class cavs_launch_time(ct.Structure):
    _fields_ = [("name", ct.c_char * 96), ("row0", _i32), ("rows", _i32), ("ms", ct.c_double)]


class cavs_embedding(ct.Structure):
    _fields_ = [("e_type", _i32), ("x_type", _i32), ("n_words", _i32), ("D", _i32), ("E", _vp),
                ("scale", ct.c_float)]


class cavs_vocab(ct.Structure):
    _fields_ = [("h_type", _i32), ("w_type", _i32), ("n", _i32), ("H", _i32), ("C", _i32),
                ("h", _vp), ("Ws", _vp), ("bs", _vp), ("label", _vp), ("K", _i32),
                ("top_word", _vp), ("top_logit", _vp), ("alpha", ct.c_float),
                ("temp", ct.c_float)]


class cavs_grad(ct.Structure):
    _fields_ = [("g", _vp), ("out", _vp), ("n", ct.c_int64), ("g_type", _i32), ("out_type", _i32)]


class cavs_quant(ct.Structure):
    _fields_ = [("H", _i32), ("C", _i32), ("group", _i32), ("shift", _i32), ("data", _vp)]


class cavs_rules(ct.Structure):
    _fields_ = [("z_type", _i32), ("out_type", _i32), ("n", _i32), ("C", _i32), ("L", _i32),
                ("past", _vp), ("repeat", _vp), ("presence", _vp), ("frequency", _vp), ("bias", _vp),
                ("K", _i32), ("extra_word", _vp), ("extra", _vp), ("M", _i32), ("mask", _vp),
                ("mask_row", _vp), ("temp", _vp)]


EXPORTS = ["cavs_create", "cavs_set_stream", "cavs_destroy", "cavs_last_error", "cavs_sync",
           "cavs_schedule_workspace_bytes", "cavs_schedule", "cavs_schedule_static",
           "cavs_workspace_bytes",
           "cavs_forward", "cavs_backward", "cavs_infer_workspace_bytes", "cavs_infer",
           "cavs_embed", "cavs_embed_grad_workspace_bytes", "cavs_embed_grad",
           "cavs_vocab_workspace_bytes", "cavs_vocab_loss", "cavs_vocab_grad",
           "cavs_clip_workspace_bytes", "cavs_clip_grads", "cavs_quant_bytes", "cavs_quant_pack",
           "cavs_quant_unpack", "cavs_quant_product", "cavs_adjust_workspace_bytes",
           "cavs_adjust_logits",
           "cavs_timing_enable", "cavs_timing_read"]

_lib = None


def lib():
    """Loads libcavs.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libcavs.so is not built: run `python -m paper_1712_04048_amd.build`")
        L = ct.CDLL(LIB_PATH)
        L.cavs_create.restype = _i32
        L.cavs_create.argtypes = [ct.POINTER(_vp), _i32, _vp]
        L.cavs_set_stream.restype = _i32
        L.cavs_set_stream.argtypes = [_vp, _vp]
        L.cavs_destroy.restype = None
        L.cavs_destroy.argtypes = [_vp]
        L.cavs_last_error.restype = ct.c_char_p
        L.cavs_last_error.argtypes = [_vp]
        L.cavs_sync.restype = _i32
        L.cavs_sync.argtypes = [_vp]
        L.cavs_schedule_workspace_bytes.restype = ct.c_size_t
        L.cavs_schedule_workspace_bytes.argtypes = [_i32, _i32, _i32]
        L.cavs_schedule.restype = _i32
        L.cavs_schedule.argtypes = [_vp, ct.POINTER(cavs_graphs), ct.POINTER(cavs_sched), _vp,
                                    ct.c_size_t]
        L.cavs_schedule_static.restype = _i32
        L.cavs_schedule_static.argtypes = [_vp, ct.POINTER(cavs_graphs), ct.POINTER(cavs_sched)]
        L.cavs_workspace_bytes.restype = ct.c_size_t
        L.cavs_workspace_bytes.argtypes = [ct.POINTER(cavs_params), ct.POINTER(cavs_sched)]
        L.cavs_forward.restype = _i32
        L.cavs_forward.argtypes = [_vp, ct.POINTER(cavs_params), ct.POINTER(cavs_sched),
                                   ct.POINTER(cavs_inputs), _vp, _vp, _vp, _vp, ct.c_size_t]
        L.cavs_backward.restype = _i32
        L.cavs_backward.argtypes = [_vp, ct.POINTER(cavs_params), ct.POINTER(cavs_sched),
                                    ct.POINTER(cavs_inputs), _vp, ct.c_size_t,
                                    ct.POINTER(cavs_grads)]
        L.cavs_infer_workspace_bytes.restype = ct.c_size_t
        L.cavs_infer_workspace_bytes.argtypes = [ct.POINTER(cavs_params), ct.POINTER(cavs_sched)]
        L.cavs_infer.restype = _i32
        L.cavs_infer.argtypes = L.cavs_forward.argtypes
        emb, voc = ct.POINTER(cavs_embedding), ct.POINTER(cavs_vocab)
        L.cavs_embed.restype = _i32
        L.cavs_embed.argtypes = [_vp, emb, _vp, _i32, _vp]
        L.cavs_embed_grad_workspace_bytes.restype = ct.c_size_t
        L.cavs_embed_grad_workspace_bytes.argtypes = [emb, _i32]
        L.cavs_embed_grad.restype = _i32
        L.cavs_embed_grad.argtypes = [_vp, emb, _vp, _i32, _vp, _vp, _vp, ct.c_size_t]
        L.cavs_vocab_workspace_bytes.restype = ct.c_size_t
        L.cavs_vocab_workspace_bytes.argtypes = [voc, _i32]
        L.cavs_vocab_loss.restype = _i32
        L.cavs_vocab_loss.argtypes = [_vp, voc, _vp, _vp, _vp, ct.c_size_t]
        L.cavs_vocab_grad.restype = _i32
        L.cavs_vocab_grad.argtypes = [_vp, voc, _vp, _vp, _vp, _vp, _vp, _vp, ct.c_size_t]
        quant, f32 = ct.POINTER(cavs_quant), ct.c_float
        L.cavs_clip_workspace_bytes.restype = ct.c_size_t
        L.cavs_clip_workspace_bytes.argtypes = []
        L.cavs_clip_grads.restype = _i32
        L.cavs_clip_grads.argtypes = [_vp, ct.POINTER(cavs_grad), _i32, f32, f32, _vp, _vp, ct.c_size_t]
        L.cavs_quant_bytes.restype = ct.c_size_t
        L.cavs_quant_bytes.argtypes = [quant]
        L.cavs_quant_pack.restype = _i32
        L.cavs_quant_pack.argtypes = [_vp, quant, _i32, _vp, _vp]
        L.cavs_quant_unpack.restype = _i32
        L.cavs_quant_unpack.argtypes = [_vp, quant, _i32, _vp]
        L.cavs_quant_product.restype = _i32
        L.cavs_quant_product.argtypes = [_vp, quant, _i32, _vp, _i32, _vp, _i32, _vp]
        L.cavs_adjust_workspace_bytes.restype = ct.c_size_t
        L.cavs_adjust_workspace_bytes.argtypes = [_i32, _i32]
        L.cavs_adjust_logits.restype = _i32
        L.cavs_adjust_logits.argtypes = [_vp, ct.POINTER(cavs_rules), _vp, _vp, _vp, _vp, _vp, ct.c_size_t]
        L.cavs_timing_enable.restype = _i32
        L.cavs_timing_enable.argtypes = [_vp, _i32]
        L.cavs_timing_read.restype = _i32
        L.cavs_timing_read.argtypes = [_vp, ct.POINTER(cavs_launch_time), _i32]
        _lib = L
    return _lib


class CavsError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("cavs status %d: %s" % (status, msg))
        self.status = status


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr()


class Context:
    """A library context bound to one device and the current torch stream."""

    def __init__(self, device: int = 0, stream: Optional[torch.cuda.Stream] = None):
        self.device = device
        self.torch_device = torch.device("cuda", device)
        s = stream if stream is not None else torch.cuda.current_stream(self.torch_device)
        self._h = _vp()
        st = lib().cavs_create(ct.byref(self._h), device, s.cuda_stream)
        if st != OK:
            raise CavsError(st, "cavs_create failed")

    def close(self):
        if self._h:
            lib().cavs_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def check(self, st: int):
        if st != OK:
            raise CavsError(st, lib().cavs_last_error(self._h).decode())

    def sync(self):
        """cavs_sync: waits for the context's stream; raises on a kernel-recorded error."""
        self.check(lib().cavs_sync(self._h))

    def set_stream(self, stream: torch.cuda.Stream):
        self.check(lib().cavs_set_stream(self._h, stream.cuda_stream))

    def timing(self, on: bool):
        """Per-launch HIP-event timing of every library kernel (instrumentation)."""
        self.check(lib().cavs_timing_enable(self._h, int(bool(on))))

    def timing_read(self) -> list:
        """[(kernel name, row0, rows, ms)] per launch since the last read; synchronises."""
        cap = 1 << 16
        buf = (cavs_launch_time * cap)()
        n = lib().cavs_timing_read(self._h, buf, cap)
        if n < 0:
            self.check(n)
        return [(buf[i].name.decode(), int(buf[i].row0), int(buf[i].rows), float(buf[i].ms))
                for i in range(min(n, cap))]


@dataclass
class Schedule:
    """Schedule outputs (device tensors, host counts and offsets) plus the
    schedule workspace, reusable across batches of the same size."""
    raw: cavs_sched
    tensors: dict
    level_offsets_host: np.ndarray
    ws: torch.Tensor

    @property
    def T(self) -> int:
        return int(self.raw.T)

    def host(self) -> dict:
        d = {k: v.cpu().numpy() for k, v in self.tensors.items()
             if k not in ("in_offsets", "in_edges")}
        if self.raw.dag:
            d["in_offsets"] = self.tensors["in_offsets"].cpu().numpy()
            d["in_edges"] = self.tensors["in_edges"].cpu().numpy()
        d["level_offsets"] = d["level_offsets"][: self.T + 1]
        d["pull_list"] = d["pull_list"][: self.raw.n_pull]
        d["child_pos"] = d["child_pos"].reshape(-1, self.raw.N)
        d["T"] = self.T
        for k in ("n_pull", "n_labelled", "n_leaf_noinput", "n_inner_input"):
            d[k] = int(getattr(self.raw, k))
        return d


def alloc_schedule(ctx: Context, V: int, N: int, n_x: int) -> Schedule:
    """Allocates the schedule's output arrays and workspace for V vertices."""
    dev = ctx.torch_device
    i32 = dict(dtype=torch.int32, device=dev)
    t = dict(level=torch.empty(V, **i32), order=torch.empty(V, **i32), pos=torch.empty(V, **i32),
             child_pos=torch.empty(V * N, **i32), parent_pos=torch.empty(V, **i32),
             pull_pos=torch.empty(V, **i32), push_pos=torch.empty(V, **i32),
             pull_list=torch.empty(V, **i32), level_offsets=torch.empty(V + 1, **i32),
             in_offsets=torch.empty(V + 1, **i32), in_edges=torch.empty(V * N, **i32))
    host_off = np.zeros(V + 1, dtype=np.int32)
    s = cavs_sched()
    for k, v in t.items():
        setattr(s, k, v.data_ptr() if V > 0 else None)
    s.level_offsets_host = host_off.ctypes.data
    nbytes = lib().cavs_schedule_workspace_bytes(V, N, int(n_x))
    ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    return Schedule(raw=s, tensors=t, level_offsets_host=host_off, ws=ws)


def run_schedule(ctx: Context, sched: Schedule, child: torch.Tensor,
                 parent: Optional[torch.Tensor],
                 pull_idx: Optional[torch.Tensor] = None,
                 push_idx: Optional[torch.Tensor] = None, n_x: int = 0, n_push: int = 0):
    """cavs_schedule into a previously allocated Schedule (one synchronisation).
    parent=None: graph inputs (a vertex may be read by several vertices)."""
    V = int(child.shape[0])
    N = int(child.shape[1]) if child.dim() == 2 else 1
    g = cavs_graphs(V, N, int(n_x), int(n_push), _ptr(child), _ptr(parent), _ptr(pull_idx),
                    _ptr(push_idx))
    nbytes = sched.ws.numel()
    ctx.check(lib().cavs_schedule(ctx._h, ct.byref(g), ct.byref(sched.raw),
                                  sched.ws.data_ptr(), nbytes))
    return sched


SCHEDULE_STATIC_BYTES = 4 << 20   # CAVS_SCHEDULE_STATIC_BYTES


def run_schedule_static(ctx: Context, sched: Schedule, child: torch.Tensor,
                        parent: Optional[torch.Tensor],
                        pull_idx: Optional[torch.Tensor] = None,
                        push_idx: Optional[torch.Tensor] = None, n_x: int = 0, n_push: int = 0):
    """cavs_schedule_static into a previously allocated Schedule: the
    scheduler's scratch comes from the library's static device array, so
    ``sched.ws`` is not used."""
    V = int(child.shape[0])
    N = int(child.shape[1]) if child.dim() == 2 else 1
    g = cavs_graphs(V, N, int(n_x), int(n_push), _ptr(child), _ptr(parent), _ptr(pull_idx),
                    _ptr(push_idx))
    ctx.check(lib().cavs_schedule_static(ctx._h, ct.byref(g), ct.byref(sched.raw)))
    return sched


def schedule(ctx: Context, child: torch.Tensor, parent: Optional[torch.Tensor],
             pull_idx: Optional[torch.Tensor] = None, push_idx: Optional[torch.Tensor] = None,
             n_x: int = 0, n_push: int = 0) -> Schedule:
    """cavs_schedule: int32 device tensors child [V, N], parent [V] (None for
    graph inputs), ..."""
    V = int(child.shape[0])
    N = int(child.shape[1]) if child.dim() == 2 else 1
    sched = alloc_schedule(ctx, V, N, n_x)
    return run_schedule(ctx, sched, child, parent, pull_idx, push_idx, n_x, n_push)


@dataclass
class Params:
    cell: int
    prec: int
    loss: int
    D: int
    H: int
    N: int
    C: int
    Wx: Optional[torch.Tensor]
    U: torch.Tensor
    b: torch.Tensor
    Ws: Optional[torch.Tensor]
    bs: Optional[torch.Tensor]

    def raw(self) -> cavs_params:
        return cavs_params(self.cell, self.prec, self.loss, self.D, self.H, self.N, self.C,
                           _ptr(self.Wx), _ptr(self.U), _ptr(self.b), _ptr(self.Ws),
                           _ptr(self.bs))


def workspace_bytes(params: Params, sched: Schedule) -> int:
    p = params.raw()
    return int(lib().cavs_workspace_bytes(ct.byref(p), ct.byref(sched.raw)))


def forward(ctx: Context, params: Params, sched: Schedule, X: Optional[torch.Tensor],
            Y: Optional[torch.Tensor], ws: torch.Tensor, h_out: torch.Tensor,
            c_out: Optional[torch.Tensor], loss_out: torch.Tensor) -> None:
    """cavs_forward (asynchronous on the context's stream)."""
    p = params.raw()
    inp = cavs_inputs(_ptr(X), _ptr(Y), int(Y.shape[0]) if Y is not None else 0)
    ctx.check(lib().cavs_forward(ctx._h, ct.byref(p), ct.byref(sched.raw), ct.byref(inp),
                                 _ptr(h_out), _ptr(c_out), _ptr(loss_out), ws.data_ptr(),
                                 ws.numel()))


def infer_workspace_bytes(params: Params, sched: Schedule) -> int:
    p = params.raw()
    return int(lib().cavs_infer_workspace_bytes(ct.byref(p), ct.byref(sched.raw)))


def infer(ctx: Context, params: Params, sched: Schedule, X: Optional[torch.Tensor],
          Y: Optional[torch.Tensor], ws: torch.Tensor, h_out: torch.Tensor,
          c_out: Optional[torch.Tensor], loss_out: torch.Tensor) -> None:
    """cavs_infer (asynchronous on the context's stream)."""
    p = params.raw()
    inp = cavs_inputs(_ptr(X), _ptr(Y), int(Y.shape[0]) if Y is not None else 0)
    ctx.check(lib().cavs_infer(ctx._h, ct.byref(p), ct.byref(sched.raw), ct.byref(inp),
                               _ptr(h_out), _ptr(c_out), _ptr(loss_out), ws.data_ptr(),
                               ws.numel()))


def backward(ctx: Context, params: Params, sched: Schedule, X: Optional[torch.Tensor],
             Y: Optional[torch.Tensor], ws: torch.Tensor, grads: dict,
             dH_ext: Optional[torch.Tensor] = None) -> None:
    """cavs_backward (asynchronous); ``grads`` holds dWx, dU, db, dWs, dbs, dX
    tensors; ``dH_ext`` [V, H] (vertex-id rows) is an external gradient of the
    pushed states."""
    p = params.raw()
    inp = cavs_inputs(_ptr(X), _ptr(Y), int(Y.shape[0]) if Y is not None else 0,
                      _ptr(dH_ext))
    g = cavs_grads(*[_ptr(grads.get(k)) for k in ("dWx", "dU", "db", "dWs", "dbs", "dX")])
    ctx.check(lib().cavs_backward(ctx._h, ct.byref(p), ct.byref(sched.raw), ct.byref(inp),
                                  ws.data_ptr(), ws.numel(), ct.byref(g)))


# --------------------------------------------------------------------------
# The two ends of a language model (embedding, vocabulary head)
# --------------------------------------------------------------------------

_TYPES = {torch.float32: T_F32, torch.bfloat16: T_BF16}


def _operand(name: str, t: Optional[torch.Tensor], shape, dtypes, device) -> Optional[int]:
    """The address of a tensor after the checks that the C ABI cannot make."""
    if (isinstance(t, torch.Tensor) and t.dtype in dtypes and t.shape == shape
            and (device is None or t.device == device) and t.is_contiguous()):
        return t.data_ptr() or None   # as most calls pass them, all at once
    if not isinstance(t, torch.Tensor):
        raise CavsError(ERR_ARG, "%s: a tensor is required" % name)
    if t.dtype not in dtypes:
        raise CavsError(ERR_ARG, "%s: %s, not %s" % (name, t.dtype, " or ".join(map(str, dtypes))))
    if tuple(t.shape) != tuple(shape):
        raise CavsError(ERR_ARG, "%s: shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    if device is not None and t.device != device:
        raise CavsError(ERR_ARG, "%s is on %s, the context on %s" % (name, t.device, device))
    if not t.is_contiguous():
        raise CavsError(ERR_ARG, "%s is not contiguous" % name)
    return t.data_ptr() if t.numel() else None


def _sized(name: str, t: torch.Tensor) -> int:
    """The elements of a tensor whose other properties _operand checks."""
    try:
        return t.numel()
    except AttributeError:
        raise CavsError(ERR_ARG, "%s: a tensor is required" % name) from None


def _workspace(ws: torch.Tensor, device):
    n = _sized("ws", ws)
    return _operand("ws", ws, (n,), (torch.uint8,), device), n


@dataclass
class Embedding:
    """A table of word vectors: E [n_words, D] (float32 or bfloat16), scale."""
    E: torch.Tensor
    scale: float = 1.0

    def raw(self, x_dtype, device=None) -> cavs_embedding:
        if not isinstance(self.E, torch.Tensor) or self.E.dim() != 2:
            raise CavsError(ERR_ARG, "E: a tensor [n_words, D] is required")
        if x_dtype not in _TYPES:
            raise CavsError(ERR_ARG, "X: %s is not supported" % x_dtype)
        p = _operand("E", self.E, self.E.shape, _TYPES, device)
        return cavs_embedding(_TYPES[self.E.dtype], _TYPES[x_dtype], int(self.E.shape[0]),
                              int(self.E.shape[1]), p, float(self.scale))


def embed(ctx: Context, emb: Embedding, word: torch.Tensor, X: torch.Tensor) -> None:
    """cavs_embed: X [n, D] = scale * E[word] (asynchronous); int32 word -1: zeros."""
    dev, n = ctx.torch_device, _sized("word", word)
    e = emb.raw(getattr(X, "dtype", None), dev)
    ctx.check(lib().cavs_embed(ctx._h, ct.byref(e), _operand("word", word, (n,), (torch.int32,), dev),
                               n, _operand("X", X, (n, e.D), _TYPES, dev)))


def embed_grad_workspace_bytes(emb: Embedding, n: int) -> int:
    e = emb.raw(torch.float32)
    return int(lib().cavs_embed_grad_workspace_bytes(ct.byref(e), int(n)))


def embed_grad(ctx: Context, emb: Embedding, word: torch.Tensor, dX: torch.Tensor,
               dE: torch.Tensor, ws: torch.Tensor) -> None:
    """cavs_embed_grad: dE [n_words, D] of E's type, overwritten, from dX [n, D]
    (asynchronous)."""
    dev, n = ctx.torch_device, _sized("word", word)
    e = emb.raw(getattr(dX, "dtype", None), dev)
    ctx.check(lib().cavs_embed_grad(
        ctx._h, ct.byref(e), _operand("word", word, (n,), (torch.int32,), dev), n,
        _operand("dX", dX, (n, e.D), _TYPES, dev),
        _operand("dE", dE, (e.n_words, e.D), (emb.E.dtype,), dev), *_workspace(ws, dev)))


@dataclass
class VocabHead:
    """A softmax head over a large vocabulary: h [n, H], Ws [H, C] (float32 or
    bfloat16), bs [C] float32, label [n] int32 (-1: not scored), and a
    teacher's words and logits [n, K] (int32, float32) with their weight alpha
    and temperature temp."""
    h: torch.Tensor
    Ws: torch.Tensor
    bs: Optional[torch.Tensor] = None
    label: Optional[torch.Tensor] = None
    top_word: Optional[torch.Tensor] = None
    top_logit: Optional[torch.Tensor] = None
    alpha: float = 0.0
    temp: float = 1.0

    def raw(self, device=None) -> cavs_vocab:
        for k, t in (("h", self.h), ("Ws", self.Ws)):
            if not isinstance(t, torch.Tensor) or t.dim() != 2:
                raise CavsError(ERR_ARG, "%s: a matrix is required" % k)
        n, H, C = int(self.h.shape[0]), int(self.h.shape[1]), int(self.Ws.shape[1])
        K = 0
        if self.top_word is not None or self.top_logit is not None:
            if (not isinstance(self.top_word, torch.Tensor) or self.top_logit is None
                    or self.top_word.dim() != 2):
                raise CavsError(ERR_ARG, "top_word and top_logit [n, K] go together")
            K = int(self.top_word.shape[1])
        f, i = (torch.float32,), (torch.int32,)
        p = lambda name, t, shape, types: (None if t is None else
                                           _operand(name, t, shape, types, device))
        return cavs_vocab(
            _TYPES.get(self.h.dtype, -1), _TYPES.get(self.Ws.dtype, -1), n, H, C,
            p("h", self.h, (n, H), _TYPES), p("Ws", self.Ws, (H, C), _TYPES),
            p("bs", self.bs, (C,), f), p("label", self.label, (n,), i), K,
            p("top_word", self.top_word, (n, K), i), p("top_logit", self.top_logit, (n, K), f),
            float(self.alpha), float(self.temp))


def vocab_workspace_bytes(head: VocabHead, train: bool) -> int:
    v = head.raw()
    return int(lib().cavs_vocab_workspace_bytes(ct.byref(v), int(bool(train))))


def vocab_loss(ctx: Context, head: VocabHead, loss: torch.Tensor,
               row_loss: Optional[torch.Tensor], ws: torch.Tensor) -> None:
    """cavs_vocab_loss (asynchronous): loss [1], row_loss [n] or None."""
    dev, f = ctx.torch_device, (torch.float32,)
    v = head.raw(dev)
    ctx.check(lib().cavs_vocab_loss(
        ctx._h, ct.byref(v), _operand("loss", loss, (1,), f, dev),
        None if row_loss is None else _operand("row_loss", row_loss, (v.n,), f, dev),
        *_workspace(ws, dev)))


def vocab_grad(ctx: Context, head: VocabHead, loss: torch.Tensor,
               row_loss: Optional[torch.Tensor], dh: torch.Tensor, dWs: torch.Tensor,
               dbs: Optional[torch.Tensor], ws: torch.Tensor) -> None:
    """cavs_vocab_grad (asynchronous): the loss and the gradients dh [n, H],
    dWs [H, C] (of h's and Ws's types) and dbs [C], overwritten."""
    dev, f = ctx.torch_device, (torch.float32,)
    v = head.raw(dev)
    ctx.check(lib().cavs_vocab_grad(
        ctx._h, ct.byref(v), _operand("loss", loss, (1,), f, dev),
        None if row_loss is None else _operand("row_loss", row_loss, (v.n,), f, dev),
        _operand("dh", dh, (v.n, v.H), (head.h.dtype,), dev),
        _operand("dWs", dWs, (v.H, v.C), (head.Ws.dtype,), dev),
        None if dbs is None else _operand("dbs", dbs, (v.C,), f, dev), *_workspace(ws, dev)))


# --------------------------------------------------------------------------
# The end of a training step (gradient norm and clipping)
# --------------------------------------------------------------------------


class GradList:
    """Gradients (float32 or bfloat16, any shapes) and where they go scaled:
    ``out`` a list of as many tensors of the same shapes (None: not written), or
    None for in place.  Holds the tensors; made once for many calls."""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        if len(self.out) != len(self.grads):
            raise CavsError(ERR_ARG, "out: %d tensors for %d gradients" % (len(self.out), len(self.grads)))
        device = None
        self.raw = (cavs_grad * len(self.grads))()
        for k, (g, o) in enumerate(zip(self.grads, self.out)):
            if not isinstance(g, torch.Tensor):
                raise CavsError(ERR_ARG, "gradient %d: a tensor is required" % k)
            device = device if device is not None else g.device
            p = _operand("gradient %d" % k, g, g.shape, _TYPES, device)
            q = None if o is None else _operand("out %d" % k, o, g.shape, _TYPES, device)
            self.raw[k] = cavs_grad(p, q, g.numel(), _TYPES[g.dtype], _TYPES[(g if o is None else o).dtype])
        self.device = device
        written = [r.out for r in self.raw if r.out]
        if len(set(written)) != len(written):
            raise CavsError(ERR_ARG, "out: the same memory twice")


def clip_workspace_bytes() -> int:
    return int(lib().cavs_clip_workspace_bytes())


def clip_grads(ctx: Context, grads: GradList, max_norm: float, norm: torch.Tensor, ws: torch.Tensor,
               scale: float = 1.0) -> None:
    """cavs_clip_grads (asynchronous): norm [1] of all gradients times scale, and
    the gradients times scale, and times max_norm / norm where that is below 1: also
    where float32 holds the norm only as infinity.  A gradient that is not finite leaves
    all of them unclipped."""
    dev = ctx.torch_device
    if not isinstance(grads, GradList):
        raise CavsError(ERR_ARG, "grads: a GradList is required")
    if grads.device is not None and grads.device != dev:
        raise CavsError(ERR_ARG, "the gradients are on %s, the context on %s" % (grads.device, dev))
    ctx.check(lib().cavs_clip_grads(ctx._h, grads.raw, len(grads.grads), float(scale), float(max_norm),
                                    _operand("norm", norm, (1,), (torch.float32,), dev),
                                    *_workspace(ws, dev)))


# --------------------------------------------------------------------------
# The next word (a head in 4 bits, rules on logits)
# --------------------------------------------------------------------------


def quant_bytes(H: int, C: int, group: int = 128, shift: bool = False) -> int:
    """Bytes of the packed weights; 0 for sizes that are refused."""
    q = cavs_quant(int(H), int(C), int(group), int(bool(shift)), None)
    return int(lib().cavs_quant_bytes(ct.byref(q)))


@dataclass
class QuantWeights:
    """Weights [H, C] in 4 bits: data, a uint8 tensor of quant_bytes(H, C, group,
    shift), as quant_pack writes it; group rows share a scale, and with shift a
    shift."""
    data: torch.Tensor
    H: int
    C: int
    group: int = 128
    shift: bool = False

    def raw(self, device=None) -> cavs_quant:
        H, C, group, shift = int(self.H), int(self.C), int(self.group), int(bool(self.shift))
        shape = getattr(self.data, "shape", ())
        if H > 0 and C > 0 and group in (32, 64, 128):
            # cavs_quant_bytes, without a call for each product
            shape = (-(-C // 16) * -(-H // 128) * 16 * (64 + 128 // group * (4 if shift else 2)),)
        # refused sizes are the library's to name
        return cavs_quant(H, C, group, shift, _operand("data", self.data, shape, (torch.uint8,), device))


def quant_pack(ctx: Context, q: QuantWeights, W: torch.Tensor) -> None:
    """cavs_quant_pack (asynchronous): q's data from W [H, C]."""
    dev = ctx.torch_device
    r = q.raw(dev)
    p = _operand("W", W, (q.H, q.C), _TYPES, dev)
    ctx.check(lib().cavs_quant_pack(ctx._h, ct.byref(r), _TYPES[W.dtype], p, r.data))


def quant_unpack(ctx: Context, q: QuantWeights, W: torch.Tensor) -> None:
    """cavs_quant_unpack (asynchronous): W [H, C], the weights that q stands for."""
    dev = ctx.torch_device
    r = q.raw(dev)
    p = _operand("W", W, (q.H, q.C), _TYPES, dev)
    ctx.check(lib().cavs_quant_unpack(ctx._h, ct.byref(r), _TYPES[W.dtype], p))


def quant_product(ctx: Context, q: QuantWeights, x: torch.Tensor, y: torch.Tensor,
                  bias: Optional[torch.Tensor] = None) -> None:
    """cavs_quant_product (asynchronous): y [n, C] = x [n, H] What + bias [C]."""
    dev = ctx.torch_device
    r = q.raw(dev)
    _columns("x", x)
    n = int(x.shape[0])
    px, py = _operand("x", x, (n, q.H), _TYPES, dev), _operand("y", y, (n, q.C), _TYPES, dev)
    pb = None if bias is None else _operand("bias", bias, (q.C,), (torch.float32,), dev)
    ctx.check(lib().cavs_quant_product(ctx._h, ct.byref(r), _TYPES[x.dtype], px, n, pb, _TYPES[y.dtype], py))


_FLOAT, _INT = (torch.float32,), (torch.int32,)


def _columns(name: str, t: torch.Tensor) -> int:
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise CavsError(ERR_ARG, "%s: a matrix is required" % name)
    return int(t.shape[1])


@dataclass
class LogitRules:
    """What turns a model's logits [n, C] into those that its next word is taken
    from: words so far past [n, L] int32 (-1: none) with repeat, presence and
    frequency [n]; bias [C]; extra_word [n, K] int32 with extra [n, K]; mask
    [M, ceil(C / 32)] int32 (bit c % 32 of word c / 32: c may come) with mask_row
    [n] int32 (-1: no mask); temp [n].  Floats are float32; None leaves a rule out."""
    bias: Optional[torch.Tensor] = None
    past: Optional[torch.Tensor] = None
    repeat: Optional[torch.Tensor] = None
    presence: Optional[torch.Tensor] = None
    frequency: Optional[torch.Tensor] = None
    extra_word: Optional[torch.Tensor] = None
    extra: Optional[torch.Tensor] = None
    mask: Optional[torch.Tensor] = None
    mask_row: Optional[torch.Tensor] = None
    temp: Optional[torch.Tensor] = None

    def raw(self, n: int, C: int, z_type: int, out_type: int, device=None) -> cavs_rules:
        r = cavs_rules(z_type, out_type, n, C)
        if self.past is not None:
            r.L = _columns("past", self.past)
            r.past = _operand("past", self.past, (n, r.L), _INT, device)
        elif self.repeat is not None or self.presence is not None or self.frequency is not None:
            raise CavsError(ERR_ARG, "repeat, presence and frequency need past")
        if self.repeat is not None:
            r.repeat = _operand("repeat", self.repeat, (n,), _FLOAT, device)
        if self.presence is not None:
            r.presence = _operand("presence", self.presence, (n,), _FLOAT, device)
        if self.frequency is not None:
            r.frequency = _operand("frequency", self.frequency, (n,), _FLOAT, device)
        if self.bias is not None:
            r.bias = _operand("bias", self.bias, (C,), _FLOAT, device)
        if self.extra_word is not None or self.extra is not None:
            if self.extra_word is None or self.extra is None:
                raise CavsError(ERR_ARG, "extra_word and extra [n, K] go together")
            r.K = _columns("extra_word", self.extra_word)
            r.extra_word = _operand("extra_word", self.extra_word, (n, r.K), _INT, device)
            r.extra = _operand("extra", self.extra, (n, r.K), _FLOAT, device)
        if self.mask is not None:
            _columns("mask", self.mask)
            r.M = int(self.mask.shape[0])
            r.mask = _operand("mask", self.mask, (r.M, -(-C // 32)), _INT, device)
        if self.mask_row is not None:
            r.mask_row = _operand("mask_row", self.mask_row, (n,), _INT, device)
        if self.temp is not None:
            r.temp = _operand("temp", self.temp, (n,), _FLOAT, device)
        return r


def adjust_workspace_bytes(n: int, C: int) -> int:
    return int(lib().cavs_adjust_workspace_bytes(int(n), int(C)))


def adjust_logits(ctx: Context, rules: LogitRules, z: torch.Tensor, out: Optional[torch.Tensor],
                  best: Optional[torch.Tensor], lse: Optional[torch.Tensor], ws: torch.Tensor) -> None:
    """cavs_adjust_logits (asynchronous): out [n, C] (may be z), best [n] int32,
    lse [n] float32; what is None is not written."""
    dev, C = ctx.torch_device, _columns("z", z)
    n = int(z.shape[0])
    pz = _operand("z", z, (n, C), _TYPES, dev)
    po = None if out is None else _operand("out", out, (n, C), _TYPES, dev)
    r = rules.raw(n, C, _TYPES[z.dtype], _TYPES[(z if out is None else out).dtype], dev)
    pb = None if best is None else _operand("best", best, (n,), _INT, dev)
    pl = None if lse is None else _operand("lse", lse, (n,), _FLOAT, dev)
    ctx.check(lib().cavs_adjust_logits(ctx._h, ct.byref(r), pz, po, pb, pl, *_workspace(ws, dev)))
