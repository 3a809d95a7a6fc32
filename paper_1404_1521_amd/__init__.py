"""Python binding of libpolyglot.so, the MI355X (gfx950) HIP library for the
minibatch SGD step of the Polyglot window-ranking language model
(Kulkarni et al., arXiv:1404.1521; model per §1 Introduction, embedding
scatter-add per §4.2-§4.3).

This module only marshals arguments: it checks tensor dtypes, devices and
shapes, passes raw device pointers and the HIP stream to the C ABI of
include/polyglot.h, and raises on a nonzero return code.  Every step of the
computation runs in the library's HIP kernels.  PyTorch supplies device
memory and streams.  There is no fallback: if the library is not built, or no
GPU is present, the calls raise.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import NamedTuple

import torch  # loaded first: the library then binds to torch's HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpolyglot.so")

OK, EINVAL, ENULL, EBATCH, EHIP, EID, ESTATE, EOFFSETS = 0, -1, -2, -3, -4, -5, -6, -7
SCATTER_SORTED, SCATTER_ATOMIC = 0, 1
F32, BF16, F16 = 0, 1, 2      # storage formats of scatter_update
OP_INC, OP_SET = 0, 1         # its operations
GATE_RAW, GATE_SIGMOID = 0, 1  # what a recurrence's gate tensor holds
_CODE_NAMES = {EINVAL: "EINVAL", ENULL: "ENULL", EBATCH: "EBATCH", EHIP: "EHIP", EID: "EID",
               ESTATE: "ESTATE", EOFFSETS: "EOFFSETS"}
_FORMATS = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

# Every entry point declared in include/polyglot.h.
EXPORTS = ("polyglot_init", "polyglot_destroy", "polyglot_set_stream", "polyglot_train_step",
           "polyglot_train_step_sync", "polyglot_train_steps", "polyglot_score", "polyglot_gather", "polyglot_scatter_add",
           "polyglot_scatter_update", "polyglot_scatter_add_noalloc",
           "polyglot_touched_rows", "polyglot_status", "polyglot_last_error",
           "polyglot_set_timing", "polyglot_kernel_times",
           "polyglot_dropout", "polyglot_recurrence", "polyglot_recurrence_grad",
           "polyglot_reserve_recurrence", "polyglot_logits", "polyglot_reserve_logits",
           "polyglot_operator_times",
           "polyglot_convolution", "polyglot_convolution_grad", "polyglot_selective",
           "polyglot_selective_grad", "polyglot_reserve_selective", "polyglot_beam",
           "polyglot_reserve_beam", "polyglot_reorder")
KERNEL_NAMES = ("fwdbwd", "sort", "update", "gather", "scatter", "score", "segfix", "wide_dw1",
                "wide_g")
OPERATOR_NAMES = ("dropout", "recurrence", "recurrence_grad", "logits", "convolution",
                  "convolution_grad", "selective", "selective_grad", "beam", "reorder")
SELECTIVE_MARK = 16  # POLYGLOT_SELECTIVE_MARK


class PolyglotError(RuntimeError):
    def __init__(self, rc: int, msg: str):
        super().__init__(f"{_CODE_NAMES.get(rc, rc)}: {msg}")
        self.rc = rc


class Config(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int32), ("d", ctypes.c_int32), ("win", ctypes.c_int32),
                ("H", ctypes.c_int32), ("max_batch", ctypes.c_int32),
                ("scatter_mode", ctypes.c_int32), ("max_scatter", ctypes.c_int32),
                ("max_rows", ctypes.c_int32)]


def _args(name, *fields):
    """The ctypes mirror of an argument block of include/polyglot.h, with ``pack``: all
    fields in order to the block's bytes, which an entry point takes as it takes a
    pointer to the block."""
    kinds = {"p": (ctypes.c_void_p, "P"), "i": (ctypes.c_int32, "i"), "q": (ctypes.c_int64, "q"),
             "u": (ctypes.c_uint32, "I"), "Q": (ctypes.c_uint64, "Q"), "f": (ctypes.c_float, "f")}
    each = [(n, kinds[k]) for k, names in fields for n in names.split()]
    cls = type(name, (ctypes.Structure,), {"_fields_": [(n, c) for n, (c, _) in each]})
    block = struct.Struct("@" + "".join(f for _, (_, f) in each) + "0q")
    assert block.size == ctypes.sizeof(cls)
    cls.pack = block.pack
    return cls


DropoutArgs = _args("DropoutArgs", ("p", "x add y ids site_dev"), ("q", "rows ld_x ld_add ld_y"),
                    ("Q", "seed first_row"), ("u", "site"), ("f", "p"),
                    ("i", "d dtype id_bytes table_rows whole_rows"))
RecurrenceArgs = _args("RecurrenceArgs", ("p", "gate x h0 offsets h last"),
                       ("q", "tokens ld_gate ld_x ld_h"),
                       ("i", "nseq D group dtype offset_bytes form reverse"))
RecurrenceGradArgs = _args("RecurrenceGradArgs",
                           ("p", "gate x h dh h0 dlast offsets dgate dx dh0"),
                           ("q", "tokens ld_gate ld_x ld_h ld_dh ld_dgate ld_dx"),
                           ("i", "nseq D group dtype offset_bytes form reverse"))
LogitsArgs = _args("LogitsArgs",
                   ("p", "logits out history lengths prompt repetition presence frequency bias "
                         "mask mask_rows token lse"),
                   ("q", "ld_logits ld_out ld_history ld_bias ld_mask"),
                   ("i", "rows V dtype history_cap masks"))

ConvolutionArgs = _args("ConvolutionArgs", ("p", "x weight bias state offsets y last"),
                        ("q", "tokens ld_x ld_y"),
                        ("i", "nseq D taps dtype offset_bytes silu"))
ConvolutionGradArgs = _args("ConvolutionGradArgs",
                            ("p", "x weight bias state dy dlast offsets dx dweight dbias dstate"),
                            ("q", "tokens ld_x ld_dy ld_dx"),
                            ("i", "nseq D taps dtype offset_bytes silu"))
SelectiveArgs = _args("SelectiveArgs",
                      ("p", "x delta B C z A skip delta_bias h0 offsets y last marks"),
                      ("q", "tokens ld_x ld_delta ld_B ld_C ld_z ld_y"),
                      ("i", "nseq D states groups dtype offset_bytes softplus"))
SelectiveGradArgs = _args("SelectiveGradArgs",
                          ("p", "x delta B C z dy A skip delta_bias h0 dlast marks offsets dx "
                                "ddelta dB dC dz dA dskip ddelta_bias dh0"),
                          ("q", "tokens ld_x ld_delta ld_B ld_C ld_z ld_dy ld_dx ld_ddelta ld_dB "
                                "ld_dC ld_dz"),
                          ("i", "nseq D states groups dtype offset_bytes softplus"))
BeamArgs = _args("BeamArgs", ("p", "scores total lse finished parent token out"),
                 ("q", "ld_scores"), ("i", "groups beams V picks end dtype"))
RowCopy = _args("RowCopy", ("p", "in_ out"), ("q", "row_bytes ld_in ld_out"),
                ("i", "in_rows reserved"))


class ConvolutionGrads(NamedTuple):
    """The gradients of a convolution's inputs; state is None where none was given."""
    x: torch.Tensor
    weight: torch.Tensor
    bias: torch.Tensor | None
    state: torch.Tensor | None


class SelectiveGrads(NamedTuple):
    """The gradients of a selective scan's inputs, None for those that were not given."""
    x: torch.Tensor
    delta: torch.Tensor
    A: torch.Tensor
    B: torch.Tensor
    C: torch.Tensor
    skip: torch.Tensor | None
    z: torch.Tensor | None
    delta_bias: torch.Tensor | None
    state: torch.Tensor | None


_lib = None


def load_library():
    """Loads libpolyglot.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run paper_1404_1521_amd.build.build()")
    lib = ctypes.CDLL(LIB_PATH)
    p, i32, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
    sig = {
        "polyglot_init": [ctypes.POINTER(Config), p, ctypes.POINTER(p)],
        "polyglot_destroy": [p],
        "polyglot_set_stream": [p, p],
        "polyglot_train_step": [p] + [p] * 7 + [i32, f32, p],
        "polyglot_train_step_sync": [p] + [p] * 7 + [i32, f32, ctypes.POINTER(f32)],
        "polyglot_train_steps": [p] + [p] * 7 + [i32, i32, f32, p],
        "polyglot_score": [p] + [p] * 6 + [i32, p],
        "polyglot_gather": [p, p, p, p, i32, p, p],
        "polyglot_scatter_add": [p, p, i32, i32, p, p, i32, f32, i32],
        "polyglot_scatter_update": [p, p, i32, i32, i32, p, i32, p, i32, f32, i32, i32],
        "polyglot_scatter_add_noalloc": [p, i32, i32, p, p, i32, f32, p, p],
        "polyglot_touched_rows": [p, p, i32, p],
        "polyglot_status": [p],
        "polyglot_last_error": [p],
        "polyglot_set_timing": [p, ctypes.c_int],
        "polyglot_kernel_times": [p, p, p],
        "polyglot_dropout": [p, p],
        "polyglot_recurrence": [p, p],
        "polyglot_recurrence_grad": [p, p],
        "polyglot_reserve_recurrence": [p, ctypes.c_int64, i32],
        "polyglot_logits": [p, p],
        "polyglot_reserve_logits": [p, i32, i32],
        "polyglot_operator_times": [p, p, p],
        "polyglot_convolution": [p, p],
        "polyglot_convolution_grad": [p, p],
        "polyglot_selective": [p, p],
        "polyglot_selective_grad": [p, p],
        "polyglot_reserve_selective": [p, ctypes.c_int64, i32, i32],
        "polyglot_beam": [p, p],
        "polyglot_reserve_beam": [p, i32, i32, i32],
        "polyglot_reorder": [p, p, i32, p, i32],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_char_p if name == "polyglot_last_error" else ctypes.c_int
    _lib = lib
    return lib


def _dev_tensor(t, dtype, name, shape=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a device (cuda) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _row_tensor(t, dtype, name, rows, width):
    """Pointer and row distance of a device tensor [rows][width] whose rows are
    consecutive elements, any distance apart."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device (cuda) tensor")
    if t.shape != (rows, width):
        raise ValueError(f"{name} must have shape {(rows, width)}, got {tuple(t.shape)}")
    if t.is_contiguous():
        return t.data_ptr(), width
    ld, one = t.stride()
    if one != 1 and width > 1 and rows > 0:
        raise ValueError(f"{name} must have consecutive elements in its rows")
    return t.data_ptr(), ld if rows > 1 else width


def _vector(t, dtype, name, n):
    """Pointer of a contiguous device vector of n values (None: 0)."""
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device (cuda) tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != (n,):
        raise ValueError(f"{name} must have shape {(n,)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _state(t, name, nseq, D):
    """Pointer of a contiguous float32 device tensor [nseq][D] (None: 0)."""
    if t is None:
        return 0
    p, ld = _row_tensor(t, torch.float32, name, nseq, D)
    if ld != D:
        raise ValueError(f"{name} must be contiguous")
    return p


def _format(t, name):
    """A tensor's storage format and dtype."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    code = _FORMATS.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code, t.dtype


def _offsets(t):
    """Pointer and size of an offset of a vector of sequence offsets (None: 0, 0)."""
    if t is None:
        return 0, 0
    if t.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"offsets must be int32 or int64, got {t.dtype}")
    return _vector(t, t.dtype, "offsets", t.shape[0]), t.element_size()


def _block(t, dtype, name, shape):
    """Pointer of a contiguous device tensor of this shape (None: 0)."""
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device (cuda) tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _like(t):
    """A new contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _flat(t):
    """A [nseq][T][width] tensor as rows of tokens."""
    return t if t is None or t.dim() == 2 else t.view(-1, t.shape[-1])


NOALLOC_MAX_N = 8192  # POLYGLOT_NOALLOC_MAX_N


def scatter_add_noalloc(table, idx, Y, alpha: float = 1.0, status=None, stream=None) -> None:
    """table[idx[k]] += alpha * Y[k] (sorted mode) through the entry point that
    allocates nothing and needs no context (N <= NOALLOC_MAX_N).  status: an
    optional int32 device tensor of one element that receives OK or EID on
    the device.  Asynchronous on `stream` (default: torch's current stream)."""
    lib = load_library()
    rows, d = table.shape
    N = idx.shape[0]
    st = stream if stream is not None else torch.cuda.current_stream()
    sp = None if status is None else _dev_tensor(status, torch.int32, "status", (1,))
    rc = lib.polyglot_scatter_add_noalloc(
        _dev_tensor(table, torch.float32, "table"), rows, d,
        _dev_tensor(idx, torch.int32, "idx", (N,)),
        _dev_tensor(Y, torch.float32, "Y", (N, d)), N, alpha, sp,
        ctypes.c_void_p(st.cuda_stream))
    if rc != OK:
        raise PolyglotError(rc, "scatter_add_noalloc")


class Context:
    """A library context (workspace + stream) for one model shape."""

    def __init__(self, V: int, d: int, win: int, H: int, max_batch: int,
                 scatter_mode: int = SCATTER_SORTED, max_scatter: int = 0, max_rows: int = 0,
                 stream: torch.cuda.Stream | None = None):
        self._lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the Polyglot HIP library needs an MI355X device")
        self.cfg = Config(V, d, win, H, max_batch, scatter_mode, max_scatter, max_rows)
        self.V, self.d, self.win, self.H = V, d, win, H
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        h = ctypes.c_void_p()
        rc = self._lib.polyglot_init(ctypes.byref(self.cfg), ctypes.c_void_p(self.stream.cuda_stream),
                                     ctypes.byref(h))
        if rc != OK:
            raise PolyglotError(rc, "polyglot_init failed")
        self._h = h

    # ------------------------------------------------------------------ helpers
    def _check(self, rc: int, what: str):
        if rc != OK:
            msg = self._lib.polyglot_last_error(self._h)
            raise PolyglotError(rc, f"{what}: {msg.decode() if msg else ''}")

    def _params(self, params: dict):
        V, d, win, H = self.V, self.d, self.win, self.H
        return [_dev_tensor(params["E"], torch.float32, "E", (V, d)),
                _dev_tensor(params["W1"], torch.float32, "W1", (H, win * d)),
                _dev_tensor(params["b1"], torch.float32, "b1", (H,)),
                _dev_tensor(params["w2"], torch.float32, "w2", (H,)),
                _dev_tensor(params["b2"], torch.float32, "b2", (1,))]

    # -------------------------------------------------------------- entry points
    def train_step(self, params: dict, windows, corrupt, lr: float, loss_out=None) -> None:
        """One SGD step in place on params (asynchronous on the context stream)."""
        B = windows.shape[0]
        args = self._params(params)
        w = _dev_tensor(windows, torch.int32, "windows", (B, self.win))
        c = _dev_tensor(corrupt, torch.int32, "corrupt", (B,))
        lo = None if loss_out is None else _dev_tensor(loss_out, torch.float32, "loss_out")
        self._check(self._lib.polyglot_train_step(self._h, *args, w, c, B, lr, lo), "train_step")

    def train_step_sync(self, params: dict, windows, corrupt, lr: float) -> float:
        """One SGD step in place on params; synchronises the context stream and
        returns the step's mean loss as a Python float."""
        B = windows.shape[0]
        args = self._params(params)
        w = _dev_tensor(windows, torch.int32, "windows", (B, self.win))
        c = _dev_tensor(corrupt, torch.int32, "corrupt", (B,))
        loss = ctypes.c_float(0.0)
        self._check(self._lib.polyglot_train_step_sync(self._h, *args, w, c, B, lr,
                                                       ctypes.byref(loss)), "train_step_sync")
        return loss.value

    def train_steps(self, params: dict, windows, corrupt, lr: float, losses_out=None) -> None:
        """S steps over windows[S][B][win], corrupt[S][B] (graph-replayed)."""
        S, B = windows.shape[0], windows.shape[1]
        args = self._params(params)
        w = _dev_tensor(windows, torch.int32, "windows", (S, B, self.win))
        c = _dev_tensor(corrupt, torch.int32, "corrupt", (S, B))
        lo = None if losses_out is None else _dev_tensor(losses_out, torch.float32, "losses", (S,))
        self._check(self._lib.polyglot_train_steps(self._h, *args, w, c, S, B, lr, lo),
                    "train_steps")

    def score(self, params: dict, windows, out=None):
        B = windows.shape[0]
        if out is None:
            out = torch.empty(B, dtype=torch.float32, device=windows.device)
        args = self._params(params)
        w = _dev_tensor(windows, torch.int32, "windows", (B, self.win))
        o = _dev_tensor(out, torch.float32, "scores", (B,))
        self._check(self._lib.polyglot_score(self._h, *args, w, B, o), "score")
        return out

    def gather(self, E, windows, corrupt, X=None, Xc=None):
        B = windows.shape[0]
        if X is None:
            X = torch.empty(B, self.win * self.d, dtype=torch.float32, device=E.device)
        if Xc is None:
            Xc = torch.empty(B, self.d, dtype=torch.float32, device=E.device)
        self._check(self._lib.polyglot_gather(
            self._h, _dev_tensor(E, torch.float32, "E", (self.V, self.d)),
            _dev_tensor(windows, torch.int32, "windows", (B, self.win)),
            _dev_tensor(corrupt, torch.int32, "corrupt", (B,)), B,
            _dev_tensor(X, torch.float32, "X", (B, self.win * self.d)),
            _dev_tensor(Xc, torch.float32, "Xc", (B, self.d))), "gather")
        return X, Xc

    def scatter_add(self, table, idx, Y, alpha: float = 1.0, mode: int = SCATTER_SORTED) -> None:
        """table[idx[k]] += alpha * Y[k] for every k (repeated indices accumulate)."""
        rows, d = table.shape
        N = idx.shape[0]
        self._check(self._lib.polyglot_scatter_add(
            self._h, _dev_tensor(table, torch.float32, "table"), rows, d,
            _dev_tensor(idx, torch.int32, "idx", (N,)),
            _dev_tensor(Y, torch.float32, "Y", (N, d)), N, alpha, mode), "scatter_add")

    def scatter_update(self, table, idx, Y, alpha: float = 1.0, op: int = OP_INC,
                       mode: int = SCATTER_SORTED) -> None:
        """The general advanced-indexing op on a float32, bfloat16 or float16
        table (Y in the same dtype) with int32 or int64 indices: op=OP_INC
        adds alpha * Y[k] into row idx[k]; op=OP_SET assigns Y[k] (the last
        k of a row wins)."""
        codes = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
        if table.dtype not in codes:
            raise TypeError(f"table must be float32, bfloat16 or float16, got {table.dtype}")
        if idx.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"idx must be int32 or int64, got {idx.dtype}")
        rows, d = table.shape
        N = idx.shape[0]
        self._check(self._lib.polyglot_scatter_update(
            self._h, _dev_tensor(table, table.dtype, "table"), codes[table.dtype], rows, d,
            _dev_tensor(idx, idx.dtype, "idx", (N,)), idx.element_size(),
            _dev_tensor(Y, table.dtype, "Y", (N, d)), N, alpha, op, mode), "scatter_update")

    def touched_rows(self):
        n = ctypes.c_int32()
        self._check(self._lib.polyglot_touched_rows(self._h, None, 0, ctypes.byref(n)),
                    "touched_rows")
        buf = (ctypes.c_int32 * max(n.value, 1))()
        self._check(self._lib.polyglot_touched_rows(self._h, buf, n.value, ctypes.byref(n)),
                    "touched_rows")
        return list(buf)[: n.value]

    def set_timing(self, enable: bool) -> None:
        self._check(self._lib.polyglot_set_timing(self._h, int(enable)), "set_timing")

    def kernel_times(self) -> dict:
        """{kernel name: (total ms, launches)} since the last call; synchronises."""
        ms = (ctypes.c_double * len(KERNEL_NAMES))()
        n = (ctypes.c_int32 * len(KERNEL_NAMES))()
        self._check(self._lib.polyglot_kernel_times(self._h, ms, n), "kernel_times")
        return {name: (ms[i], n[i]) for i, name in enumerate(KERNEL_NAMES)}

    # ------------------------------------------------------------ sequences
    def reserve_recurrence(self, max_tokens: int, max_width: int) -> None:
        """Workspace for recurrences of up to max_tokens tokens and max_width channels."""
        self._check(self._lib.polyglot_reserve_recurrence(self._h, max_tokens, max_width),
                    "reserve_recurrence")

    def reserve_logits(self, max_rows: int, max_vocab: int) -> None:
        """Workspace for the choices of up to max_rows rows of max_vocab scores."""
        self._check(self._lib.polyglot_reserve_logits(self._h, max_rows, max_vocab),
                    "reserve_logits")

    def dropout(self, x, p: float, seed: int, *, site: int = 0, site_dev=None, first_row: int = 0,
                ids=None, add=None, whole_rows: bool = False, out=None):
        """out[r] = dropout(x[r]) (+ add[r]), or of the rows ids[r] of a table x.  The mask
        is a function of (seed, site + site_dev, first_row + r, column) alone and is never
        stored; dropout_backward computes it again.  float32, bfloat16 or float16."""
        code, dtype = _format(x, "x")
        if x.dim() != 2:
            raise ValueError("x must have two dimensions")
        rows, d = x.shape
        px, ld_x = _row_tensor(x, dtype, "x", rows, d)
        pids = id_bytes = table_rows = padd = ld_add = 0
        if ids is not None:
            if ids.dtype not in (torch.int32, torch.int64):
                raise TypeError(f"ids must be int32 or int64, got {ids.dtype}")
            table_rows, rows = rows, ids.shape[0]
            pids, id_bytes = _vector(ids, ids.dtype, "ids", rows), ids.element_size()
        if add is not None:
            padd, ld_add = _row_tensor(add, dtype, "add", rows, d)
        if out is None:
            out = _like(x) if ids is None else x.new_empty((rows, d))
        py, ld_y = _row_tensor(out, dtype, "out", rows, d)
        rc = self._lib.polyglot_dropout(self._h, DropoutArgs.pack(
            px, padd, py, pids, _vector(site_dev, torch.int32, "site_dev", 1), rows, ld_x, ld_add,
            ld_y, seed & 0xFFFFFFFFFFFFFFFF, first_row, site & 0xFFFFFFFF, p, d, code, id_bytes,
            table_rows, whole_rows))
        if rc != OK:
            self._check(rc, "dropout")
        return out

    def dropout_backward(self, dy, p: float, seed: int, *, site: int = 0, site_dev=None,
                         first_row: int = 0, whole_rows: bool = False, out=None):
        """The gradient of dropout's x (per row read, when x was a table), for the same
        seed, site and first_row.  That of its add is dy itself."""
        return self.dropout(dy, p, seed, site=site, site_dev=site_dev, first_row=first_row,
                            whole_rows=whole_rows, out=out)

    @staticmethod
    def _sequences(x, gate, offsets):
        """What a recurrence and its gradient share of their inputs' checks: storage format,
        dtype, token count, channels, gates, and the gate's, x's and the offsets' pointers."""
        code, dtype = _format(x, "x")
        tokens, D = x.shape
        gates = gate.shape[-1]
        if gates < 1 or D % gates:
            raise ValueError(f"gate has {gates} columns, which do not divide {D} channels")
        poff = off_bytes = 0
        if offsets is not None:
            if offsets.dtype not in (torch.int32, torch.int64):
                raise TypeError(f"offsets must be int32 or int64, got {offsets.dtype}")
            poff = _vector(offsets, offsets.dtype, "offsets", offsets.shape[0])
            off_bytes = offsets.element_size()
        return (code, dtype, tokens, D, gates, *_row_tensor(gate, dtype, "gate", tokens, gates),
                *_row_tensor(x, dtype, "x", tokens, D), poff, off_bytes)

    def _forward(self, what, gate, x, offsets, nseq, h0, form, reverse, out, last):
        code, dtype, tokens, D, gates, pg_, ld_g, px, ld_x, poff, off_bytes = self._sequences(
            x, gate, offsets)
        if last is None:
            last = x.new_empty((nseq, D), dtype=torch.float32)
        ph, ld_h = _row_tensor(_flat(out), dtype, "out", tokens, D)
        rc = self._lib.polyglot_recurrence(self._h, RecurrenceArgs.pack(
            pg_, px, _state(h0, "h0", nseq, D), poff, ph, _state(last, "last", nseq, D), tokens,
            ld_g, ld_x, ld_h, nseq, D, D // gates, code, off_bytes, form, reverse))
        if rc != OK:
            self._check(rc, what)
        return out, last

    def recurrence(self, gate, x, offsets=None, *, h0=None, form: int = GATE_SIGMOID,
                   reverse: bool = False, out=None, last=None):
        """h_t = a_t h_{t-1} + x_t (GATE_RAW) or a_t h_{t-1} + (1 - a_t) x_t (GATE_SIGMOID,
        a the gate's sigmoid) over the sequences of x: [tokens][D] with offsets[nseq + 1],
        [nseq][T][D] without, or one sequence [T][D].  gate has D columns, or fewer that
        divide D, each for D / columns consecutive channels.  h0 and last are float32
        [nseq][D].  Returns (h, last)."""
        nseq = offsets.shape[0] - 1 if offsets is not None else x.shape[0] if x.dim() == 3 else 1
        if out is None:
            out = _like(x)
        return self._forward("recurrence", _flat(gate), _flat(x), offsets, nseq, h0, form, reverse,
                             out, last)

    def recurrence_step(self, gate, x, state=None, *, form: int = GATE_SIGMOID, out=None,
                        last=None):
        """One token x[nseq][D] for each of nseq sequences whose float32 states are
        state[nseq][D].  Returns (h, the new states); last=state updates them in place."""
        if out is None:
            out = _like(x)
        if last is None and state is not None:
            last = _like(state)
        return self._forward("recurrence_step", gate, x, None, x.shape[0], state, form, False, out,
                             last)

    def recurrence_backward(self, gate, x, h, dh, offsets=None, *, h0=None, dlast=None,
                            form: int = GATE_SIGMOID, reverse: bool = False, dgate=None, dx=None,
                            dh0=None):
        """The gradient of recurrence, for its inputs, its output h and the gradients dh of h
        and dlast of last.  Returns (dgate, dx, dh0); dh0 is None unless h0 or dh0 is given."""
        nseq = offsets.shape[0] - 1 if offsets is not None else x.shape[0] if x.dim() == 3 else 1
        if dgate is None:
            dgate = _like(gate)
        if dx is None:
            dx = _like(x)
        code, dtype, tokens, D, gates, pg_, ld_g, px, ld_x, poff, off_bytes = self._sequences(
            _flat(x), _flat(gate), offsets)
        if dh0 is None and h0 is not None:
            dh0 = x.new_empty((nseq, D), dtype=torch.float32)
        ph, ld_h = _row_tensor(_flat(h), dtype, "h", tokens, D)
        pdh, ld_dh = _row_tensor(_flat(dh), dtype, "dh", tokens, D)
        pdg, ld_dg = _row_tensor(_flat(dgate), dtype, "dgate", tokens, gates)
        pdx, ld_dx = _row_tensor(_flat(dx), dtype, "dx", tokens, D)
        rc = self._lib.polyglot_recurrence_grad(self._h, RecurrenceGradArgs.pack(
            pg_, px, ph, pdh, _state(h0, "h0", nseq, D), _state(dlast, "dlast", nseq, D), poff, pdg,
            pdx, _state(dh0, "dh0", nseq, D), tokens, ld_g, ld_x, ld_h, ld_dh, ld_dg, ld_dx, nseq,
            D, D // gates, code, off_bytes, form, reverse))
        if rc != OK:
            self._check(rc, "recurrence_backward")
        return dgate, dx, dh0

    def logits(self, logits, *, history=None, lengths=None, prompt=None, repetition=None,
               presence=None, frequency=None, bias=None, mask=None, mask_rows=None, out=None,
               write: bool = True):
        """The scores logits[rows][V] with penalties for the words of history[rows][cap], a
        bias[V] or [rows][V], and the mask's bits (int32 words; see polyglot_logits).
        Returns (out, token, lse): the scores in their own dtype (out may be logits itself;
        None with write=False), the int32 choice of each row and its float32 log-sum-exp."""
        code, dtype = _format(logits, "logits")
        if logits.dim() != 2:
            raise ValueError("logits must have two dimensions")
        rows, V = logits.shape
        pl, ld_l = _row_tensor(logits, dtype, "logits", rows, V)
        po = ld_o = ph = ld_h = cap = plen = ppr = pb = ld_b = pm = ld_m = masks = pmr = 0
        if out is None and write:
            out = _like(logits)
        if out is not None:
            po, ld_o = _row_tensor(out, dtype, "out", rows, V)
        if history is not None:
            cap = history.shape[1]
            ph, ld_h = _row_tensor(history, torch.int32, "history", rows, cap)
            plen = _vector(lengths, torch.int32, "lengths", rows)
            ppr = _vector(prompt, torch.int32, "prompt", rows)
        if bias is not None and bias.dim() == 1:
            pb = _vector(bias, torch.float32, "bias", V)
        elif bias is not None:
            pb, ld_b = _row_tensor(bias, torch.float32, "bias", rows, V)
        if mask is not None:
            masks = mask.shape[0]
            pm, ld_m = _row_tensor(mask, torch.int32, "mask", masks, (V + 31) // 32)
            pmr = _vector(mask_rows, torch.int32, "mask_rows", rows)
        token = logits.new_empty(rows, dtype=torch.int32)
        lse = logits.new_empty(rows, dtype=torch.float32)
        rc = self._lib.polyglot_logits(self._h, LogitsArgs.pack(
            pl, po, ph, plen, ppr, _vector(repetition, torch.float32, "repetition", rows),
            _vector(presence, torch.float32, "presence", rows),
            _vector(frequency, torch.float32, "frequency", rows), pb, pm, pmr, token.data_ptr(),
            lse.data_ptr(), ld_l, ld_o, ld_h, ld_b, ld_m, rows, V, code, cap, masks))
        if rc != OK:
            self._check(rc, "logits")
        return out, token, lse

    def reserve_selective(self, max_tokens: int, max_width: int, max_states: int) -> None:
        """Workspace for selective scans, their gradients and the convolution's of up to max_width
        channels and max_states states; for the scan's gradient of up to max_tokens tokens (0
        where nothing is trained)."""
        self._check(self._lib.polyglot_reserve_selective(self._h, max_tokens, max_width,
                                                         max_states), "reserve_selective")

    def reserve_beam(self, max_rows: int, max_vocab: int, max_picks: int) -> None:
        """Workspace for selections among up to max_rows beams of max_vocab scores."""
        self._check(self._lib.polyglot_reserve_beam(self._h, max_rows, max_vocab, max_picks),
                    "reserve_beam")

    @staticmethod
    def _nseq(x, offsets):
        return offsets.shape[0] - 1 if offsets is not None else x.shape[0] if x.dim() == 3 else 1

    def _convolution(self, what, x, weight, bias, offsets, nseq, state, silu, out, last):
        code, dtype = _format(x, "x")
        tokens, D = x.shape
        K = weight.shape[-1]
        poff, off_bytes = _offsets(offsets)
        if last is None:
            last = x.new_empty((nseq, K - 1, D))
        elif last is False:
            last = None
        px, ld_x = _row_tensor(x, dtype, "x", tokens, D)
        py, ld_y = _row_tensor(_flat(out), dtype, "out", tokens, D)
        rows = (nseq, K - 1, D)
        rc = self._lib.polyglot_convolution(self._h, ConvolutionArgs.pack(
            px, _block(weight, torch.float32, "weight", (D, K)),
            _vector(bias, torch.float32, "bias", D), _block(state, dtype, "state", rows), poff, py,
            _block(last, dtype, "last", rows), tokens, ld_x, ld_y, nseq, D, K, code, off_bytes,
            silu))
        if rc != OK:
            self._check(rc, what)
        return out, last

    def convolution(self, x, weight, bias=None, offsets=None, *, state=None, silu: bool = True,
                    out=None, last=None):
        """The short causal convolution of every channel, y_t = bias + sum over k of
        weight[:, k] x_{t - taps + 1 + k} (silu: times its sigmoid), over the sequences of x
        as in recurrence.  weight[D][taps] and bias[D] are float32; state and last
        [nseq][taps - 1][D], in x's type, are the inputs before and at the end of each
        sequence; last=False leaves the latter out.  Returns (y, last)."""
        if out is None:
            out = _like(x)
        return self._convolution("convolution", _flat(x), weight, bias, offsets,
                                 self._nseq(x, offsets), state, silu, out, last)

    def convolution_step(self, x, weight, bias=None, state=None, *, silu: bool = True, out=None,
                         last=None):
        """One token x[nseq][D] for each of nseq sequences after the inputs in
        state[nseq][taps - 1][D].  Returns (y, the new states); last=state updates them in
        place."""
        if out is None:
            out = _like(x)
        return self._convolution("convolution_step", x, weight, bias, None, x.shape[0], state,
                                 silu, out, last)

    def convolution_backward(self, x, weight, bias, dy, offsets=None, *, state=None, dlast=None,
                             silu: bool = True, out: ConvolutionGrads | None = None):
        """The gradient of convolution for the gradients dy of y and dlast of last, into the
        tensors of out where it has any.  Returns ConvolutionGrads."""
        code, dtype = _format(x, "x")
        nseq, shape = self._nseq(x, offsets), x.shape
        x = _flat(x)
        tokens, D = x.shape
        K = weight.shape[-1]
        rows = (nseq, K - 1, D)
        dx, dweight, dbias, dstate = out if out is not None else (None,) * 4
        if dx is None:
            dx = x.new_empty(shape)
        if dweight is None:
            dweight = x.new_empty((D, K), dtype=torch.float32)
        if dbias is None and bias is not None:
            dbias = x.new_empty(D, dtype=torch.float32)
        if dstate is None and state is not None:
            dstate = x.new_empty(rows)
        poff, off_bytes = _offsets(offsets)
        px, ld_x = _row_tensor(x, dtype, "x", tokens, D)
        pdy, ld_dy = _row_tensor(_flat(dy), dtype, "dy", tokens, D)
        pdx, ld_dx = _row_tensor(_flat(dx), dtype, "dx", tokens, D)
        rc = self._lib.polyglot_convolution_grad(self._h, ConvolutionGradArgs.pack(
            px, _block(weight, torch.float32, "weight", (D, K)),
            _vector(bias, torch.float32, "bias", D), _block(state, dtype, "state", rows), pdy,
            _block(dlast, dtype, "dlast", rows), poff, pdx,
            _block(dweight, torch.float32, "dweight", (D, K)),
            _vector(dbias, torch.float32, "dbias", D), _block(dstate, dtype, "dstate", rows),
            tokens, ld_x, ld_dy, ld_dx, nseq, D, K, code, off_bytes, silu))
        if rc != OK:
            self._check(rc, "convolution_backward")
        return ConvolutionGrads(dx, dweight, dbias, dstate)

    @staticmethod
    def _selective_inputs(x, delta, A, B, C, z):
        """What a selective scan and its gradient share of their inputs' checks: the shape,
        and the pointers and row distances of x, delta, B, C and z."""
        code, dtype = _format(x, "x")
        tokens, D = x.shape
        N = A.shape[-1]
        if A.dim() != 2 or N < 1:
            raise ValueError(f"A must have shape {(D, 'states')}, got {tuple(A.shape)}")
        GN = B.shape[-1]
        if GN < 1 or GN % N:
            raise ValueError(f"B has {GN} columns, which are not whole heads of {N} states")
        pz = (0, 0) if z is None else _row_tensor(z, dtype, "z", tokens, D)
        return (code, dtype, tokens, D, N, GN // N, _row_tensor(x, dtype, "x", tokens, D),
                _row_tensor(delta, dtype, "delta", tokens, D),
                _row_tensor(B, dtype, "B", tokens, GN), _row_tensor(C, dtype, "C", tokens, GN), pz)

    def _selective(self, what, x, delta, A, B, C, offsets, nseq, state, skip, z, delta_bias,
                   softplus, out, last, marks):
        code, dtype, tokens, D, N, G, px, pd, pb, pc, pz = self._selective_inputs(
            x, delta, A, B, C, z)
        poff, off_bytes = _offsets(offsets)
        shape = (nseq, D, N)
        if last is None:
            last = x.new_empty(shape, dtype=torch.float32)
        elif last is False:
            last = None
        room = (-(-tokens // SELECTIVE_MARK), D, -(-N // 4) * 4)
        if marks is True:
            marks = x.new_empty(room, dtype=torch.float32)
        elif marks is False:
            marks = None
        py = _row_tensor(_flat(out), dtype, "out", tokens, D)
        f32 = torch.float32
        rc = self._lib.polyglot_selective(self._h, SelectiveArgs.pack(
            px[0], pd[0], pb[0], pc[0], pz[0], _block(A, f32, "A", (D, N)),
            _vector(skip, f32, "skip", D), _vector(delta_bias, f32, "delta_bias", D),
            _block(state, f32, "state", shape), poff, py[0], _block(last, f32, "last", shape),
            _block(marks, f32, "marks", room), tokens, px[1], pd[1], pb[1], pc[1], pz[1], py[1],
            nseq, D, N, G, code, off_bytes, softplus))
        if rc != OK:
            self._check(rc, what)
        return out, last, marks

    def selective_scan(self, x, delta, A, B, C, offsets=None, *, state=None, skip=None, z=None,
                       delta_bias=None, softplus: bool = True, out=None, last=None, marks=False):
        """The selective state space scan h_t = e^(s_t A) h_{t-1} + s_t x_t B_t, v_t = C_t h_t
        + skip x_t, y = v or, with z, v z sigmoid(z), with s = softplus(delta + delta_bias)
        (or delta + delta_bias), over the sequences of x as in recurrence.  A[D][states],
        skip[D], delta_bias[D] and the states[nseq][D][states] are float32; B and C have
        states columns, or as many for each of several heads of consecutive channels.
        marks=True keeps what selective_backward needs, last=False leaves the sequences' last
        states out.  Returns (y, last, marks)."""
        if out is None:
            out = _like(x)
        return self._selective("selective_scan", _flat(x), _flat(delta), A, _flat(B), _flat(C),
                               offsets, self._nseq(x, offsets), state, skip, _flat(z), delta_bias,
                               softplus, out, last, marks)

    def selective_step(self, x, delta, A, B, C, state=None, *, skip=None, z=None, delta_bias=None,
                       softplus: bool = True, out=None, last=None):
        """One token x[nseq][D] for each of nseq sequences whose states are
        state[nseq][D][states].  Returns (y, the new states); last=state updates them in
        place."""
        if out is None:
            out = _like(x)
        return self._selective("selective_step", x, delta, A, B, C, None, x.shape[0], state, skip,
                               z, delta_bias, softplus, out, last, None)[:2]

    def selective_backward(self, x, delta, A, B, C, dy, marks, offsets=None, *, state=None,
                           dlast=None, skip=None, z=None, delta_bias=None, softplus: bool = True,
                           out: SelectiveGrads | None = None):
        """The gradient of selective_scan, for its inputs, its marks and the gradients dy of y
        and dlast of last, into the tensors of out where it has any.  Returns SelectiveGrads."""
        nseq = self._nseq(x, offsets)
        given = [None] * 9 if out is None else list(out)
        f32 = torch.float32
        for i, like in enumerate((x, delta, A, B, C, skip, z, delta_bias, state)):
            if given[i] is None and like is not None:
                given[i] = _like(like)
            elif like is None and i in (5, 6, 7):
                given[i] = None
        g = SelectiveGrads(*given)
        code, dtype, tokens, D, N, G, px, pd, pb, pc, pz = self._selective_inputs(
            _flat(x), _flat(delta), A, _flat(B), _flat(C), _flat(z))
        shape = (nseq, D, N)
        poff, off_bytes = _offsets(offsets)
        pdy = _row_tensor(_flat(dy), dtype, "dy", tokens, D)
        gx = _row_tensor(_flat(g.x), dtype, "out.x", tokens, D)
        gd = _row_tensor(_flat(g.delta), dtype, "out.delta", tokens, D)
        gb = _row_tensor(_flat(g.B), dtype, "out.B", tokens, G * N)
        gc = _row_tensor(_flat(g.C), dtype, "out.C", tokens, G * N)
        gz = (0, 0) if z is None else _row_tensor(_flat(g.z), dtype, "out.z", tokens, D)
        rc = self._lib.polyglot_selective_grad(self._h, SelectiveGradArgs.pack(
            px[0], pd[0], pb[0], pc[0], pz[0], pdy[0], _block(A, f32, "A", (D, N)),
            _vector(skip, f32, "skip", D), _vector(delta_bias, f32, "delta_bias", D),
            _block(state, f32, "state", shape), _block(dlast, f32, "dlast", shape),
            _block(marks, f32, "marks", (-(-tokens // SELECTIVE_MARK), D, -(-N // 4) * 4)), poff,
            gx[0], gd[0], gb[0], gc[0], gz[0], _block(g.A, f32, "out.A", (D, N)),
            _vector(g.skip, f32, "out.skip", D), _vector(g.delta_bias, f32, "out.delta_bias", D),
            _block(g.state, f32, "out.state", shape), tokens, px[1], pd[1], pb[1], pc[1], pz[1],
            pdy[1], gx[1], gd[1], gb[1], gc[1], gz[1], nseq, D, N, G, code, off_bytes, softplus))
        if rc != OK:
            self._check(rc, "selective_backward")
        return g

    def beam(self, scores, total, *, beams: int, picks: int, lse=None, finished=None, end: int = 0,
             out=None):
        """For every group of `beams` rows of scores[rows][V], the `picks` largest of
        scores[r][v] + (total[r] - lse[r]) over its rows and words, of equal ones the first;
        a row whose finished (int32) is set offers the word `end` with total[r] alone.
        out: (parent, token, total) to write to.  Returns them, [groups][picks]: the picks'
        rows of scores (int32, what reorder takes), words (int32, -1 where nothing is left) and
        sums (float32)."""
        code, dtype = _format(scores, "scores")
        if scores.dim() != 2:
            raise ValueError("scores must have two dimensions")
        rows, V = scores.shape
        if beams < 1 or rows % beams:
            raise ValueError(f"{rows} rows are not whole groups of {beams} beams")
        shape = (rows // beams, picks)
        ps, ld = _row_tensor(scores, dtype, "scores", rows, V)
        if out is None:
            out = (scores.new_empty(shape, dtype=torch.int32),
                   scores.new_empty(shape, dtype=torch.int32),
                   scores.new_empty(shape, dtype=torch.float32))
        rc = self._lib.polyglot_beam(self._h, BeamArgs.pack(
            ps, _vector(total, torch.float32, "total", rows),
            _vector(lse, torch.float32, "lse", rows),
            _vector(finished, torch.int32, "finished", rows),
            _block(out[0], torch.int32, "out[0]", shape),
            _block(out[1], torch.int32, "out[1]", shape),
            _block(out[2], torch.float32, "out[2]", shape), ld, shape[0], beams, V, picks, end,
            code))
        if rc != OK:
            self._check(rc, "beam")
        return out

    def reorder(self, tensors, ids, outs=None):
        """[t[ids] for t in tensors], all of them in one launch, bytes as they are: rows of
        any shape and type, contiguous within a row; ids int32, of any shape.  outs: tensors
        to write to, none of which may overlap an input.  Returns the list."""
        rows = ids.numel()
        pid = _vector(ids if ids.dim() == 1 else ids.view(-1), torch.int32, "ids", rows)
        if outs is None:
            outs = [torch.empty_like(t) if t.shape[:1] == (rows,) and t.is_contiguous()
                    else t.new_empty((rows, *t.shape[1:])) for t in tensors]
        else:
            if len(outs) != len(tensors):
                raise ValueError(f"{len(tensors)} tensors, {len(outs)} outputs")
            for t, o in zip(tensors, outs):
                if not o.is_cuda or t.dtype is not o.dtype or o.shape != (rows, *t.shape[1:]):
                    raise ValueError(f"an output of {(rows, *t.shape[1:])} {t.dtype} on the device "
                                     f"is needed, got {tuple(o.shape)} {o.dtype}")
        items = []
        for t, o in zip(tensors, outs):
            if not t.is_cuda or t.dim() < 1:
                raise ValueError("tensors must be device (cuda) tensors of rows")
            have = t.shape[0]
            if not have:
                if rows:
                    raise ValueError("a tensor without rows has none to give")
                continue
            if t.is_contiguous():
                width = ld_t = t.nbytes // have
            else:
                width = t[0].nbytes
                ld_t = t.stride(0) * t.element_size() if have > 1 else width
                if not t[0].is_contiguous():
                    raise ValueError("rows must be contiguous")
            ld_o = width
            if not o.is_contiguous():
                if rows and not o[0].is_contiguous():
                    raise ValueError("rows must be contiguous")
                ld_o = o.stride(0) * o.element_size() if rows > 1 else width
            items.append(RowCopy.pack(t.data_ptr(), o.data_ptr(), width, ld_t, ld_o, have, 0))
        rc = self._lib.polyglot_reorder(self._h, b"".join(items), len(items), pid, rows)
        if rc != OK:
            self._check(rc, "reorder")
        return outs

    def operator_times(self) -> dict:
        """kernel_times for the sequence operators: {operator: (total ms, launches)}."""
        ms = (ctypes.c_double * len(OPERATOR_NAMES))()
        n = (ctypes.c_int32 * len(OPERATOR_NAMES))()
        self._check(self._lib.polyglot_operator_times(self._h, ms, n), "operator_times")
        return {name: (ms[i], n[i]) for i, name in enumerate(OPERATOR_NAMES)}

    def status(self) -> int:
        """Synchronises; returns OK, EID or EOFFSETS (the sticky device flag), clearing it."""
        return self._lib.polyglot_status(self._h)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.polyglot_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
