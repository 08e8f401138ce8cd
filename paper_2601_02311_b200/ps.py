"""Python binding of the CUDA library (``libps_b200.so``): argument marshalling
only.  Every step of the evaluation runs in the library's kernels; torch is
used for device memory and streams.  Importing this module fails if the library
has not been built (``python -m paper_2601_02311_b200.build``) -- there is no
CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libps_b200.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build the CUDA library first "
        "(python -m paper_2601_02311_b200.build); there is no CPU fallback")
_lib = C.CDLL(LIB_PATH)

# ---- constants of ps.h
OK = 0
E_NULLPTR, E_ALIGN, E_RANGE, E_BADINDEX, E_TRUNCATED, E_CUDA, E_UNIMPLEMENTED, E_DEVICE = \
    -1, -2, -3, -4, -5, -6, -7, -8
E_NOALLOC_LIMIT = -10
NOALLOC_MAX_GROUPS = 131072
F_GI, F_SC, F_CV, F_FEASIBLE = 1, 2, 4, 8
F_T_DIV_HEADS, F_K_DIV_LAYERS, F_TP_LE_MAX, F_AXIS_FORM = 16, 32, 64, 128
F_THETA_AVAIL, F_ACT_AVAIL, F_GRAD_COVER, F_USES_HOST, F_PAPER_PRICED = 256, 512, 1024, 2048, 4096
F_VALID = F_GI | F_SC | F_CV
COMM_PAPER, COMM_PAPER_PLUS_EXT = 0, 1
REDUCE_PARETO, REDUCE_TOPK = 0, 1
NO_LIMIT = (1 << 64) - 1
TOPK_MAX = 64
# A result up to this size is read back through pinned memory: a sweep's of 1.6 MB comes in 101 us instead of 200
# through pageable memory, one of 4 MB in 160 instead of 363.  Inputs up to this size go up through it as well.
PINNED_RESULT_BYTES = 4 << 20

SELECT_QUERY_DTYPE = np.dtype([("param_elems", "<u8"), ("layer_elems", "<u8"), ("device_bytes", "<u8"),
                               ("n_devices", "<u4"), ("w_param", "u1"), ("w_grad", "u1"), ("w_opt", "u1"),
                               ("fast_interconnect", "u1")])
SELECT_RESULT_DTYPE = np.dtype([("mem", "<u8"), ("comm", "<u8"), ("branch", "<u4"), ("T", "<u4"),
                                ("code_dp", "<u4"), ("flags", "<u4")])
ENTRY_DTYPE = np.dtype([("mem", "<u8"), ("comm", "<u8"), ("host", "<u8"), ("idx", "<u8"),
                        ("flags", "<u4"), ("pad", "<u4")])

EXPORTS = ("ps_create", "ps_destroy", "ps_status", "ps_strerror", "ps_space_create",
           "ps_space_destroy", "ps_space_set_models", "ps_space_rederive", "ps_space_size",
           "ps_space_points_per_model", "ps_space_decode", "ps_eval_batch", "ps_sweep_pareto",
           "ps_check_composition", "ps_int_peak", "ps_eval_compact_noalloc", "ps_select",
           "ps_verify_batch", "ps_select_compare", "ps_dropout", "ps_embed_forward", "ps_embed_backward_bytes",
           "ps_embed_backward", "ps_attention_forward", "ps_attention_forward_bytes", "ps_attention_backward_bytes", "ps_attention_backward",
           "ps_layer_norm_forward", "ps_layer_norm_backward_bytes", "ps_layer_norm_backward", "ps_rotary", "ps_linear_forward",
           "ps_linear_backward_bytes", "ps_linear_backward")


class _SpaceDesc(C.Structure):
    _fields_ = [("models", C.c_void_p), ("n_models", C.c_uint32),
                ("n_values", C.c_void_p), ("n_n", C.c_uint32),
                ("t_enum_max", C.c_uint32), ("k_enum_max", C.c_uint32),
                ("tp_max_valid", C.c_uint32), ("n_act_variants", C.c_uint32),
                ("n_tpa_variants", C.c_uint32), ("mode_mask", C.c_uint32),
                ("tp_coll_per_layer", C.c_uint32), ("sstar_units", C.c_uint32),
                ("grad_accum_steps", C.c_uint32), ("replication_k", C.c_uint32)]


class _Filter(C.Structure):
    _fields_ = [("host_cap", C.c_uint64), ("require_flags", C.c_uint32),
                ("comm_kind", C.c_uint32), ("cap_bytes", C.c_uint64),
                ("skip_rejected", C.c_uint32), ("pad", C.c_uint32)]


class _OutSoa(C.Structure):
    _fields_ = [("mem", C.c_void_p), ("comm_paper", C.c_void_p), ("comm_ext", C.c_void_p),
                ("host", C.c_void_p), ("flags", C.c_void_p)]


class _VerifyShape(C.Structure):
    _fields_ = [("units", C.c_uint32), ("h", C.c_uint32), ("b", C.c_uint32), ("accum", C.c_uint32),
                ("steps", C.c_uint32), ("gather_buffers", C.c_uint32), ("w_theta", C.c_uint32),
                ("w_omega", C.c_uint32), ("w_grad", C.c_uint32), ("pad", C.c_uint32),
                ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("rtol", C.c_double), ("atol", C.c_double)]


SELECT_COMPARE_DTYPE = np.dtype([("alg_mem", "<u8"), ("alg_comm", "<u8"), ("alg_idx", "<u8"), ("best_mem", "<u8"),
                                 ("best_comm", "<u8"), ("best_idx", "<u8"), ("branch", "<u4"), ("T", "<u4"),
                                 ("code_dp", "<u4"), ("alg_flags", "<u4"), ("status", "<u4"), ("pad", "<u4")])
SEL_IN_SPACE, SEL_SURVIVOR, SEL_ON_FRONTIER, SEL_DOMINATED, SEL_FRONTIER_EMPTY, SEL_FRONTIER_TRUNCATED = \
    1, 2, 4, 8, 16, 32
VERIFY_CASE_DTYPE = np.dtype([("code", "<u4"), ("D", "<u4"), ("data_offset", "<u8")])
VERIFY_RESULT_DTYPE = np.dtype([("mem", "<u8"), ("comm", "<u8"), ("host", "<u8"), ("match", "<u4"),
                                ("pad", "<u4"), ("max_rel_err", "<f8")])


# The training step's descriptors (ps_dropout_desc, ps_embed_desc, ps_heads, ps_attention_shape, ...) as bytes: a ctypes
# Structure of as many fields takes a call several microseconds longer.
_DROPOUT_DESC = struct.Struct("9QdII").pack
_EMBED_DESC = struct.Struct("6Qd4I").pack
_HEADS = struct.Struct("4Q").pack
_ATTENTION_SHAPE = struct.Struct("8IfI").pack
_MATRIX = struct.Struct("2Q").pack
_LAYER_NORM_DESC = struct.Struct("2Qd4I").pack
_ROTARY_DESC = struct.Struct("10IQq6d").pack
_LINEAR_DESC = struct.Struct("3Q6I").pack
ACTIVATIONS = {"none": 0, None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}   # PS_ACT_*
_FLOAT_MOST = torch.finfo(torch.float32).max
_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # PS_F32, PS_BF16, PS_F16


class _Point(C.Structure):
    _fields_ = [("model", C.c_uint32), ("N", C.c_uint32), ("T", C.c_uint32), ("K", C.c_uint32),
                ("D", C.c_uint32), ("act_variant", C.c_uint32), ("tpa_variant", C.c_uint32),
                ("code_dp", C.c_uint16), ("code_tp", C.c_uint16), ("code_pp", C.c_uint16),
                ("pad", C.c_uint16)]


_lib.ps_strerror.restype = C.c_char_p
_lib.ps_strerror.argtypes = [C.c_int]
_lib.ps_create.argtypes = [C.POINTER(C.c_void_p), C.c_int, C.c_void_p]
_lib.ps_destroy.argtypes = [C.c_void_p]
_lib.ps_destroy.restype = None
_lib.ps_status.argtypes = [C.c_void_p]
_lib.ps_space_create.argtypes = [C.c_void_p, C.POINTER(_SpaceDesc), C.POINTER(C.c_void_p)]
_lib.ps_space_destroy.argtypes = [C.c_void_p]
_lib.ps_space_destroy.restype = None
_lib.ps_space_set_models.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32]
_lib.ps_space_rederive.argtypes = [C.c_void_p]
_lib.ps_space_size.argtypes = [C.c_void_p]
_lib.ps_space_size.restype = C.c_uint64
_lib.ps_space_points_per_model.argtypes = [C.c_void_p]
_lib.ps_space_points_per_model.restype = C.c_uint64
_lib.ps_space_decode.argtypes = [C.c_void_p, C.c_uint64, C.POINTER(_Point)]
_lib.ps_eval_batch.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_uint64, C.POINTER(_Filter),
                               _OutSoa, C.c_void_p, C.c_void_p]
_lib.ps_eval_compact_noalloc.argtypes = _lib.ps_eval_batch.argtypes
_lib.ps_sweep_pareto.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(_Filter), C.c_void_p,
                                 C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p]
_lib.ps_check_composition.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint32, C.c_uint32,
                                      C.c_uint32, C.c_uint16, C.c_uint16, C.c_uint16, C.c_uint32,
                                      C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p]
_lib.ps_select.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32,
                           C.c_uint32, C.c_uint32, C.c_void_p]
_lib.ps_select_compare.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32,
                                   C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint32, C.POINTER(_Filter), C.c_void_p,
                                   C.c_void_p, C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p]
_lib.ps_verify_batch.argtypes = [C.c_void_p, C.POINTER(_VerifyShape), C.c_void_p, C.c_uint64, C.c_void_p,
                                 C.c_uint64, C.c_void_p, C.c_void_p]
_lib.ps_dropout.argtypes = [C.c_void_p] * 5
_lib.ps_embed_forward.argtypes = [C.c_void_p] * 5
_lib.ps_embed_backward_bytes.argtypes = [C.c_void_p]
_lib.ps_embed_backward_bytes.restype = C.c_uint64
_lib.ps_embed_backward.argtypes = [C.c_void_p] * 6 + [C.c_uint64]
_lib.ps_attention_forward.argtypes = [C.c_void_p] * 10 + [C.c_uint64]
_lib.ps_attention_forward_bytes.argtypes = [C.c_void_p]
_lib.ps_attention_forward_bytes.restype = C.c_uint64
_lib.ps_attention_backward_bytes.argtypes = [C.c_void_p]
_lib.ps_attention_backward_bytes.restype = C.c_uint64
_lib.ps_attention_backward.argtypes = [C.c_void_p] * 14 + [C.c_uint64]
_lib.ps_layer_norm_forward.argtypes = [C.c_void_p] * 8
_lib.ps_layer_norm_backward_bytes.argtypes = [C.c_void_p]
_lib.ps_layer_norm_backward_bytes.restype = C.c_uint64
_lib.ps_layer_norm_backward.argtypes = [C.c_void_p] * 12 + [C.c_uint64]
_lib.ps_rotary.argtypes = [C.c_void_p] * 7
_lib.ps_linear_forward.argtypes = [C.c_void_p] * 8
_lib.ps_linear_backward_bytes.argtypes = [C.c_void_p]
_lib.ps_linear_backward_bytes.restype = C.c_uint64
_lib.ps_linear_backward.argtypes = [C.c_void_p] * 12 + [C.c_uint64]
_lib.ps_int_peak.argtypes = [C.c_void_p, C.c_uint32, C.c_uint32, C.c_void_p,
                             C.POINTER(C.c_uint64)]


class PsError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_lib.ps_strerror(code).decode()} ({code})")


def _check(code: int, where: str):
    if code != OK:
        raise PsError(code, where)


def strerror(code: int) -> str:
    return _lib.ps_strerror(code).decode()


def _mk_filter(filt: dict) -> _Filter:
    return _Filter(filt.get("host_cap", NO_LIMIT), filt.get("require_flags", 0),
                   filt.get("comm_kind", COMM_PAPER_PLUS_EXT), filt.get("cap_bytes", NO_LIMIT),
                   1 if filt.get("skip_rejected") else 0, 0)


def _dptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _on_own_stream(method):
    """For methods that allocate: their tensors come into being, and are filled and read back, on the
    stream that the library enqueues on.  On torch's current stream, where that is another one, a
    buffer's zeros could land after the kernel's results, or a kernel write to memory that work
    before it still uses."""
    @functools.wraps(method)
    def run(self, *args, **kwargs):
        ctx = self if isinstance(self, Context) else self.ctx
        if torch._C._cuda_getCurrentRawStream(ctx.device) == ctx._raw_stream:      # (ctx.on_current_stream)
            return method(self, *args, **kwargs)
        with torch.cuda.stream(ctx.stream if ctx.stream is not None else torch.cuda.default_stream(ctx.device)):
            return method(self, *args, **kwargs)
    return run


class Context:
    """ps_ctx: one per (device, stream); without a stream it enqueues on the device's default stream."""

    def __init__(self, device: int = 0, stream: torch.cuda.Stream | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("the placement-semantics library needs a CUDA device")
        self.device = device
        self.torch_device = torch.device("cuda", device)
        self.stream = stream
        self._raw_stream = stream.cuda_stream if stream is not None else 0
        handle = C.c_void_p()
        sptr = C.c_void_p(stream.cuda_stream) if stream is not None else None
        _check(_lib.ps_create(C.byref(handle), device, sptr), "ps_create")
        self._h = handle

    def close(self):
        # at interpreter shutdown the module's globals may be gone before the last
        # handle: the process is ending, the driver releases the device memory
        if getattr(self, "_h", None) and _lib is not None:
            _lib.ps_destroy(self._h)
        self._h = None

    __del__ = close

    def on_current_stream(self) -> bool:
        """Whether torch's current stream on the device is the one the library enqueues on."""
        # (asked before every call that allocates: a Stream object made for it costs a sweep of 60 us 2 us)
        return torch._C._cuda_getCurrentRawStream(self.device) == self._raw_stream

    def status(self) -> int:
        return _lib.ps_status(self._h)

    def check_status(self, allow_truncated: bool = False) -> int:
        """Synchronise and raise on any error a kernel reported.  With
        ``allow_truncated`` the notice that a frontier was longer than the caller's
        rows (E_TRUNCATED: heads written, counts true) is returned instead of raised."""
        rc = self.status()
        if not (allow_truncated and rc == E_TRUNCATED):
            _check(rc, "ps_status")
        return rc

    def space(self, space: dict) -> "Space":
        return Space(self, space)

    def check_composition(self, shape: np.ndarray, N, T, K, D, code_tp, code_pp, code_dp,
                          act_variant=0, cap_bytes=NO_LIMIT, tp_max_valid=8, tp_coll_per_layer=4,
                          comm_kind=COMM_PAPER_PLUS_EXT) -> dict:
        shape = np.ascontiguousarray(shape)
        out = np.zeros(1, dtype=ENTRY_DTYPE)
        _check(_lib.ps_check_composition(self._h, shape.ctypes.data, N, T, K, D, code_tp, code_pp,
                                         code_dp, act_variant, cap_bytes, tp_max_valid,
                                         tp_coll_per_layer, comm_kind, out.ctypes.data),
               "ps_check_composition")
        return {k: int(out[0][k]) for k in ("mem", "comm", "host", "flags")}

    def select_into(self, d_queries: torch.Tensor, n: int, d_out: torch.Tensor, headroom=(7, 10),
                    layer=(3, 10), tp_degree=8):
        """ps_select on device buffers (uint8 tensors of 32-byte records)."""
        _check(_lib.ps_select(self._h, _dptr(d_queries), n, headroom[0], headroom[1], layer[0], layer[1],
                              tp_degree, _dptr(d_out)), "ps_select")

    @_on_own_stream
    def select(self, queries: np.ndarray, headroom=(7, 10), layer=(3, 10), tp_degree=8) -> np.ndarray:
        """Algorithm 1 for a structured array of SELECT_QUERY_DTYPE; returns SELECT_RESULT_DTYPE."""
        q = np.ascontiguousarray(queries)
        assert q.dtype.itemsize == 32
        d_q = torch.from_numpy(q.view(np.uint8).reshape(-1).copy()).to(self.torch_device)
        d_o = torch.empty(max(len(q), 1) * 32, dtype=torch.uint8, device=self.torch_device)
        self.select_into(d_q, len(q), d_o, headroom, layer, tp_degree)
        self.check_status()
        return d_o.cpu().numpy()[:len(q) * 32].view(SELECT_RESULT_DTYPE)

    @_on_own_stream
    def verify_batch(self, shape: dict, cases: np.ndarray, data: np.ndarray, want_theta: bool = False):
        """ps_verify_batch: `cases` a VERIFY_CASE_DTYPE array, `data` a float64 array holding every
        case's problem; returns VERIFY_RESULT_DTYPE records (and the final parameters).  Both are views of
        one buffer; up to PINNED_RESULT_BYTES it is page-locked for as long as either is kept."""
        sh = _VerifyShape(shape["units"], shape["h"], shape["b"], shape.get("accum", 1), shape.get("steps", 3),
                          shape.get("gather_buffers", 1), shape.get("w_theta", 2), shape.get("w_omega", 12),
                          shape.get("w_grad", 2), 0, shape.get("lr", 0.05), shape.get("beta1", 0.9),
                          shape.get("beta2", 0.999), shape.get("eps", 1e-8), shape.get("rtol", 1e-12),
                          shape.get("atol", 1e-14))
        cases = np.ascontiguousarray(cases)
        assert cases.dtype.itemsize == 16
        data = np.ascontiguousarray(data, dtype=np.float64)
        n = len(cases)
        P = shape["units"] * shape["h"]
        # The cases and their problems go up together, the parameters and records come back together.  (More inputs
        # than the limit go up as they are: another copy of 13.5 MB for it took 2.2 ms a call instead of 1.5.)
        size = cases.nbytes + data.nbytes
        if 0 < size <= PINNED_RESULT_BYTES:
            up = torch.empty(size, dtype=torch.uint8, pin_memory=True)
            up.numpy()[:cases.nbytes] = cases.view(np.uint8).reshape(-1)
            up.numpy()[cases.nbytes:] = data.view(np.uint8).reshape(-1)
            d_in = up.to(self.torch_device, non_blocking=True)
        else:
            d_in = torch.empty(size, dtype=torch.uint8, device=self.torch_device)
            for at, part in ((0, cases), (cases.nbytes, data)):
                part = part.view(np.uint8).reshape(-1)
                d_in[at:at + len(part)].copy_(torch.from_numpy(part if part.flags.writeable else part.copy()))
        at = n * P * 8 if want_theta else 0
        d_all = torch.empty(max(at + n * 40, 1), dtype=torch.uint8, device=self.torch_device)
        into, base = d_in.data_ptr(), d_all.data_ptr()
        _check(_lib.ps_verify_batch(self._h, C.byref(sh), into, n, into + cases.nbytes if len(data) else None, len(data),
                                    base + at, base if want_theta else None), "ps_verify_batch")
        host, _ = self._read_back(d_all)
        res = host[at:at + n * 40].view(VERIFY_RESULT_DTYPE)
        if want_theta:
            return res, host[:at].view(np.float64).reshape(n, P)
        return res

    def _read_back(self, d_all: torch.Tensor, allow_truncated: bool = False):
        """A uint8 buffer's bytes on the host once the work before has been done and found in order,
        and check_status's answer.  A small buffer is copied behind that work through pinned memory,
        and one wait covers both."""
        if d_all.numel() <= PINNED_RESULT_BYTES:
            host = torch.empty(d_all.numel(), dtype=torch.uint8, pin_memory=True)
            host.copy_(d_all, non_blocking=True)
            return host.numpy(), self.check_status(allow_truncated)
        status = self.check_status(allow_truncated)
        return d_all.cpu().numpy(), status

    # ---- operators of a training step.  Tensors live on the context's device, and a call takes its place in the order of
    # torch's current stream, as one of torch's own would: its tensors may come from there and its results be used there at
    # once, and they and its work buffer are allocated there.  The library sees sizes and strides, so what it cannot see is
    # refused here, with its codes: another device, another type, a shape that does not match.

    def _enqueue(self, where: str, call, *args):
        """The library's call, on the context's stream.  Where that is not torch's current one, it waits for what the current one
        has been given so far, and the current one for the call (8 us on the host; contexts whose calls are to
        overlap are used with their own streams current).  So memory that torch gives out again there is not in use
        any more, and a capture of the current stream takes the call in."""
        if torch._C._cuda_getCurrentRawStream(self.device) == self._raw_stream:
            return _check(call(self._h, *args), where)
        current = torch.cuda.current_stream(self.device)
        own = self.stream if self.stream is not None else torch.cuda.default_stream(self.device)
        own.wait_stream(current)
        try:
            _check(call(self._h, *args), where)
        finally:
            current.wait_stream(own)

    def _refuse(self, code: int, where: str, what: str):
        raise PsError(code, f"{where}: {what}")

    def _row_stride(self, t: torch.Tensor, where: str, name: str, shape, dtype) -> int:
        """Elements between the rows of [rows, cols] whose columns are contiguous."""
        if t.shape != shape or t.dtype != dtype or dtype not in _DTYPE or len(shape) != 2 or t.get_device() != self.device:
            self._refuse(E_RANGE, where, f"{name} is {t.dtype} of {tuple(t.shape)} on {t.device}, wanted {dtype} of two "
                         f"dimensions {tuple(shape)} on device {self.device}")
        rows, cols = shape
        stride = t.stride()
        if cols > 1 and stride[1] != 1:
            self._refuse(E_ALIGN, where, f"{name}'s columns are not contiguous")
        return stride[0] if rows > 1 else max(cols, 1)

    def _tokens(self, t: torch.Tensor, where: str) -> int:
        """Bytes of a token."""
        if t.dim() != 1 or t.dtype not in (torch.int64, torch.int32) or t.get_device() != self.device:
            self._refuse(E_RANGE, where, f"tokens have to be a row of int32 or int64 on device {self.device}")
        if not t.is_contiguous():
            self._refuse(E_ALIGN, where, "tokens are not contiguous")
        return t.element_size()

    def _work(self, work: torch.Tensor | None, need: int, where: str) -> torch.Tensor:
        if work is None:                # (freed when the call returns: torch gives it out again on the current stream only)
            return torch.empty(max(need, 1), dtype=torch.uint8, device=self.torch_device)
        if work.get_device() != self.device or work.dtype != torch.uint8 or not work.is_contiguous():
            self._refuse(E_RANGE, where, f"work has to be a contiguous uint8 tensor on device {self.device}")
        return work

    def dropout_into(self, x: torch.Tensor, y: torch.Tensor, p: float, seed: int, stream: int = 0,
                     residual: torch.Tensor | None = None, first: int = 0, pitch: int | None = None):
        """ps_dropout on [rows, cols]; `pitch` is the rows' length in the whole tensor (default cols)."""
        where, shape, dtype = "ps_dropout", x.shape, x.dtype
        x_stride = self._row_stride(x, where, "x", shape, dtype)
        y_stride = self._row_stride(y, where, "y", shape, dtype)
        r_stride = 0 if residual is None else self._row_stride(residual, where, "residual", shape, dtype)
        rows, cols = shape
        if pitch is None:
            pitch = cols
        if not (0 <= seed < 1 << 64 and 0 <= stream < 1 << 64 and 0 <= first < 1 << 63 and 0 <= pitch < 1 << 63):
            self._refuse(E_RANGE, where, "seed, stream, first or pitch")
        self._enqueue(where, _lib.ps_dropout,
                      _DROPOUT_DESC(rows, cols, x_stride, r_stride, y_stride, seed, stream, first, pitch, p, _DTYPE[dtype], 0),
                      x.data_ptr(), None if residual is None else residual.data_ptr(), y.data_ptr())

    def dropout(self, x: torch.Tensor, p: float, seed: int, stream: int = 0, residual: torch.Tensor | None = None,
                first: int = 0, pitch: int | None = None) -> torch.Tensor:
        """x with a share p of its elements dropped and the others divided by 1 - p, plus `residual`.
        The gradient of x is the same call on the result's gradient, without a residual."""
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        self.dropout_into(x, y, p, seed, stream, residual, first, pitch)
        return y

    def embed_forward_into(self, table: torch.Tensor, tokens: torch.Tensor, out: torch.Tensor, scale: float = 1.0,
                           first_row: int = 0):
        """ps_embed_forward: out[t] = scale * table[tokens[t] - first_row], zeros where that row is not held."""
        where, shape, dtype = "ps_embed_forward", table.shape, table.dtype
        width, n = self._tokens(tokens, where), tokens.shape[0]
        t_stride = self._row_stride(table, where, "table", shape, dtype)
        o_stride = self._row_stride(out, where, "out", (n, shape[1]), dtype)
        if not 0 <= first_row < 1 << 62:
            self._refuse(E_RANGE, where, "first_row")
        code = _DTYPE[dtype]
        self._enqueue(where, _lib.ps_embed_forward,
                      _EMBED_DESC(n, first_row, shape[0], shape[1], t_stride, o_stride, scale, code, code, width, 0),
                      table.data_ptr(), tokens.data_ptr(), out.data_ptr())

    def embed_forward(self, table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, first_row: int = 0) -> torch.Tensor:
        """The scaled rows [tokens, dim] of the table that the tokens name."""
        out = table.new_empty((tokens.numel(), table.shape[-1]))
        self.embed_forward_into(table, tokens, out, scale, first_row)
        return out

    def embed_backward_into(self, d_out: torch.Tensor, tokens: torch.Tensor, d_table: torch.Tensor, scale: float = 1.0,
                            first_row: int = 0, accumulate: bool = False, work: torch.Tensor | None = None):
        """ps_embed_backward: the gradient of the table, written to or (accumulate) added to d_table.
        `work`: a uint8 buffer of embed_backward_bytes; without it one is allocated for the call."""
        where, shape = "ps_embed_backward", d_table.shape
        width, n = self._tokens(tokens, where), tokens.shape[0]
        g_stride = self._row_stride(d_table, where, "d_table", shape, d_table.dtype)
        o_stride = self._row_stride(d_out, where, "d_out", (n, shape[1]), d_out.dtype)
        if not 0 <= first_row < 1 << 62:
            self._refuse(E_RANGE, where, "first_row")
        desc = _EMBED_DESC(n, first_row, shape[0], shape[1], g_stride, o_stride, scale, _DTYPE[d_out.dtype],
                           _DTYPE[d_table.dtype], width, 1 if accumulate else 0)
        work = self._work(work, _lib.ps_embed_backward_bytes(desc), where)
        self._enqueue(where, _lib.ps_embed_backward, desc, d_out.data_ptr(), tokens.data_ptr(), d_table.data_ptr(), work.data_ptr(),
                      work.numel())

    def embed_backward(self, d_out: torch.Tensor, tokens: torch.Tensor, rows: int, scale: float = 1.0, first_row: int = 0,
                       dtype: torch.dtype | None = None) -> torch.Tensor:
        """The gradient [rows, dim] of the table, in d_out's type or `dtype`."""
        d_table = d_out.new_empty((rows, d_out.shape[-1]), dtype=dtype)
        self.embed_backward_into(d_out, tokens, d_table, scale, first_row)
        return d_table

    @staticmethod
    def embed_backward_bytes(tokens: int, rows: int, dim: int) -> int:
        """Bytes of the work buffer that embed_backward_into takes."""
        return _lib.ps_embed_backward_bytes(_EMBED_DESC(tokens, 0, rows, dim, dim, dim, 1.0, 0, 0, 8, 0))

    def _heads(self, t: torch.Tensor, where: str, name: str, shape, dtype) -> bytes:
        if t.shape != shape or t.dtype != dtype or t.get_device() != self.device:
            self._refuse(E_RANGE, where, f"{name} is {t.dtype} of {tuple(t.shape)} on {t.device}, wanted {dtype} of "
                         f"{tuple(shape)} on device {self.device}")
        b, n, h, d = t.stride()
        if d != 1 and shape[3] > 1:
            self._refuse(E_ALIGN, where, f"{name}'s last dimension is not contiguous")
        return _HEADS(t.data_ptr(), b, n, h)

    def _attention(self, q, k, where, scale, causal, q_lens, k_lens, lse):
        """The shape's bytes, the shape of q and of k, and the lengths' pointers."""
        if q.dim() != 4 or k.dim() != 4 or q.dtype not in _DTYPE:
            self._refuse(E_RANGE, where, "q and k are [batch, len, heads, dim] of a 16-bit type")
        queries, (_, k_len, kv_heads, _) = q.shape, k.shape
        batch, q_len, heads, dim = queries
        for name, lens in (("q_lens", q_lens), ("k_lens", k_lens)):
            if lens is not None and (lens.dtype != torch.int32 or lens.shape != (batch,) or lens.get_device() != self.device
                                     or not lens.is_contiguous()):
                self._refuse(E_RANGE, where, f"{name} has to be {batch} contiguous int32 on device {self.device}")
        if lse.dtype != torch.float32 or lse.shape != (batch, heads, q_len) or lse.get_device() != self.device \
                or not lse.is_contiguous():
            self._refuse(E_RANGE, where, f"lse has to be contiguous float32 [batch, heads, q_len] on device {self.device}")
        if scale is not None and not -_FLOAT_MOST <= scale <= _FLOAT_MOST:
            self._refuse(E_RANGE, where, "scale")
        shape = _ATTENTION_SHAPE(batch, q_len, k_len, heads, kv_heads, dim, _DTYPE[q.dtype], 1 if causal else 0,
                                 (dim or 1) ** -0.5 if scale is None else scale, 0)
        return (shape, queries, (batch, k_len, kv_heads, dim), None if q_lens is None else q_lens.data_ptr(),
                None if k_lens is None else k_lens.data_ptr())

    def attention_forward_into(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                               scale: float | None = None, causal: bool = True, q_lens: torch.Tensor | None = None,
                               k_lens: torch.Tensor | None = None, work: torch.Tensor | None = None):
        """ps_attention_forward on [batch, len, heads, dim] of any strides; scale defaults to dim ** -0.5.
        `work`: a uint8 buffer of attention_forward_bytes; without it one is allocated for a call that needs it."""
        where, dtype = "ps_attention_forward", q.dtype
        shape, qs, ks, ql, kl = self._attention(q, k, where, scale, causal, q_lens, k_lens, lse)
        at, size = None, 0
        need = _lib.ps_attention_forward_bytes(shape)
        if need or work is not None:
            work = self._work(work, need, where)
            at, size = work.data_ptr(), work.numel()
        self._enqueue(
            where, _lib.ps_attention_forward, shape, self._heads(q, where, "q", qs, dtype), self._heads(k, where, "k", ks, dtype),
            self._heads(v, where, "v", ks, dtype), self._heads(out, where, "out", qs, dtype), lse.data_ptr(), ql, kl, at, size)

    def attention_forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float | None = None,
                          causal: bool = True, q_lens: torch.Tensor | None = None, k_lens: torch.Tensor | None = None):
        """(out [batch, q_len, heads, dim], lse [batch, heads, q_len])."""
        if q.dim() != 4:
            self._refuse(E_RANGE, "ps_attention_forward", "q has to be [batch, len, heads, dim]")
        shape = q.shape
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = q.new_empty((shape[0], shape[2], shape[1]), dtype=torch.float32)
        self.attention_forward_into(q, k, v, out, lse, scale, causal, q_lens, k_lens)
        return out, lse

    def attention_backward_into(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                                d_out: torch.Tensor, d_q: torch.Tensor, d_k: torch.Tensor, d_v: torch.Tensor,
                                scale: float | None = None, causal: bool = True, q_lens: torch.Tensor | None = None,
                                k_lens: torch.Tensor | None = None, work: torch.Tensor | None = None):
        """ps_attention_backward: gradients of q, k and v from what the forward pass took and gave.
        `work`: a uint8 buffer of attention_backward_bytes; without it one is allocated for the call."""
        where, dtype = "ps_attention_backward", q.dtype
        shape, qs, ks, ql, kl = self._attention(q, k, where, scale, causal, q_lens, k_lens, lse)
        work = self._work(work, _lib.ps_attention_backward_bytes(shape), where)
        self._enqueue(
            where, _lib.ps_attention_backward, shape, self._heads(q, where, "q", qs, dtype), self._heads(k, where, "k", ks, dtype),
            self._heads(v, where, "v", ks, dtype), self._heads(out, where, "out", qs, dtype), lse.data_ptr(),
            self._heads(d_out, where, "d_out", qs, dtype), self._heads(d_q, where, "d_q", qs, dtype),
            self._heads(d_k, where, "d_k", ks, dtype), self._heads(d_v, where, "d_v", ks, dtype), ql, kl, work.data_ptr(),
            work.numel())

    def attention_backward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                           d_out: torch.Tensor, scale: float | None = None, causal: bool = True,
                           q_lens: torch.Tensor | None = None, k_lens: torch.Tensor | None = None):
        """(d_q, d_k, d_v), contiguous."""
        d_q, d_k, d_v = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v))
        self.attention_backward_into(q, k, v, out, lse, d_out, d_q, d_k, d_v, scale, causal, q_lens, k_lens)
        return d_q, d_k, d_v

    @staticmethod
    def attention_forward_bytes(batch: int, q_len: int, k_len: int, heads: int, kv_heads: int, dim: int) -> int:
        """Bytes of the work buffer that attention_forward_into takes: 0 unless few queries go over many keys."""
        return _lib.ps_attention_forward_bytes(_ATTENTION_SHAPE(batch, q_len, k_len, heads, kv_heads, dim, 1, 0, 1.0, 0))

    @staticmethod
    def attention_backward_bytes(batch: int, q_len: int, k_len: int, heads: int, kv_heads: int, dim: int) -> int:
        """Bytes of the work buffer that attention_backward_into takes."""
        return _lib.ps_attention_backward_bytes(_ATTENTION_SHAPE(batch, q_len, k_len, heads, kv_heads, dim, 1, 0, 1.0, 0))

    def _matrix(self, t: torch.Tensor | None, where: str, name: str, shape, dtype) -> bytes | None:
        if t is None:
            return None
        return _MATRIX(t.data_ptr(), self._row_stride(t, where, name, shape, dtype))

    def _vector(self, t: torch.Tensor | None, where: str, name: str, n: int, dtype) -> int | None:
        if t is None:
            return None
        if t.shape != (n,) or t.dtype != dtype or t.get_device() != self.device or (n > 1 and t.stride(0) != 1):
            self._refuse(E_RANGE, where, f"{name} has to be {n} contiguous {dtype} on device {self.device}")
        return t.data_ptr()

    def _rows(self, x: torch.Tensor, where: str, name: str):
        if x.dim() != 2 or x.dtype not in _DTYPE:
            self._refuse(E_RANGE, where, f"{name} has to be [rows, cols] of float32, bfloat16 or float16")
        return x.shape

    def _finite(self, where: str, name: str, value: float):
        if not -_FLOAT_MOST <= value <= _FLOAT_MOST:
            self._refuse(E_RANGE, where, name)

    def layer_norm_forward_into(self, x: torch.Tensor, y: torch.Tensor, weight: torch.Tensor | None = None,
                                bias: torch.Tensor | None = None, eps: float = 1e-5, mean: torch.Tensor | None = None,
                                rstd: torch.Tensor | None = None):
        """ps_layer_norm_forward on [rows, cols]; `mean` and `rstd`, float32 [rows], are written where they are given.  y may be x."""
        where = "ps_layer_norm_forward"
        rows, _ = shape = self._rows(x, where, "x")
        self._norm_forward(x, weight, bias, eps, self._matrix(y, where, "y", shape, x.dtype), self._vector(mean, where, "mean", rows, torch.float32),
                           self._vector(rstd, where, "rstd", rows, torch.float32))

    def _norm_forward(self, x, weight, bias, eps, y: bytes, mean: int | None, rstd: int | None):
        where, dtype = "ps_layer_norm_forward", x.dtype
        rows, cols = shape = self._rows(x, where, "x")
        self._finite(where, "eps", eps)
        self._enqueue(where, _lib.ps_layer_norm_forward, _LAYER_NORM_DESC(rows, cols, eps, _DTYPE[dtype], 0, 0, 0),
                      self._matrix(x, where, "x", shape, dtype), self._vector(weight, where, "weight", cols, dtype),
                      self._vector(bias, where, "bias", cols, dtype), y, mean, rstd)

    def layer_norm_forward(self, x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                           eps: float = 1e-5):
        """(y [rows, cols], mean [rows], rstd [rows])."""
        rows, cols = self._rows(x, "ps_layer_norm_forward", "x")
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind()
        at = mean.data_ptr()
        self._norm_forward(x, weight, bias, eps, _MATRIX(y.data_ptr(), cols), at, at + 4 * rows)
        return y, mean, rstd

    def layer_norm_backward_into(self, d_y: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, d_x: torch.Tensor,
                                 weight: torch.Tensor | None = None, residual: torch.Tensor | None = None,
                                 d_weight: torch.Tensor | None = None, d_bias: torch.Tensor | None = None, accumulate: bool = False,
                                 work: torch.Tensor | None = None):
        """ps_layer_norm_backward: the gradient of x, plus `residual`, to d_x (which may be d_y, x or residual), and those of
        weight and bias where they are given, written or (accumulate) added to.
        `work`: a uint8 buffer of layer_norm_backward_bytes; without it one is allocated for a call that needs it."""
        where, dtype = "ps_layer_norm_backward", x.dtype
        rows, cols = shape = self._rows(x, where, "x")
        sums = d_weight if d_weight is not None else d_bias
        wide = dtype if sums is None else sums.dtype
        if wide not in _DTYPE:
            self._refuse(E_RANGE, where, "d_weight and d_bias have to be of float32, bfloat16 or float16")
        desc = _LAYER_NORM_DESC(rows, cols, 0.0, _DTYPE[dtype], _DTYPE[wide], 1 if accumulate else 0, 0)
        at, size = None, 0
        if sums is not None:
            work = self._work(work, _lib.ps_layer_norm_backward_bytes(desc), where)
            at, size = work.data_ptr(), work.numel()
        self._enqueue(where, _lib.ps_layer_norm_backward, desc, self._matrix(d_y, where, "d_y", shape, dtype),
                      self._matrix(x, where, "x", shape, dtype), self._vector(mean, where, "mean", rows, torch.float32),
                      self._vector(rstd, where, "rstd", rows, torch.float32), self._vector(weight, where, "weight", cols, dtype),
                      self._matrix(residual, where, "residual", shape, dtype), self._matrix(d_x, where, "d_x", shape, dtype),
                      self._vector(d_weight, where, "d_weight", cols, wide), self._vector(d_bias, where, "d_bias", cols, wide), at, size)

    def layer_norm_backward(self, d_y: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            weight: torch.Tensor | None = None, residual: torch.Tensor | None = None, dtype: torch.dtype | None = None):
        """(d_x, d_weight, d_bias), the last two in x's type or `dtype`."""
        d_x = torch.empty_like(x, memory_format=torch.contiguous_format)
        d_weight, d_bias = (x.new_empty(x.shape[-1:], dtype=dtype) for _ in range(2))
        self.layer_norm_backward_into(d_y, x, mean, rstd, d_x, weight, residual, d_weight, d_bias)
        return d_x, d_weight, d_bias

    @staticmethod
    def layer_norm_backward_bytes(rows: int, cols: int, dtype: torch.dtype) -> int:
        """Bytes of the work buffer that layer_norm_backward_into takes for gradients of weight and bias."""
        return _lib.ps_layer_norm_backward_bytes(_LAYER_NORM_DESC(rows, cols, 0.0, _DTYPE[dtype], 0, 0, 0))

    def rotary_into(self, q: torch.Tensor, q_out: torch.Tensor, k: torch.Tensor | None = None, k_out: torch.Tensor | None = None,
                    positions: torch.Tensor | None = None, first: int = 0, base: float = 10000.0, dims: int | None = None,
                    interleaved: bool = False, factor: float = 1.0, original: float = 0.0, low: float = 1.0, high: float = 32.0,
                    magnitude: float = 1.0, inverse: bool = False):
        """ps_rotary on [batch, len, heads, dim] of any strides; q_out may be q, k_out k.  `positions`: int32 or int64,
        [len] or [batch, len]; without them a token's position is its place in the sequence.  `first` is added to all;
        `dims` of a head's elements are turned (default: all)."""
        where, dtype = "ps_rotary", q.dtype
        if (k is None) != (k_out is None) or q.dim() != 4 or (k is not None and k.dim() != 4):
            self._refuse(E_RANGE, where, "q, and k with k_out, are [batch, len, heads, dim]")
        self._rotary(q, self._heads(q_out, where, "q_out", q.shape, dtype), k, None if k is None else self._heads(k_out, where, "k_out", (*q.shape[:2], k.shape[2], q.shape[3]), dtype),
                     positions, first, base, dims, interleaved, factor, original, low, high, magnitude, inverse)

    def _rotary(self, q, q_out: bytes, k, k_out: bytes | None, positions=None, first=0, base=10000.0, dims=None, interleaved=False, factor=1.0,
                original=0.0, low=1.0, high=32.0, magnitude=1.0, inverse=False):
        where, dtype = "ps_rotary", q.dtype
        if dtype not in _DTYPE:
            self._refuse(E_RANGE, where, "q has to be of float32, bfloat16 or float16")
        batch, length, heads, dim = q.shape
        kv_heads = 0 if k is None else k.shape[2]
        width, apart, at = 4, 0, None
        if positions is not None:
            if positions.dtype not in (torch.int32, torch.int64) or positions.shape not in ((length,), (batch, length)) \
                    or positions.get_device() != self.device:
                self._refuse(E_RANGE, where, f"positions have to be [len] or [batch, len] of int32 or int64 on device {self.device}")
            if length > 1 and positions.stride(-1) != 1:
                self._refuse(E_ALIGN, where, "positions are not contiguous")
            width, apart, at = positions.element_size(), positions.stride(0) if positions.dim() == 2 and batch > 1 else 0, positions.data_ptr()
        if not -(1 << 63) <= first < 1 << 63:
            self._refuse(E_RANGE, where, "first")
        self._finite(where, "magnitude", magnitude)
        dims = dim if dims is None else dims
        if not 0 <= dims <= dim:
            self._refuse(E_RANGE, where, "dims")
        desc = _ROTARY_DESC(batch, length, heads, kv_heads, dim, dims, _DTYPE[dtype], 1 if interleaved else 0, 1 if inverse else 0, width,
                            apart, first, base, factor, original, low, high, magnitude)
        self._enqueue(where, _lib.ps_rotary, desc, self._heads(q, where, "q", q.shape, dtype), q_out,
                      None if k is None else self._heads(k, where, "k", (batch, length, kv_heads, dim), dtype), k_out, at)

    def rotary(self, q: torch.Tensor, k: torch.Tensor | None = None, **how):
        """q, or (q, k), turned by their positions; `how` as for rotary_into.  The gradient is the same call on the result's
        gradients with inverse=True."""
        if q.dim() != 4 or (k is not None and k.dim() != 4):
            self._refuse(E_RANGE, "ps_rotary", "q and k are [batch, len, heads, dim]")
        q_out, q_heads = self._new_heads(q)
        if k is None:
            self._rotary(q, q_heads, None, None, **how)
            return q_out
        k_out, k_heads = self._new_heads(k)
        self._rotary(q, q_heads, k, k_heads, **how)
        return q_out, k_out

    @staticmethod
    def _new_heads(like: torch.Tensor):
        """A contiguous tensor of that shape, and the library's description of it."""
        _, length, heads, dim = shape = like.shape
        t = torch.empty_like(like, memory_format=torch.contiguous_format)
        return t, _HEADS(t.data_ptr(), length * heads * dim, heads * dim, dim)

    def _activation(self, where: str, name) -> int:
        if name not in ACTIVATIONS:
            self._refuse(E_RANGE, where, f"activation {name!r} is none of {', '.join(n for n in ACTIVATIONS if n)}")
        return ACTIVATIONS[name]

    def linear_forward_into(self, x: torch.Tensor, weight: torch.Tensor, y: torch.Tensor, bias: torch.Tensor | None = None,
                            activation: str | None = None, residual: torch.Tensor | None = None, pre: torch.Tensor | None = None):
        """ps_linear_forward: y [tokens, outputs] = act(x weight^T + bias) + residual, and what goes into the activation to
        `pre` where it is given.  Rows of the matrices begin at multiples of 16 bytes; residual may be y."""
        where, dtype = "ps_linear_forward", x.dtype
        shape = self._rows(x, where, "x")[0], self._rows(weight, where, "weight")[0]
        self._linear_forward(x, weight, bias, activation, residual, self._matrix(y, where, "y", shape, dtype), self._matrix(pre, where, "pre", shape, dtype))

    def _linear_forward(self, x, weight, bias, activation, residual, y: bytes, pre: bytes | None):
        where, dtype = "ps_linear_forward", x.dtype
        tokens, inputs = x.shape
        outputs = weight.shape[0]
        code, of = self._activation(where, activation), _DTYPE[dtype]
        self._enqueue(where, _lib.ps_linear_forward, _LINEAR_DESC(tokens, inputs, outputs, of, of, code, 0, 0, 0),
                      self._matrix(x, where, "x", (tokens, inputs), dtype), self._matrix(weight, where, "weight", (outputs, inputs), dtype),
                      self._vector(bias, where, "bias", outputs, dtype), self._matrix(residual, where, "residual", (tokens, outputs), dtype), y, pre)

    @staticmethod
    def _new_rows(like: torch.Tensor, rows: int, cols: int, dtype: torch.dtype | None = None):
        """[rows, cols] whose rows begin at multiples of 16 bytes, and the library's description of it."""
        pack = 4 if (dtype or like.dtype) == torch.float32 else 8
        if cols % pack == 0:
            t = like.new_empty((rows, cols), dtype=dtype)
            return t, _MATRIX(t.data_ptr(), cols)
        stride = (cols + pack - 1) // pack * pack
        t = like.new_empty((rows, stride), dtype=dtype)[:, :cols]
        return t, _MATRIX(t.data_ptr(), stride)

    def linear_forward(self, x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, activation: str | None = None,
                       residual: torch.Tensor | None = None, keep: bool = False):
        """y, or with `keep` (y, pre): pre is what linear_backward takes.  (Columns of a larger tensor where outputs are no
        multiple of 8.)"""
        where = "ps_linear_forward"
        tokens, outputs = self._rows(x, where, "x")[0], self._rows(weight, where, "weight")[0]
        y, y_rows = self._new_rows(x, tokens, outputs)
        if not keep:
            self._linear_forward(x, weight, bias, activation, residual, y_rows, None)
            return y
        pre, pre_rows = self._new_rows(x, tokens, outputs)
        self._linear_forward(x, weight, bias, activation, residual, y_rows, pre_rows)
        return y, pre

    def linear_backward_into(self, d_y: torch.Tensor, x: torch.Tensor | None, weight: torch.Tensor | None,
                             d_x: torch.Tensor | None = None, d_weight: torch.Tensor | None = None, d_bias: torch.Tensor | None = None,
                             pre: torch.Tensor | None = None, activation: str | None = None, below: torch.Tensor | None = None,
                             below_activation: str | None = None, residual: torch.Tensor | None = None, accumulate: bool = False,
                             work: torch.Tensor | None = None):
        """ps_linear_backward: those of the gradients of x, weight and bias that are given.  `pre` with an activation; `below` is
        what x came out of by below_activation: d_x is then the gradient of that.  `residual` is added to d_x and may be
        it.  accumulate adds to d_weight and d_bias.  x may be None without d_weight, weight without d_x.
        `work`: a uint8 buffer of linear_backward_bytes; without it one is allocated for the call."""
        where, dtype = "ps_linear_backward", d_y.dtype
        tokens, outputs = self._rows(d_y, where, "d_y")
        inputs = 1
        for t, of in ((x, d_weight), (weight, d_x)):
            if t is not None:
                inputs = self._rows(t, where, "x and weight")[1]
            elif of is not None:
                self._refuse(E_NULLPTR, where, "the gradient of weight needs x, that of x needs weight")
        sums = d_weight if d_weight is not None else d_bias
        wide = dtype if sums is None else sums.dtype
        self._linear_backward(d_y, x, weight, inputs, wide, self._matrix(d_x, where, "d_x", (tokens, inputs), dtype),
                              self._matrix(d_weight, where, "d_weight", (outputs, inputs), wide), self._vector(d_bias, where, "d_bias", outputs, wide),
                              pre, activation, below, below_activation, residual, accumulate, work)

    def _linear_backward(self, d_y, x, weight, inputs: int, wide, d_x: bytes | None, d_weight: bytes | None, d_bias: int | None, pre, activation, below,
                         below_activation, residual, accumulate, work):
        where, dtype = "ps_linear_backward", d_y.dtype
        tokens, outputs = d_y.shape
        if wide is not dtype and wide != torch.float32:
            self._refuse(E_RANGE, where, f"d_weight and d_bias have to be {dtype} or float32")
        code, below_code = self._activation(where, activation), self._activation(where, below_activation)
        shape, in_shape = (tokens, outputs), (tokens, inputs)
        desc = _LINEAR_DESC(tokens, inputs, outputs, _DTYPE[dtype], _DTYPE[wide], code, below_code, 1 if accumulate else 0, 0)
        work = self._work(work, _lib.ps_linear_backward_bytes(desc), where)
        self._enqueue(where, _lib.ps_linear_backward, desc, self._matrix(d_y, where, "d_y", shape, dtype),
                      self._matrix(x, where, "x", in_shape, dtype), self._matrix(weight, where, "weight", (outputs, inputs), dtype),
                      self._matrix(pre, where, "pre", shape, dtype), self._matrix(below, where, "below", in_shape, dtype),
                      self._matrix(residual, where, "residual", in_shape, dtype), d_x, d_weight, d_bias, work.data_ptr(), work.numel())

    def linear_backward(self, d_y: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, pre: torch.Tensor | None = None,
                        activation: str | None = None, below: torch.Tensor | None = None, below_activation: str | None = None,
                        residual: torch.Tensor | None = None, dtype: torch.dtype | None = None):
        """(d_x, d_weight, d_bias), the last two in x's type or `dtype`."""
        where = "ps_linear_backward"
        self._rows(d_y, where, "d_y")
        tokens, inputs = self._rows(x, where, "x")
        outputs = self._rows(weight, where, "weight")[0]
        (d_x, x_rows), (d_weight, w_rows) = self._new_rows(x, tokens, inputs), self._new_rows(weight, outputs, inputs, dtype)
        d_bias = weight.new_empty((outputs,), dtype=dtype)
        self._linear_backward(d_y, x, weight, inputs, d_weight.dtype, x_rows, w_rows, d_bias.data_ptr(), pre, activation, below, below_activation, residual,
                              False, None)
        return d_x, d_weight, d_bias

    @staticmethod
    def linear_backward_bytes(tokens: int, inputs: int, outputs: int, activation: str | None = None, dtype: torch.dtype | None = None) -> int:
        """Bytes of the work buffer that linear_backward_into takes; `dtype`: of the gradients of weight and bias (default: enough for any)."""
        wide = _DTYPE[torch.float32 if dtype is None else dtype]
        return _lib.ps_linear_backward_bytes(_LINEAR_DESC(tokens, inputs, outputs, wide or _DTYPE[torch.bfloat16], wide, ACTIVATIONS[activation], 0, 0, 0))

    def int_peak(self, blocks: int, iters: int, sink: torch.Tensor) -> int:
        ops = C.c_uint64()
        _check(_lib.ps_int_peak(self._h, blocks, iters, _dptr(sink), C.byref(ops)), "ps_int_peak")
        return ops.value


class Space:
    """ps_space: the device copy of a model table plus the enumeration."""

    def __init__(self, ctx: Context, space: dict):
        self.ctx = ctx
        models = np.ascontiguousarray(space["models"])
        assert models.dtype.itemsize == 48
        n_values = np.ascontiguousarray(space["n_values"], dtype=np.uint32)
        desc = _SpaceDesc(models.ctypes.data, len(models), n_values.ctypes.data, len(n_values),
                          space["t_enum_max"], space["k_enum_max"], space["tp_max_valid"],
                          space["n_act_variants"], space["n_tpa_variants"], space["mode_mask"],
                          space["tp_coll_per_layer"], space.get("sstar_units", 1),
                          space.get("grad_accum_steps", 1), space.get("replication_k", 1))
        handle = C.c_void_p()
        _check(_lib.ps_space_create(ctx._h, C.byref(desc), C.byref(handle)), "ps_space_create")
        self._h = handle
        self.n_models = len(models)

    def close(self):
        if getattr(self, "_h", None) and getattr(self.ctx, "_h", None) and _lib is not None:
            _lib.ps_space_destroy(self._h)
        self._h = None

    __del__ = close

    @property
    def size(self) -> int:
        return _lib.ps_space_size(self._h)

    @property
    def points_per_model(self) -> int:
        return _lib.ps_space_points_per_model(self._h)

    def decode(self, idx: int) -> dict:
        p = _Point()
        _check(_lib.ps_space_decode(self._h, idx, C.byref(p)), "ps_space_decode")
        return {f: getattr(p, f) for f, _ in _Point._fields_ if f != "pad"}

    def set_models(self, models_host) -> None:
        """Replace the shape table from host memory (numpy array or a pinned torch
        uint8 tensor of 48-byte records)."""
        if isinstance(models_host, torch.Tensor):
            ptr, n = models_host.data_ptr(), models_host.numel() * models_host.element_size() // 48
        else:
            models_host = np.ascontiguousarray(models_host)
            ptr, n = models_host.ctypes.data, len(models_host)
        _check(_lib.ps_space_set_models(self._h, ptr, n), "ps_space_set_models")

    def rederive(self) -> None:
        _check(_lib.ps_space_rederive(self._h), "ps_space_rederive")

    # ---- ps_eval_batch
    def eval_batch_into(self, first: int, count: int, out: dict, filt: dict | None = None,
                        idx_out: torch.Tensor | None = None, n_out: torch.Tensor | None = None):
        """Raw call: `out` maps any of mem/comm_paper/comm_ext/host/flags to device tensors."""
        soa = _OutSoa(*(None if out.get(k) is None else out[k].data_ptr()
                        for k in ("mem", "comm_paper", "comm_ext", "host", "flags")))
        f = _mk_filter(filt) if filt is not None else None
        _check(_lib.ps_eval_batch(self.ctx._h, self._h, first, count,
                                  C.byref(f) if f is not None else None, soa, _dptr(idx_out),
                                  _dptr(n_out)), "ps_eval_batch")

    def alloc_outputs(self, count: int, fields=("mem", "comm_paper", "comm_ext", "host", "flags")):
        dev = self.ctx.torch_device
        out = {}
        for k in fields:
            dt = torch.int32 if k == "flags" else torch.int64
            out[k] = torch.empty(max(count, 1), dtype=dt, device=dev)
        return out

    @_on_own_stream
    def eval_batch(self, first: int, count: int,
                   fields=("mem", "comm_paper", "comm_ext", "host", "flags")) -> dict:
        """Materialise [first, first+count) and return numpy arrays (unsigned)."""
        out = self.alloc_outputs(count, fields)
        self.eval_batch_into(first, count, out)
        self.ctx.check_status()
        return {k: _to_unsigned(v[:count]) for k, v in out.items()}

    @_on_own_stream
    def compact(self, first: int, count: int, filt: dict,
                fields=("mem", "comm_paper", "comm_ext", "host", "flags")) -> dict:
        """Filter and compact; returns numpy arrays of the survivors incl. 'idx'."""
        dev = self.ctx.torch_device
        out = self.alloc_outputs(count, fields)
        idx = torch.empty(max(count, 1), dtype=torch.int64, device=dev)
        n = torch.zeros(1, dtype=torch.int64, device=dev)
        self.eval_batch_into(first, count, out, filt, idx, n)
        self.ctx.check_status()
        k = int(n.item())
        res = {name: _to_unsigned(v[:k]) for name, v in out.items()}
        res["idx"] = _to_unsigned(idx[:k])
        return res

    def compact_noalloc_into(self, first: int, count: int, out: dict, filt: dict,
                             idx_out: torch.Tensor | None, n_out: torch.Tensor):
        """ps_eval_compact_noalloc: same contract as the filtered eval_batch_into, but the
        library allocates nothing (fixed scratch; at most NOALLOC_MAX_GROUPS groups per
        call; calls on one device must not overlap)."""
        soa = _OutSoa(*(None if out.get(k) is None else out[k].data_ptr()
                        for k in ("mem", "comm_paper", "comm_ext", "host", "flags")))
        f = _mk_filter(filt)
        _check(_lib.ps_eval_compact_noalloc(self.ctx._h, self._h, first, count, C.byref(f), soa,
                                            _dptr(idx_out), _dptr(n_out)), "ps_eval_compact_noalloc")

    # ---- ps_sweep_pareto
    def sweep_into(self, filt: dict, caps, kind: int, max_entries: int, d_out: torch.Tensor,
                   d_counts: torch.Tensor):
        self._sweep(filt, caps, kind, max_entries, _dptr(d_out), _dptr(d_counts))

    def _sweep(self, filt, caps, kind, max_entries, out_ptr, counts_ptr):
        caps = np.ascontiguousarray(caps, dtype=np.uint64)
        f = _mk_filter(filt)
        _check(_lib.ps_sweep_pareto(self.ctx._h, self._h, C.byref(f), caps.ctypes.data, len(caps),
                                    kind, max_entries, out_ptr, counts_ptr),
               "ps_sweep_pareto")

    @_on_own_stream
    def select_compare(self, n_index: int, device_bytes: int, filt: dict, d_frontier: torch.Tensor,
                       d_counts: torch.Tensor, n_caps: int, cap_index: int, max_entries: int, fast: int = 1,
                       headroom=(7, 10), layer=(3, 10), tp_degree: int = 8) -> np.ndarray:
        """ps_select_compare on the device outputs of a Pareto sweep; returns SELECT_COMPARE_DTYPE records."""
        d_out = torch.zeros(self.n_models * 72, dtype=torch.uint8, device=self.ctx.torch_device)
        f = _mk_filter(filt)
        _check(_lib.ps_select_compare(self.ctx._h, self._h, n_index, device_bytes, fast, headroom[0], headroom[1],
                                      layer[0], layer[1], tp_degree, C.byref(f), _dptr(d_frontier), _dptr(d_counts),
                                      n_caps, cap_index, max_entries, _dptr(d_out)), "ps_select_compare")
        self.ctx.check_status()
        return d_out.cpu().numpy().view(SELECT_COMPARE_DTYPE)

    def alloc_sweep(self, n_caps: int, max_entries: int):
        dev = self.ctx.torch_device
        d_out = torch.empty(self.n_models * n_caps * max_entries * 40, dtype=torch.uint8, device=dev)
        d_counts = torch.empty(self.n_models * n_caps, dtype=torch.int32, device=dev)
        return d_out, d_counts

    @_on_own_stream
    def sweep(self, filt: dict, caps, kind: int, max_entries: int):
        """Returns (entries[n_models, n_caps, max_entries] structured, counts[n_models, n_caps]).  Both are
        views of one buffer; up to PINNED_RESULT_BYTES it is page-locked for as long as either is kept."""
        rows = self.n_models * len(caps)
        at = rows * max_entries * 40                   # the counts lie behind the entries: one copy brings both
        d_all = torch.empty(at + rows * 4, dtype=torch.uint8, device=self.ctx.torch_device)
        base = d_all.data_ptr()
        self._sweep(filt, caps, kind, max_entries, base, base + at)
        flat, self.last_sweep_status = self.ctx._read_back(d_all, allow_truncated=True)
        entries = flat[:at].view(ENTRY_DTYPE).reshape(self.n_models, len(caps), max_entries)
        counts = flat[at:].view(np.uint32).reshape(self.n_models, len(caps))
        return entries, counts


def _to_unsigned(t: torch.Tensor) -> np.ndarray:
    a = t.cpu().numpy()
    return a.view(np.uint64 if a.dtype == np.int64 else np.uint32)
