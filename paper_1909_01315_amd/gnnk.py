"""Python binding of libgnnk.so (the C ABI declared in include/gnnk.h).

Argument marshalling only: every operation runs in the HIP library.  PyTorch
provides device memory (outputs are allocated here with torch.empty and
handed to the library, which computes their sizes' contents) and the current
HIP stream.  There is no CPU fallback: if the library is missing or cannot be
loaded, every call raises.

Tensors are torch tensors on the GPU, float32 or bfloat16, shaped (rows, heads,
feat) -- a 2-D (rows, d) tensor is read as (rows, 1, d) -- with the last two
dimensions contiguous (the row stride may be larger).  Outputs that are passed
in must not overlap what a call reads or each other, unless it says so.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgnnk.so")

OK, EINVAL, EUNSUPPORTED, EHIP, ERANGE, ENOMEM = range(6)
I32, I64 = 0, 1
F32, BF16 = 0, 1
OPS = {"copy_lhs": 0, "copy_rhs": 1, "add": 2, "sub": 3, "mul": 4, "div": 5, "dot": 6}
REDUCES = {"sum": 0, "mean": 1, "max": 2, "min": 3}
TARGETS = {"u": 0, "e": 1, "v": 2}

_lib = None


class GnnkError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"gnnk status {status}: {msg}")
        self.status = status


# gnnk_tensor (data, rows, heads, feat, row_stride, dtype, reserved) as bytes:
# packed in 0.3 us, where filling a ctypes structure takes 1.2 us
_TENSOR = struct.Struct("=QqIIqII")


class _Info(ctypes.Structure):
    _fields_ = [("num_src", ctypes.c_int64), ("num_dst", ctypes.c_int64), ("num_edges", ctypes.c_int64),
                ("ptr_type", ctypes.c_int32), ("identity_eids", ctypes.c_int32),
                ("max_in_degree", ctypes.c_int64), ("max_out_degree", ctypes.c_int64),
                ("empty_dst_rows", ctypes.c_int64), ("empty_src_rows", ctypes.c_int64),
                ("seg_edges", ctypes.c_int64), ("hub_dst_rows", ctypes.c_int64), ("hub_src_rows", ctypes.c_int64),
                ("segments_in", ctypes.c_int64), ("segments_out", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_size_t), ("seg_edges_out", ctypes.c_int64),
                ("seg_edges_gather", ctypes.c_int64), ("segments_gather", ctypes.c_int64),
                ("seg_edges_in_gather", ctypes.c_int64), ("segments_in_gather", ctypes.c_int64),
                ("kept_bytes", ctypes.c_size_t), ("lists_bytes", ctypes.c_size_t),
                ("neighbour_lists", ctypes.c_int32), ("reserved", ctypes.c_int32)]


# gnnk_build_memory (workspace, bytes, temporaries, bytes, lists, ctx) as bytes
_MEMORY = struct.Struct("=QQQQQQ")
# what the build that runs on this thread gives its neighbour lists: device, tensor
_building = threading.local()


@ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t)
def _allocate_lists(_ctx, nbytes):
    try:
        _building.lists = torch.empty(nbytes, dtype=torch.uint8, device=_building.device)
    except RuntimeError:  # out of memory: the graph does without
        return None
    return _building.lists.data_ptr()


_ALLOCATE_LISTS = ctypes.cast(_allocate_lists, ctypes.c_void_p).value


SYMBOLS = {
    "graph_workspace_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p],
    "graph_create_coo": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                         ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p],
    "graph_create_csr": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int,
                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                         ctypes.c_void_p],
    "graph_build_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                          ctypes.c_void_p],
    "graph_build_coo": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                        ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "graph_build_csr": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int,
                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "graph_info": [ctypes.c_void_p, ctypes.c_void_p],
    "graph_in_degrees": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "graph_out_degrees": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "graph_csr_export": [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                         ctypes.c_void_p],
    "graph_validate": [ctypes.c_void_p, ctypes.c_void_p],
    "graph_destroy": [ctypes.c_void_p],
    "gspmm": [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "gspmm_noalloc": [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "gsddmm": [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
               ctypes.c_void_p, ctypes.c_void_p],
    "gspmm_backward": [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                       ctypes.c_void_p],
    "gsddmm_backward": [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "edge_softmax": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "edge_softmax_backward": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "edge_leaky_relu": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p],
    "edge_leaky_relu_backward": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                                 ctypes.c_void_p],
    "gat_aggregate": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "gat_aggregate_backward": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                               ctypes.c_void_p],
    "dot_aggregate": [ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_void_p] * 3,
    "dot_aggregate_backward": [ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_void_p] * 8,
    "node_rotary": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p],
    "node_norm_rotary": [ctypes.c_void_p] * 8 + [ctypes.c_float, ctypes.c_void_p],
    "node_norm_rotary_backward": [ctypes.c_void_p] * 12 + [ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t,
                                                           ctypes.c_void_p],
    "node_norm_rotary_work_bytes": [ctypes.c_void_p] * 5,
    "node_add_norm": [ctypes.c_void_p] * 3 + [ctypes.c_float] + [ctypes.c_void_p] * 3,
    "node_add_norm_i8": [ctypes.c_void_p] * 3 + [ctypes.c_float] + [ctypes.c_void_p] * 3,
    "node_quantize": [ctypes.c_void_p] * 3,
    "node_add_norm_backward": [ctypes.c_void_p] * 4 + [ctypes.c_float] + [ctypes.c_void_p] * 3 + [ctypes.c_size_t,
                                                                                              ctypes.c_void_p],
    "node_add_norm_work_bytes": [ctypes.c_void_p] * 2,
    "weight8_bytes": [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p],
    "weight8_pack": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "node_linear_i8": [ctypes.c_void_p] * 5,
    "graph_scratch_bytes": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p],
    "graph_attach_scratch": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t],
    "graph_scratch_captured": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "gnnk_scratch_needed": [ctypes.c_void_p],
    "gnnk_set_option": [ctypes.c_char_p, ctypes.c_int64],
    "gnnk_last_error": [],
}


def load():
    """Load libgnnk.so (raises if it is missing)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built (run __graft_entry__.build() or "
                              "python -m paper_1909_01315_amd.build)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, args in SYMBOLS.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        lib.gnnk_last_error.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def _check(status: int):
    if status != OK:
        raise GnnkError(status, load().gnnk_last_error().decode())


# handle of the current stream of the current device, without building the
# Stream object of torch.cuda.current_stream() (0.3 us instead of 2)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


SCRATCH_ARGMAX, SCRATCH_WIDE_SUMS = 1, 2


def _run(g, stream, fn, *args):
    """Run fn (a C entry point on g) with args and the stream; when it ran
    short of scratch, lend g a buffer of the size it asked for on the call's
    stream and run it again (outputs are overwritten, never accumulated, so a
    repeated call gives the same result).  A call that needs several parts
    asks for them in turn."""
    st = fn(*args, _stream(stream))
    if st == OK:
        return
    for _ in range(4):
        if st != ENOMEM:
            break
        need = ctypes.c_size_t(0)
        load().gnnk_scratch_needed(ctypes.byref(need))
        if need.value == 0:  # short of something else (a workspace)
            break
        g.lend_scratch(need.value, stream)
        st = fn(*args, _stream(stream))
    _check(st)


def _as3(t: torch.Tensor) -> torch.Tensor:
    if t.dim() == 2:
        t = t.unsqueeze(1)
    if t.dim() != 3:
        raise ValueError("tensors are (rows, heads, feat)")
    return t


def _desc(t):
    """gnnk_tensor bytes of a (rows, heads, feat) GPU tensor."""
    if t is None:
        return None
    if t.dim() != 3:
        t = _as3(t)
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    dtype = t.dtype
    if dtype is torch.float32:
        dt = F32
    elif dtype is torch.bfloat16:
        dt = BF16
    else:
        raise TypeError(f"unsupported dtype {dtype}")
    rows, h, f = t.shape
    s0, s1, s2 = t.stride()
    stride = h * f
    if rows and stride:  # (of an empty tensor no element is addressed: any strides will do)
        if (f > 1 and s2 != 1) or (h > 1 and s1 != f):
            raise ValueError("the last two dimensions must be contiguous")
        if rows > 1:
            if s0 < stride:
                raise ValueError("row stride smaller than heads * feat")
            stride = s0
    return _TENSOR.pack(t.data_ptr(), rows, h & 0xFFFFFFFF, f & 0xFFFFFFFF, stride, dt, 0)


def _ref(d):
    """argument of a const gnnk_tensor* parameter (the bytes' own storage)"""
    return d


def _ptr(t):
    return t.data_ptr() if t is not None else None


def set_option(key: str, value: int):
    _check(load().gnnk_set_option(key.encode(), int(value)))


class Graph:
    """A gnnk graph handle with its device workspace (and any borrowed arrays)."""

    def __init__(self, handle, keep, num_src, num_dst, num_edges):
        self._h = handle
        self._keep = keep  # tensors the handle points into
        self._lent = {}    # stream handle -> scratch buffer lent for that stream
        self._replaced = []  # smaller ones lent before, which captured graphs hold
        self.num_src, self.num_dst, self.num_edges = num_src, num_dst, num_edges

    @property
    def device(self):
        return self._keep[0].device

    def scratch_bytes(self, max_cols: int, argmax: bool = False, wide_sums: bool = False) -> int:
        """Bytes of scratch any call with messages of at most max_cols columns needs."""
        n = ctypes.c_size_t(0)
        flags = (SCRATCH_ARGMAX if argmax else 0) | (SCRATCH_WIDE_SUMS if wide_sums else 0)
        _check(load().graph_scratch_bytes(self.handle, int(max_cols), flags, ctypes.byref(n)))
        return n.value

    def lend_scratch(self, nbytes: int, stream=None):
        """Lend the handle a scratch buffer of at least nbytes for the calls on
        `stream` (default: the current stream), allocated on that stream,
        unless the one it has is large enough.  The buffer it replaces goes
        back to torch's allocator, which reuses it only for work ordered after
        the calls already queued on that stream; one that a captured call has
        taken stays with the handle, since the graph holds its address.
        Graphs captured on one stream share its buffer: their replays must not
        overlap."""
        s = stream if stream is not None else torch.cuda.current_stream()
        old = self._lent.get(s.cuda_stream)
        if old is not None and old.numel() >= nbytes:
            _check(load().graph_attach_scratch(self.handle, s.cuda_stream, old.data_ptr(), old.numel()))
            return
        captured = ctypes.c_int32(0)
        _check(load().graph_scratch_captured(self.handle, s.cuda_stream, ctypes.byref(captured)))
        size = max(int(nbytes), old.numel() * 5 // 4 if old is not None else 0, 256)
        with torch.cuda.stream(s):
            buf = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(load().graph_attach_scratch(self.handle, s.cuda_stream, buf.data_ptr(), size))
        if captured.value and old is not None:
            self._replaced.append(old)
        self._lent[s.cuda_stream] = buf

    @classmethod
    def _build(cls, fn, args, borrowed, num_src, num_dst, num_edges, ptr_t, device, neighbour_lists, stream):
        """fn (graph_build_coo or graph_build_csr) with args and the memory of
        the build: the handle keeps the workspace and its neighbour lists, the
        temporaries go back to torch's allocator, which reuses them only for
        work ordered after the build on its stream."""
        ws_bytes, tmp_bytes = ctypes.c_size_t(0), ctypes.c_size_t(0)
        _check(load().graph_build_bytes(num_src, num_dst, num_edges, ptr_t, ctypes.byref(ws_bytes),
                                        ctypes.byref(tmp_bytes)))
        ws = torch.empty(ws_bytes.value, dtype=torch.uint8, device=device)
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            tmp = torch.empty(tmp_bytes.value, dtype=torch.uint8, device=device)
        _building.device, _building.lists = device, None
        mem = _MEMORY.pack(ws.data_ptr(), ws_bytes.value, tmp.data_ptr(), tmp_bytes.value,
                           _ALLOCATE_LISTS if neighbour_lists else 0, 0)
        h = ctypes.c_void_p()
        try:
            _check(fn(num_src, num_dst, num_edges, *args, mem, _stream(stream), ctypes.byref(h)))
            return cls(h, [ws, _building.lists, *borrowed], num_src, num_dst, num_edges)
        finally:
            _building.lists = None

    @classmethod
    def from_coo(cls, src: torch.Tensor, dst: torch.Tensor, num_src: int, num_dst: int, ptr64: bool = False,
                 stream=None, neighbour_lists: bool = True) -> "Graph":
        """The graph of an edge list.  neighbour_lists: whether a graph that
        gains from it may also list its rows by neighbour (8 bytes per edge
        and direction, and two thirds of the build's time once more, which
        pays after some three passes over wide rows, ten to twenty over
        others)."""
        assert src.dtype == torch.int32 and dst.dtype == torch.int32 and src.is_cuda and dst.is_cuda
        src, dst = src.contiguous(), dst.contiguous()
        ptr_t = I64 if ptr64 else I32
        return cls._build(load().graph_build_coo, (src.data_ptr(), dst.data_ptr(), ptr_t), (), num_src, num_dst,
                          src.numel(), ptr_t, src.device, neighbour_lists, stream)

    @classmethod
    def from_csr(cls, indptr: torch.Tensor, indices: torch.Tensor, eids, num_src: int, stream=None,
                 neighbour_lists: bool = True) -> "Graph":
        """The graph of an in-CSR, whose arrays it keeps (neighbour_lists: as for from_coo)."""
        assert indptr.dtype in (torch.int32, torch.int64) and indices.dtype == torch.int32
        indptr, indices = indptr.contiguous(), indices.contiguous()
        if eids is not None:
            assert eids.dtype == torch.int32
            eids = eids.contiguous()
        ptr_t = I64 if indptr.dtype == torch.int64 else I32
        return cls._build(load().graph_build_csr, (indptr.data_ptr(), ptr_t, indices.data_ptr(), _ptr(eids)),
                          (indptr, indices, eids), num_src, indptr.numel() - 1, indices.numel(), ptr_t,
                          indices.device, neighbour_lists, stream)

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("graph destroyed")
        return self._h

    def info(self) -> dict:
        inf = _Info()
        _check(load().graph_info(self.handle, ctypes.byref(inf)))
        return {name: getattr(inf, name) for name, _ in _Info._fields_}

    def in_degrees(self, stream=None) -> torch.Tensor:
        out = torch.empty(self.num_dst, dtype=torch.int32, device=self._keep[0].device)
        _check(load().graph_in_degrees(self.handle, out.data_ptr(), _stream(stream)))
        return out

    def out_degrees(self, stream=None) -> torch.Tensor:
        out = torch.empty(self.num_src, dtype=torch.int32, device=self._keep[0].device)
        _check(load().graph_out_degrees(self.handle, out.data_ptr(), _stream(stream)))
        return out

    def csr_export(self, reverse: bool = False, stream=None):
        inf = self.info()
        dev = self._keep[0].device
        rows = self.num_src if reverse else self.num_dst
        pdt = torch.int64 if inf["ptr_type"] == I64 else torch.int32
        indptr = torch.empty(rows + 1, dtype=pdt, device=dev)
        indices = torch.empty(max(self.num_edges, 1), dtype=torch.int32, device=dev)
        eids = torch.empty(max(self.num_edges, 1), dtype=torch.int32, device=dev)
        _check(load().graph_csr_export(self.handle, int(reverse), indptr.data_ptr(), indices.data_ptr(),
                                       eids.data_ptr(), _stream(stream)))
        return indptr, indices[:self.num_edges], eids[:self.num_edges]

    def validate(self, stream=None):
        _check(load().graph_validate(self.handle, _stream(stream)))

    def destroy(self):
        if self._h is not None:
            _check(load().graph_destroy(self._h))
            self._h = None
            self._keep = None
            self._lent = self._replaced = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def rows_of(self, target: str) -> int:
        return {"u": self.num_src, "e": self.num_edges, "v": self.num_dst}[target]


def _msg_shape(op, lhs, rhs):
    if op == "copy_lhs":
        return lhs.shape[1], lhs.shape[2]
    if op == "copy_rhs":
        return rhs.shape[1], rhs.shape[2]
    return max(lhs.shape[1], rhs.shape[1]), max(lhs.shape[2], rhs.shape[2])


def _dev_dtype(*ts):
    for t in ts:
        if t is not None:
            return t.device, t.dtype
    raise ValueError("no tensor given")


def gspmm(g: Graph, op: str, reduce: str, lhs=None, rhs=None, out=None, want_args: bool = False, arg_lhs=None,
          arg_rhs=None, stream=None):
    """out[v] = reduce over in-edges (u, e, v) of op(lhs[u], rhs[e]).

    Returns out, or (out, arg_lhs, arg_rhs) for max/min with want_args (the
    arg arrays may be passed in preallocated)."""
    lhs = _as3(lhs) if lhs is not None else None
    rhs = _as3(rhs) if rhs is not None else None
    h, f = _msg_shape(op, lhs, rhs)
    dev, dt = _dev_dtype(lhs, rhs)
    if out is None:
        out = torch.empty((g.num_dst, h, f), dtype=dt, device=dev)
    arg_l, arg_r = arg_lhs, arg_rhs
    if want_args:
        if arg_l is None:
            arg_l = torch.empty((g.num_dst, h, f), dtype=torch.int32, device=dev)
        if arg_r is None:
            arg_r = torch.empty((g.num_dst, h, f), dtype=torch.int32, device=dev)
    _run(g, stream, load().gspmm, g.handle, OPS[op], REDUCES[reduce], _desc(lhs), _desc(rhs), _desc(out), _ptr(arg_l),
         _ptr(arg_r))
    return (out, arg_l, arg_r) if want_args else out


def gspmm_noalloc(g: Graph, op: str, reduce: str, lhs=None, rhs=None, out=None, arg_lhs=None, arg_rhs=None,
                  stream=None):
    """gspmm with the library's fixed per-GPU scratch buffer (no buffer is
    lent or allocated by the call; outputs and arg arrays are the caller's,
    allocated here only when not given).  Returns out, or (out, arg_lhs,
    arg_rhs) when arg arrays are given."""
    lhs = _as3(lhs) if lhs is not None else None
    rhs = _as3(rhs) if rhs is not None else None
    if out is None:
        h, f = _msg_shape(op, lhs, rhs)
        dev, dt = _dev_dtype(lhs, rhs)
        out = torch.empty((g.num_dst, h, f), dtype=dt, device=dev)
    _check(load().gspmm_noalloc(g.handle, OPS[op], REDUCES[reduce], _desc(lhs), _desc(rhs), _desc(out),
                                _ptr(arg_lhs), _ptr(arg_rhs), _stream(stream)))
    return (out, arg_lhs, arg_rhs) if (arg_lhs is not None or arg_rhs is not None) else out


def gsddmm(g: Graph, op: str, lhs, lhs_target: str, rhs, rhs_target: str, out=None, stream=None):
    """out[e] = op(lhs at its target, rhs at its target); targets 'u', 'e', 'v'."""
    lhs = _as3(lhs) if lhs is not None else None
    rhs = _as3(rhs) if rhs is not None else None
    if op == "dot":
        h, f = max(lhs.shape[1], rhs.shape[1]), 1
    else:
        h, f = _msg_shape(op, lhs, rhs)
    dev, dt = _dev_dtype(lhs, rhs)
    if out is None:
        out = torch.empty((g.num_edges, h, f), dtype=dt, device=dev)
    _run(g, stream, load().gsddmm, g.handle, OPS[op], _desc(lhs), TARGETS[lhs_target], _desc(rhs),
         TARGETS[rhs_target], _desc(out))
    return out


def gspmm_backward(g: Graph, op: str, reduce: str, lhs, rhs, grad_out, arg_rhs=None, want_lhs: bool = True,
                   want_rhs: bool = True, grad_lhs=None, grad_rhs=None, stream=None):
    """(grad_lhs, grad_rhs) of gspmm (either may be None)."""
    lhs = _as3(lhs) if lhs is not None else None
    rhs = _as3(rhs) if rhs is not None else None
    grad_out = _as3(grad_out)
    if want_lhs and lhs is not None and grad_lhs is None:
        grad_lhs = torch.empty(lhs.shape, dtype=grad_out.dtype, device=grad_out.device)
    if want_rhs and rhs is not None and grad_rhs is None:
        grad_rhs = torch.empty(rhs.shape, dtype=grad_out.dtype, device=grad_out.device)
    if not want_lhs:
        grad_lhs = None
    if not want_rhs:
        grad_rhs = None
    _run(g, stream, load().gspmm_backward, g.handle, OPS[op], REDUCES[reduce], _desc(lhs), _desc(rhs), None,
         _ptr(arg_rhs), _desc(grad_out), _desc(grad_lhs), _desc(grad_rhs))
    return grad_lhs, grad_rhs


def gsddmm_backward(g: Graph, op: str, lhs, lhs_target: str, rhs, rhs_target: str, grad_out, want_lhs=True,
                    want_rhs=True, grad_lhs=None, grad_rhs=None, stream=None):
    lhs = _as3(lhs) if lhs is not None else None
    rhs = _as3(rhs) if rhs is not None else None
    grad_out = _as3(grad_out)
    if want_lhs and lhs is not None and grad_lhs is None:
        grad_lhs = torch.empty(lhs.shape, dtype=grad_out.dtype, device=grad_out.device)
    if want_rhs and rhs is not None and grad_rhs is None:
        grad_rhs = torch.empty(rhs.shape, dtype=grad_out.dtype, device=grad_out.device)
    if not want_lhs:
        grad_lhs = None
    if not want_rhs:
        grad_rhs = None
    _run(g, stream, load().gsddmm_backward, g.handle, OPS[op], _desc(lhs), TARGETS[lhs_target], _desc(rhs),
         TARGETS[rhs_target], _desc(grad_out), _desc(grad_lhs), _desc(grad_rhs))
    return grad_lhs, grad_rhs


def edge_softmax(g: Graph, score, out=None, stream=None):
    score = _as3(score)
    if out is None:
        out = torch.empty(score.shape, dtype=score.dtype, device=score.device)
    _run(g, stream, load().edge_softmax, g.handle, _desc(score), _desc(out))
    return out


def edge_softmax_backward(g: Graph, out, grad_out, grad_score=None, stream=None):
    out, grad_out = _as3(out), _as3(grad_out)
    if grad_score is None:
        grad_score = torch.empty(out.shape, dtype=grad_out.dtype, device=grad_out.device)
    _run(g, stream, load().edge_softmax_backward, g.handle, _desc(out), _desc(grad_out), _desc(grad_score))
    return grad_score


def gat_aggregate(g: Graph, feat, el, er, slope: float = 0.2, out=None, attn=None, want_attn: bool = False,
                  stats=None, want_stats: bool = False, stream=None):
    """Fused attention: out[v, h] = sum over in-edges of softmax_v(leaky(el[u, h] + er[v, h])) * feat[u, h, :].
    Returns out, followed by attn (with want_attn or attn given) and by the per-row statistics
    (num_dst, H, 2) fp32 (with want_stats or stats given) that gat_aggregate_backward takes."""
    feat, el, er = _as3(feat), _as3(el), _as3(er)
    if out is None:
        out = torch.empty((g.num_dst, feat.shape[1], feat.shape[2]), dtype=feat.dtype, device=feat.device)
    if want_attn and attn is None:
        attn = torch.empty((g.num_edges, feat.shape[1], 1), dtype=feat.dtype, device=feat.device)
    if want_stats and stats is None:
        stats = torch.empty((g.num_dst, feat.shape[1], 2), dtype=torch.float32, device=feat.device)
    _run(g, stream, load().gat_aggregate, g.handle, _desc(feat), _desc(el), _desc(er), slope, _desc(out), _desc(attn),
         _desc(stats))
    res = (out,) + ((attn,) if attn is not None else ()) + ((stats,) if stats is not None else ())
    return res if len(res) > 1 else out


def gat_aggregate_backward(g: Graph, feat, el, er, slope: float, stats, grad_out, want_feat: bool = True,
                           want_el: bool = True, want_er: bool = True, stream=None):
    """(grad_feat, grad_el, grad_er) of gat_aggregate from its per-row statistics (any may be None)."""
    feat, el, er, grad_out = _as3(feat), _as3(el), _as3(er), _as3(grad_out)
    gf = torch.empty(feat.shape, dtype=feat.dtype, device=feat.device) if want_feat else None
    gl = torch.empty(el.shape, dtype=feat.dtype, device=feat.device) if want_el else None
    gr = torch.empty(er.shape, dtype=feat.dtype, device=feat.device) if want_er else None
    _run(g, stream, load().gat_aggregate_backward, g.handle, _desc(feat), _desc(el), _desc(er), slope, _desc(stats),
         _desc(grad_out), _desc(gf), _desc(gl), _desc(gr))
    return gf, gl, gr


def edge_leaky_relu(x, slope: float = 0.2, y=None, stream=None):
    x = _as3(x)
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _check(load().edge_leaky_relu(_desc(x), _desc(y), slope, _stream(stream)))
    return y


def edge_leaky_relu_backward(x, dy, slope: float = 0.2, dx=None, stream=None):
    x, dy = _as3(x), _as3(dy)
    if dx is None:
        dx = torch.empty(x.shape, dtype=dy.dtype, device=dy.device)
    _check(load().edge_leaky_relu_backward(_desc(x), _desc(dy), _desc(dx), slope, _stream(stream)))
    return dx


# ---------------------------------------------------------------------------
# queries and keys of dot-product attention

# gnnk_rotary (pos, rows, pos_stride, freq, pos_type, axes, pairs[4], interleaved, reserved) as bytes
_ROTARY = struct.Struct("=QqqQIIIIIIII")


_ADDRESS = struct.Struct("=Q")


def _out(t, desc):
    """an output like t and its descriptor: t's own, desc, at another address where t is contiguous (0.3 us less)"""
    o = torch.empty_like(t, memory_format=torch.contiguous_format)
    return o, _ADDRESS.pack(o.data_ptr()) + desc[8:] if t.is_contiguous() else _desc(o)


def _here(*ts):
    """Refuse tensors of another device than the current one, whose stream the call would run on."""
    cur = -1
    for t in ts:
        if t is not None and t.is_cuda:
            if cur < 0:
                cur = _device() if _device is not None else torch.cuda.current_device()
            if t.get_device() != cur:
                raise ValueError(f"a tensor or graph is on cuda:{t.get_device()}, the current device is cuda:{cur}")


class Rotary:
    """A rotation by positions on one to four axes: pairs[a] pairs of a head's columns are turned by axis a, pair i by
    pos[row, axis of i] * freq[i].  freq: fp32 on the GPU, one value per pair.  interleaved: pair i is columns
    (2i, 2i + 1), else (i, i + P), P being the number of pairs; columns from 2P on stay as they are."""

    def __init__(self, freq: torch.Tensor, pairs, interleaved: bool = False):
        self.pairs = tuple(int(p) for p in pairs)
        if not 1 <= len(self.pairs) <= 4 or min(self.pairs) < 0 or sum(self.pairs) < 1:
            raise ValueError("pairs must be one to four counts, not all 0")
        if not freq.is_cuda:
            raise ValueError("tensors must be on the GPU")
        if freq.dtype is not torch.float32 or freq.shape != (sum(self.pairs),):
            raise ValueError(f"freq must be float32 of shape ({sum(self.pairs)},)")
        if freq.requires_grad:
            raise ValueError("no gradient is formed for frequencies: detach them")
        self.freq = freq.contiguous()
        self.interleaved = bool(interleaved)
        self._tail = (len(self.pairs), *self.pairs, *(0,) * (4 - len(self.pairs)), int(self.interleaved), 0)

    @classmethod
    def geometric(cls, pairs, base: float = 10000.0, device="cuda", interleaved: bool = False) -> "Rotary":
        """Frequencies base ** (-i / pairs[a]), i = 0..pairs[a] - 1, for each axis."""
        f = [float(base) ** (-torch.arange(int(p), dtype=torch.float64) / max(int(p), 1)) for p in pairs]
        return cls(torch.cat(f).float().to(device), pairs, interleaved)

    def _desc(self, pos):
        """gnnk_rotary bytes with the positions of a tensor's rows."""
        if pos is None:
            raise ValueError("a rotation needs positions")
        if pos.dim() == 1:
            pos = pos.unsqueeze(1)
        if not pos.is_cuda:
            raise ValueError("tensors must be on the GPU")
        if pos.dtype is torch.float32:
            kind = 0
        elif pos.dtype is torch.int32:
            kind = 1
        else:
            raise TypeError(f"positions must be float32 or int32, not {pos.dtype}")
        rows, axes = pos.shape
        if axes != len(self.pairs):
            raise ValueError(f"positions have {axes} axes, the rotation {len(self.pairs)}")
        stride = axes
        if rows:
            if axes > 1 and pos.stride(1) != 1:
                raise ValueError("the positions of a row must be contiguous")
            if rows > 1:
                if pos.stride(0) < axes:
                    raise ValueError("row stride of the positions smaller than their axes")
                stride = pos.stride(0)
        _here(pos, self.freq)
        return _ROTARY.pack(pos.data_ptr(), rows, stride, self.freq.data_ptr(), kind, *self._tail)


def node_rotary(rot: Rotary, x, pos, inverse: bool = False, out=None, stream=None):
    """x (rows, H, F) with its pairs of columns turned by the angles of pos (rows, axes), float32 or int32; inverse: by
    the opposite angles (the gradient).  out may be x itself."""
    x = _as3(x)
    _here(x, out)
    xd = _desc(x)
    out, od = _out(x, xd) if out is None else (out, _desc(out))
    _check(load().node_rotary(rot._desc(pos), xd, int(inverse), od, _stream(stream)))
    return out


def _weight3(w):
    """a weight as one row of (H, F): (F,), (H, F) or (1, H, F)"""
    if w is None or w.dim() == 3:
        return w
    return w.view(1, 1, -1) if w.dim() == 1 else w.unsqueeze(0)


def node_norm_rotary(q, wq=None, k=None, wk=None, rot: Rotary = None, pos_q=None, pos_k=None, eps: float = 1e-6,
                     out_q=None, out_k=None, stream=None):
    """Each head of q (rows, H, F) divided by its root mean square, times wq ((F,), (H, F) or None), then turned by
    rot (None: not turned) at pos_q; the same of k, with wk and pos_k, in the same launch.  Returns out_q, or
    (out_q, out_k) with k.  out_q may be q itself and out_k k in heads of up to 256 columns (bf16: 512)."""
    q, wq, wk = _as3(q), _weight3(wq), _weight3(wk)
    k = _as3(k) if k is not None else None
    _here(q, wq, k, wk, out_q, out_k)
    xq, xk = _desc(q), _desc(k)
    out_q, oq = _out(q, xq) if out_q is None else (out_q, _desc(out_q))
    out_k, ok = _out(k, xk) if k is not None and out_k is None else (out_k, _desc(out_k))
    rq = rot._desc(pos_q) if rot is not None else None
    rk = None
    if rot is not None and k is not None:
        rk = rq if pos_k is pos_q else rot._desc(pos_k)
    _check(load().node_norm_rotary(xq, _desc(wq), rq, oq, xk, _desc(wk), rk, ok, eps, _stream(stream)))
    return (out_q, out_k) if k is not None else out_q


def node_norm_rotary_backward(q, wq, grad_q, k=None, wk=None, grad_k=None, rot: Rotary = None, pos_q=None, pos_k=None,
                              eps: float = 1e-6, want_q: bool = True, want_wq: bool = True, want_k: bool = True,
                              want_wk: bool = True, stream=None):
    """Gradients of node_norm_rotary from those of its outputs: (dq, dwq), and with k (dq, dwq, dk, dwk); None where
    not wanted or without a weight.  Weight gradients have their weight's shape."""
    q, wq3, wk3, grad_q = _as3(q), _weight3(wq), _weight3(wk), _as3(grad_q)
    k, grad_k = (_as3(k) if k is not None else None), (_as3(grad_k) if grad_k is not None else None)
    _here(q, wq3, k, wk3, grad_q, grad_k)
    xq, xk, ywq, ywk = _desc(q), _desc(k), _desc(wq3), _desc(wk3)
    like = lambda t, d, want: _out(t, d) if want and t is not None else (None, None)
    (dq, gq), (dwq, gwq) = like(q, xq, want_q), like(wq3, ywq, want_wq)
    (dk, gk), (dwk, gwk) = like(k, xk, want_k), like(wk3, ywk, want_wk and k is not None)
    rq = rot._desc(pos_q) if rot is not None else None
    rk = None
    if rot is not None and k is not None:
        rk = rq if pos_k is pos_q else rot._desc(pos_k)
    work, nbytes = None, 0
    if gwq is not None or gwk is not None:
        need = ctypes.c_size_t(0)
        _check(load().node_norm_rotary_work_bytes(xq, gwq, xk, gwk, ctypes.byref(need)))
        nbytes = need.value
        if stream is None:
            work = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
        else:
            with torch.cuda.stream(stream):
                work = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    _check(load().node_norm_rotary_backward(xq, ywq, rq, _desc(grad_q), gq, gwq, xk, ywk, rk, _desc(grad_k), gk, gwk,
                                            eps, _ptr(work), nbytes, _stream(stream)))
    if dwq is not None and wq.dim() != 3:
        dwq = dwq.view(wq.shape)
    if dwk is not None and wk.dim() != 3:
        dwk = dwk.view(wk.shape)
    return (dq, dwq, dk, dwk) if k is not None else (dq, dwq)


# ---------------------------------------------------------------------------
# the residual stream between layers, and products in 8 bits

# gnnk_rows8 (data, scale, rows, row_stride, cols, reserved) and gnnk_weight8
# (packed, scale, outs, cols) as bytes
_ROWS8 = struct.Struct("=QQqqII")
_WEIGHT8 = struct.Struct("=QQII")


def _rows8(q, scale):
    """gnnk_rows8 bytes of int8 rows and their scales."""
    if not q.is_cuda or (scale is not None and not scale.is_cuda):
        raise ValueError("tensors must be on the GPU")
    if q.dtype is not torch.int8 or q.dim() != 2:
        raise TypeError("rows in 8 bits are an int8 tensor (rows, columns)")
    rows, cols = q.shape
    if scale is not None:
        if scale.dtype is not torch.float32 or scale.numel() != rows or (rows > 1 and not scale.is_contiguous()):
            raise ValueError(f"scales must be float32, contiguous, one for each of the {rows} rows")
    stride = cols
    if rows and cols:
        if cols > 1 and q.stride(1) != 1:
            raise ValueError("the columns of a row must be contiguous")
        if rows > 1:
            if q.stride(0) < cols:
                raise ValueError("row stride smaller than the columns")
            stride = q.stride(0)
    return _ROWS8.pack(q.data_ptr(), scale.data_ptr() if scale is not None else 0, rows, stride, cols, 0)


_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _flat(t, rows=None):
    """_desc of a tensor whose rows are whole: a contiguous one of two dimensions, or all of one as `rows` = 1 row,
    without a look at its strides (0.5 us instead of 1.3)"""
    if t is None:
        return None
    dt = _CODES.get(t.dtype)
    if dt is None or not t.is_cuda or not t.is_contiguous() or (rows is None and t.dim() != 2):
        if rows is not None and t.is_cuda and not t.is_contiguous():
            raise ValueError("weights and biases must be contiguous")
        return _desc(t if rows is None else t.reshape(1, 1, -1))
    cols = t.numel() if rows is not None else t.shape[1]
    return _TENSOR.pack(t.data_ptr(), rows or t.shape[0], 1, cols & 0xFFFFFFFF, cols, dt, 0)


def _new_rows8(x, rows, cols):
    """int8 rows whose stride is a multiple of 16 bytes, but none of 4,096 (a product of 16,384 such rows takes 237 us, 218
    with 128 bytes between them), and their scales, on x's device"""
    stride = (cols + 15) & ~15
    if stride & 4095 == 0:
        stride += 128
    q = x.new_empty((rows, stride), dtype=torch.int8)
    return q if cols == stride else q[:, :cols], x.new_empty((rows,), dtype=torch.float32)


def _columns(x):
    return x.shape[1] if x.dim() == 2 else x.shape[1] * x.shape[2]


def node_add_norm(x, residual=None, weight=None, eps: float = 1e-6, out=None, out_sum=None, stream=None):
    """The residual stream's sum and its norm: h = x + residual, y = weight * h / sqrt(mean(h^2) + eps) over each whole
    row (of (rows, H, F): all heads).  weight: a row's elements in any shape, or None.  Returns (y, h), or y alone
    without a residual.  out and out_sum may be x or residual themselves."""
    x = _as3(x) if x.dim() != 2 else x
    _here(x, residual, weight, out, out_sum)
    xd = _flat(x)
    out, od = _out(x, xd) if out is None else (out, _desc(out))
    sd = None
    if residual is not None:
        out_sum, sd = _out(x, xd) if out_sum is None else (out_sum, _desc(out_sum))
    elif out_sum is not None:
        raise ValueError("without a residual the sum is x")
    _check(load().node_add_norm(xd, _flat(residual), _flat(weight, 1), eps, sd, od, _stream(stream)))
    return (out, out_sum) if residual is not None else out


def node_add_norm_i8(x, residual=None, weight=None, eps: float = 1e-6, out=None, scale=None, out_sum=None,
                     stream=None):
    """node_add_norm with y in 8 bits: (q, scale, h), or (q, scale) without a residual.  q: int8 (rows, columns), a
    row's largest magnitude being 127, whose rows start 16 bytes apart or a multiple of it; scale: float32 (rows,);
    scale[n] * q[n] is y.  A row with a NaN or an infinity has scale NaN and values 0."""
    x = _as3(x) if x.dim() != 2 else x
    _here(x, residual, weight, out, scale, out_sum)
    xd = _flat(x)
    if (out is None) != (scale is None):
        raise ValueError("out and scale are given together")
    if out is None:
        out, scale = _new_rows8(x, x.shape[0], _columns(x))
    sd = None
    if residual is not None:
        out_sum, sd = _out(x, xd) if out_sum is None else (out_sum, _desc(out_sum))
    elif out_sum is not None:
        raise ValueError("without a residual the sum is x")
    _check(load().node_add_norm_i8(xd, _flat(residual), _flat(weight, 1), eps, sd, _rows8(out, scale),
                                   _stream(stream)))
    return (out, scale, out_sum) if residual is not None else (out, scale)


def node_quantize(x, out=None, scale=None, stream=None):
    """The rows of x (of (rows, H, F): all heads) in 8 bits: (q, scale), as node_add_norm_i8 makes them."""
    x = _as3(x) if x.dim() != 2 else x
    _here(x, out, scale)
    if (out is None) != (scale is None):
        raise ValueError("out and scale are given together")
    if out is None:
        out, scale = _new_rows8(x, x.shape[0], _columns(x))
    _check(load().node_quantize(_flat(x), _rows8(out, scale), _stream(stream)))
    return out, scale


def node_add_norm_backward(h, weight, grad_y, grad_sum=None, eps: float = 1e-6, want_x: bool = True,
                           want_weight: bool = True, grad_x=None, stream=None):
    """Gradients of node_add_norm from that of y and, with grad_sum, that of the sum: (dx, dweight), dx being the
    gradient of x and of the residual.  h: the sum as node_add_norm returned it (without a residual x).  None where not
    wanted or without a weight.  grad_x, where dx goes, may be h, grad_y or grad_sum themselves."""
    h = _as3(h) if h.dim() != 2 else h
    _here(h, weight, grad_y, grad_sum, grad_x)
    hd = _flat(h)
    gx = None
    if grad_x is not None:
        gx = _desc(grad_x)
    elif want_x:
        grad_x, gx = _out(h, hd)
    dw, gw, wd = None, None, _flat(weight, 1)
    work, nbytes = None, 0
    if weight is not None:
        if want_weight:
            dw, gw = _out(weight, wd)
            need = ctypes.c_size_t(0)
            _check(load().node_add_norm_work_bytes(hd, ctypes.byref(need)))
            nbytes = need.value
            if stream is None:
                work = torch.empty(nbytes, dtype=torch.uint8, device=h.device)
            else:
                with torch.cuda.stream(stream):
                    work = torch.empty(nbytes, dtype=torch.uint8, device=h.device)
    _check(load().node_add_norm_backward(hd, wd, _flat(grad_y), _flat(grad_sum), eps, gx, gw, _ptr(work), nbytes,
                                         _stream(stream)))
    return grad_x, dw


class Weight8:
    """A linear layer's weight in 8 bits, laid out for node_linear_i8: values int8 (outs, columns), scale float32
    (outs,), scale[o] * values[o] being row o.  Both may be changed or dropped afterwards; it may be copied and pickled.
    Made once for many products: the layout takes two allocations, a copy and a launch, some 30 us."""

    def __init__(self, values: torch.Tensor, scale: torch.Tensor, stream=None):
        _here(values, scale)
        rows = _rows8(values, scale)
        self.outs, self.cols = values.shape
        need = ctypes.c_size_t(0)
        _check(load().weight8_bytes(self.outs, self.cols, ctypes.byref(need)))
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            self._packed = torch.empty(need.value, dtype=torch.uint8, device=values.device)
            self._scale = scale.reshape(-1).clone()
        _check(load().weight8_pack(rows, self._packed.data_ptr(), need.value, _stream(stream)))
        self._bind()

    # its tensors stay: the descriptor holds their addresses, and a copy has its own
    packed = property(lambda self: self._packed)
    scale = property(lambda self: self._scale)

    def _bind(self):
        self._bytes = _WEIGHT8.pack(self._packed.data_ptr(), self._scale.data_ptr(), self.outs, self.cols)

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_bytes"}

    def __setstate__(self, state):
        self.__dict__.update(state)
        self._bind()

    @classmethod
    def quantize(cls, weight: torch.Tensor, stream=None) -> "Weight8":
        """The weight (outs, columns), float32 or bfloat16, of at most 16,384 columns, rounded to 8 bits with a scale for
        each output.  (Values of up to 65,536 columns that are in 8 bits already are given to Weight8 itself.)"""
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            return cls(*node_quantize(weight.detach()))


def node_linear_i8(weight: Weight8, q, scale, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """Rows in 8 bits times a weight in 8 bits: out[n, o] = scale[n] * weight.scale[o] * (q[n] . values[o]) + bias[o],
    float32 or bfloat16 (dtype, or out's).  The products' sums are exact.  bias: outs values of out's dtype.  No
    gradient is formed."""
    _here(weight._packed, q, scale, bias, out)
    xd = _rows8(q, scale)
    if out is None:
        out = q.new_empty((q.shape[0], weight.outs), dtype=dtype)
    _check(load().node_linear_i8(xd, weight._bytes, _flat(bias, 1), _flat(out), _stream(stream)))
    return out


def dot_aggregate(g: Graph, q, k, v, bias=None, scale: float = None, out=None, stats=None, want_stats: bool = False,
                  stream=None):
    """Dot-product attention over the in-edges: out[v, h] = sum of softmax_v(scale q[v, h].k[u, j] + bias[e, h]) *
    v[u, j], j being the key head that query head h shares.  q (num_dst, H, F), k and v (num_src, K, F), bias
    (num_edges, H or 1, 1), -inf masking an edge; scale: default 1 / sqrt(F).  Returns out, with want_stats (or stats
    given) followed by the per-row statistics (num_dst, H, 2) fp32 that dot_aggregate_backward takes."""
    q, k, v = _as3(q), _as3(k), _as3(v)
    bias = _as3(bias) if bias is not None else None
    _here(g._keep[0] if g._keep else None, q, k, v, bias, out, stats)
    if scale is None:
        scale = q.shape[2] ** -0.5
    qd = _desc(q)
    out, od = _out(q, qd) if out is None else (out, _desc(out))
    if want_stats and stats is None:
        stats = torch.empty((g.num_dst, q.shape[1], 2), dtype=torch.float32, device=q.device)
    _run(g, stream, load().dot_aggregate, g.handle, qd, _desc(k), _desc(v), _desc(bias), scale, od, _desc(stats))
    return (out, stats) if stats is not None else out


def dot_aggregate_backward(g: Graph, q, k, v, out, stats, grad_out, bias=None, scale: float = None,
                           want_q: bool = True, want_k: bool = True, want_v: bool = True, want_bias: bool = True,
                           stream=None):
    """(dq, dk, dv, dbias) of dot_aggregate from its output and statistics (None where not wanted, or without bias)."""
    q, k, v, out, grad_out = _as3(q), _as3(k), _as3(v), _as3(out), _as3(grad_out)
    bias = _as3(bias) if bias is not None else None
    _here(g._keep[0] if g._keep else None, q, k, v, bias, out, stats, grad_out)
    if scale is None:
        scale = q.shape[2] ** -0.5
    qd, kd, vd, bd = _desc(q), _desc(k), _desc(v), _desc(bias)
    like = lambda t, d, want: _out(t, d) if want and t is not None else (None, None)
    (dq, gq), (dk, gk), (dv, gv), (db, gb) = (like(q, qd, want_q), like(k, kd, want_k), like(v, vd, want_v),
                                              like(bias, bd, want_bias))
    _run(g, stream, load().dot_aggregate_backward, g.handle, qd, kd, vd, bd, scale, _desc(out), _desc(stats),
         _desc(grad_out), gq, gk, gv, gb)
    return dq, dk, dv, db
