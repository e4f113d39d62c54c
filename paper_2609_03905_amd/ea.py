"""Python binding of libea (the C ABI declared in include/ea.h).

Argument marshalling only: every step of a join-agg or repartition runs in the
HIP kernels of libea.so.  PyTorch provides device memory (uint8 tensors) and
the current HIP stream.  If libea.so has not been built the import of a
compute function raises: there is no fallback path.
"""
from __future__ import annotations

import array
import ctypes
import os
from typing import Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libea.so")

# ---- codes (mirror include/ea.h) ------------------------------------------
OK = 0
ERR_NAMES = {-1: "EA_ERR_ARG", -2: "EA_ERR_DTYPE", -3: "EA_ERR_PARTITION", -4: "EA_ERR_CAPACITY",
             -5: "EA_ERR_SPEC", -6: "EA_ERR_JOIN", -7: "EA_ERR_UNSUPPORTED", -8: "EA_ERR_HIP",
             -9: "EA_ERR_NOPLAN"}
ERR_ARG, ERR_CAPACITY, ERR_NOPLAN = -1, -4, -9
WS_COUNTER_BYTES = 262144  # EA_WS_COUNTER_BYTES: the counter area at the start of a workspace
F32, BF16, F16, E4M3, E5M2 = 0, 1, 2, 3, 4
DTYPES = {"f32": F32, "bf16": BF16, "f16": F16, "e4m3": E4M3, "e5m2": E5M2}
ELEM_SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "e5m2": 1}
JOIN_MUL, JOIN_ADD = 0, 1
OP_RMSNORM, OP_SOFTMAX, OP_ATTENTION, OP_SWIGLU = 16, 17, 18, 19
AGG_NONE, AGG_SUM, AGG_MAX, AGG_LSE = 0, 1, 2, 3
STORE_CACHED, STORE_STREAM = 0, 1  # output store policy (EA_STORE_*)


class EAError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERR_NAMES.get(code, code)}: {msg}")
        self.code = code


class _Params(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_float), ("scale", ctypes.c_float), ("causal", ctypes.c_int32),
                ("store", ctypes.c_int32), ("residual", ctypes.c_void_p), ("gqa_group", ctypes.c_int32),
                ("n_seq", ctypes.c_int32), ("seq_ends", ctypes.c_void_p)]


class _HeadsParams(ctypes.Structure):
    _fields_ = [("d_head", ctypes.c_int32), ("eps", ctypes.c_float), ("rotary", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p)]


class _Paged(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("n_seq", ctypes.c_int32), ("q_start", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("table", ctypes.c_void_p), ("stride", ctypes.c_int32),
                ("n_group", ctypes.c_int32), ("group_start", ctypes.c_void_p), ("group_shared", ctypes.c_void_p)]


class _PageRows(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("stride", ctypes.c_int32), ("q_start", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("table", ctypes.c_void_p), ("slots", ctypes.c_void_p)]


class _Pages(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("stride", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("refs", ctypes.c_void_p), ("out_table", ctypes.c_void_p), ("out_lengths", ctypes.c_void_p),
                ("out_refs", ctypes.c_void_p), ("status", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2609_03905_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        P = ctypes.POINTER
        L.ea_version.restype = ctypes.c_int
        L.ea_last_error.restype = ctypes.c_char_p
        L.ea_dtype_size.argtypes = [i32]
        L.ea_layout_nbytes.argtypes = [i32, P(i64), i32, P(i32), P(i64), P(i64)]
        L.ea_relation_create.argtypes = [i32, P(i64), i32, P(i32), P(i64), vp, i64, P(vp)]
        L.ea_relation_destroy.argtypes = [vp]
        L.ea_relation_set_data.argtypes = [vp, vp, i64]
        L.ea_relation_num_blocks.argtypes = [vp, P(i64)]
        L.ea_relation_nbytes.argtypes = [vp, P(i64)]
        L.ea_relation_block.argtypes = [vp, i64, P(i64), P(i64), P(i64)]
        L.ea_joinagg.argtypes = [ctypes.c_char_p, i32, i32, i32, P(vp), vp, P(_Params), vp, i64, vp]
        L.ea_joinagg_workspace.argtypes = [ctypes.c_char_p, i32, i32, i32, P(vp), vp, P(_Params), P(i64), vp]
        L.ea_repartition_plan.argtypes = [vp, vp, vp]
        L.ea_joinagg_noalloc.argtypes = [ctypes.c_char_p, i32, i32, i32, P(vp), vp, P(_Params), vp]
        L.ea_join_tuples.argtypes = [ctypes.c_char_p, i32, i32, P(vp), vp, P(_Params), vp, i64, vp, i64,
                                     P(i64), P(i64), vp]
        L.ea_repartition.argtypes = [vp, vp, vp]
        L.ea_repartition_ex.argtypes = [vp, vp, i32, vp]
        L.ea_overlay.argtypes = [i32, P(i32), P(i64), P(i32), P(i64), P(i32), P(i64)]
        L.ea_logical_plan.argtypes = [i32, ctypes.c_void_p, i64, P(i32), P(i64)]
        L.ea_exprog_check.argtypes = [ctypes.c_char_p, P(i32), ctypes.c_char_p, i64]
        L.ea_exprog_naive.argtypes = [ctypes.c_char_p, ctypes.c_char_p, i64, P(i64)]
        L.ea_exprog_simulate.argtypes = [ctypes.c_char_p, ctypes.c_double, ctypes.c_double, P(ctypes.c_double)]
        L.ea_exprog_synthesize.argtypes = [ctypes.c_char_p, ctypes.c_double, ctypes.c_double, i32, ctypes.c_uint64,
                                           ctypes.c_char_p, i64, P(i64), P(ctypes.c_double)]
        L.ea_exprog_preamble.argtypes = [i32, P(i32), P(i64), i32, P(i64), P(i32), P(i32), P(i64), i32, P(i64), i32,
                                         i64, ctypes.c_char_p, i64, P(i64)]
        L.ea_heads.argtypes = [vp] * 6 + [P(_HeadsParams), vp]
        L.ea_heads_backward_workspace.argtypes = [i32, P(i64)]
        L.ea_heads_backward.argtypes = [vp] * 9 + [P(_HeadsParams), vp, i64, vp]
        L.ea_attention_paged_workspace.argtypes = [vp, vp, P(_Paged), P(i64)]
        L.ea_attention_paged.argtypes = [vp] * 4 + [P(_Paged), vp, i64, vp]
        L.ea_attention_paged8.argtypes = [vp] * 6 + [P(_Paged), vp, i64, vp]
        L.ea_pages_write.argtypes = [vp] * 6 + [P(_PageRows), vp]
        L.ea_pages_read.argtypes = [vp] * 6 + [P(_PageRows), vp]
        L.ea_pages_workspace.argtypes = [i32, i32, P(i64)]
        L.ea_pages_extend.argtypes = [P(_Pages), vp, vp, vp, i32, vp, i64, vp]
        L.ea_pages_select.argtypes = [i32, P(vp), P(_Pages), vp, vp, i64, vp]
        L.ea_pages_compact.argtypes = [i32, P(vp), P(_Pages), vp, i64, vp]
        L.ea_pages_select_scaled.argtypes = [i32, P(vp), P(vp), P(_Pages), vp, vp, i64, vp]
        L.ea_pages_compact_scaled.argtypes = [i32, P(vp), P(vp), P(_Pages), vp, i64, vp]
        L.ea_plan_cache_size.restype = i64
        L.ea_plan_cache_clear.restype = ctypes.c_int
        _lib = L
    return _lib


def _check(rc: int):
    if rc != OK:
        raise EAError(rc, lib().ea_last_error().decode())


def _arr(ctype, values):
    values = list(values)
    return (ctype * max(len(values), 1))(*values)


def _partition_args(partition):
    nb = _arr(ctypes.c_int32, [len(s) - 1 for s in partition])
    flat = array.array("q")
    for s in partition:
        flat += _points(s)
    if not flat:
        return nb, _arr(ctypes.c_int64, [])
    return nb, (ctypes.c_int64 * len(flat)).from_buffer(flat)


def _points(s) -> array.array:
    """Split points as 64-bit integers (a cache has one a page: tens of thousands)."""
    if not isinstance(s, (list, tuple, range)):
        s = list(s)  # an array reads bytes as they lie, and what it takes of an iterator is gone
    try:
        return array.array("q", s)
    except TypeError:
        return array.array("q", map(int, s))


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_gpu_seen = False  # a GPU was available once (it stays so)


def _stream(stream):
    """The HIP stream handle of ``stream`` (default: torch's current one)."""
    global _gpu_seen
    if stream is None:
        if not _gpu_seen:
            if not torch.cuda.is_available():
                return None  # host-side validation still runs; HIP calls then fail
            _gpu_seen = True
        if _raw_stream is not None:  # the handle alone: torch's Stream object costs half a call
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def version() -> int:
    return int(lib().ea_version())


def layout_nbytes(shape, dtype: str, partition) -> int:
    nb, sp = _partition_args(partition)
    out = ctypes.c_int64(0)
    _check(lib().ea_layout_nbytes(len(shape), _arr(ctypes.c_int64, shape), DTYPES[dtype], nb, sp,
                                  ctypes.byref(out)))
    return int(out.value)


def overlay(part_a, part_b):
    """Per dim, the sorted union of both partitions' split points (Section 5.3)."""
    rank = len(part_a)
    nba, spa = _partition_args(part_a)
    nbb, spb = _partition_args(part_b)
    nbo = (ctypes.c_int32 * rank)()
    spo = (ctypes.c_int64 * sum(len(a) + len(b) for a, b in zip(part_a, part_b)))()
    _check(lib().ea_overlay(rank, nba, spa, nbb, spb, nbo, spo))
    out, k = [], 0
    for d in range(rank):
        out.append([int(spo[k + i]) for i in range(nbo[d] + 1)])
        k += nbo[d] + 1
    return out


class Relation:
    """A tensor relation: a shape, a dtype, a block partition (split points
    per dim) and block-major storage in a torch uint8 device tensor."""

    def __init__(self, shape: Sequence[int], dtype: str, partition, data: torch.Tensor | None = None,
                 device: str | torch.device = "cuda", allocate: bool = True, byte_offset: int = 0):
        self.shape = tuple(int(s) for s in shape)
        self.dtype = dtype
        self.partition = [_points(s).tolist() for s in partition]
        nb, sp = _partition_args(self.partition)
        shp, n = _arr(ctypes.c_int64, self.shape), ctypes.c_int64()
        _check(lib().ea_layout_nbytes(len(self.shape), shp, DTYPES[dtype], nb, sp, ctypes.byref(n)))
        self.nbytes = int(n.value)
        if data is None and allocate:
            data = torch.empty(max(self.nbytes, 1), dtype=torch.uint8, device=device)
        self.data = data
        self._byte_offset = int(byte_offset)
        ptr, cap = None, 0
        if data is not None:
            ptr = data.data_ptr() + self._byte_offset
            cap = data.numel() * data.element_size() - self._byte_offset
        self._device = -1 if data is None else data.get_device()
        h = ctypes.c_void_p()
        _check(lib().ea_relation_create(len(self.shape), shp, DTYPES[dtype], nb, sp,
                                        ctypes.c_void_p(ptr) if ptr else None, cap, ctypes.byref(h)))
        self.handle = h
        self._h = h.value  # the handle as a plain integer

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and _lib is not None:
            _lib.ea_relation_destroy(h)
            self.handle = None

    # -- views ---------------------------------------------------------------
    def view(self, byte_offset: int, shape, dtype: str, partition) -> "Relation":
        """Another relation over this relation's storage, starting
        ``byte_offset`` bytes in (for example a per-head slice)."""
        return Relation(shape, dtype, partition, data=self.data, byte_offset=self._byte_offset + byte_offset)

    def bytes(self) -> torch.Tensor:
        """The relation's storage as a uint8 tensor (a view)."""
        return self.data[self._byte_offset:self._byte_offset + self.nbytes]

    # -- introspection -------------------------------------------------------
    def num_blocks(self) -> int:
        n = ctypes.c_int64()
        _check(lib().ea_relation_num_blocks(self.handle, ctypes.byref(n)))
        return int(n.value)

    def block(self, b: int):
        r = len(self.shape)
        lo, hi, off = (ctypes.c_int64 * r)(), (ctypes.c_int64 * r)(), ctypes.c_int64()
        _check(lib().ea_relation_block(self.handle, b, lo, hi, ctypes.byref(off)))
        return list(lo), list(hi), int(off.value)


def _params(eps=0.0, scale=0.0, causal=False, store=0, residual=None, gqa_group=0, seq_ends=None):
    """ea_params plus the host array it points at (kept alive by the caller)."""
    res = residual.handle.value if residual is not None else None
    if seq_ends is None:
        return _Params(eps, scale, int(causal), int(store), res, int(gqa_group), 0, None), None
    ends = (ctypes.c_int64 * max(1, len(seq_ends)))(*[int(e) for e in seq_ends])
    return _Params(eps, scale, int(causal), int(store), res, int(gqa_group), len(seq_ends),
                   ctypes.cast(ends, ctypes.c_void_p)), ends


_HANDLES = [ctypes.c_void_p * max(n, 1) for n in range(9)]  # array types of the usual input counts


def _handles(inputs):
    n = len(inputs)
    return (_HANDLES[n] if n < len(_HANDLES) else ctypes.c_void_p * n)(*[r._h for r in inputs])


def new_workspace(nbytes: int, device=None) -> torch.Tensor:
    """A zeroed device buffer usable as a join-agg workspace of ``nbytes``
    (the counter area must start zeroed; every call leaves it zeroed)."""
    return torch.zeros(max(int(nbytes), 1), dtype=torch.uint8, device=device or "cuda")


_WS = {}  # (device, stream handle) -> workspace tensor of the calls on that stream
_WS_RETIRED = []  # outgrown workspaces: kernels queued earlier may still use them


def _stream_workspace(nbytes: int, stream) -> torch.Tensor:
    """The binding's workspace for calls on ``stream``: calls on one stream run
    in order, so they share one buffer, grown (zeroed) when a plan needs more."""
    dev = torch.cuda.current_device()
    key = (dev, stream or 0)
    buf = _WS.get(key)
    if buf is None or buf.numel() < nbytes:
        if buf is not None:
            _WS_RETIRED.append(buf)
        buf = new_workspace(max(nbytes, 2 * buf.numel() if buf is not None else nbytes), device=dev)
        torch.cuda.synchronize(dev)  # zeroed before any stream uses it
        _WS[key] = buf
    return buf


def joinagg_workspace(spec: str, join_op: int, agg_op: int, inputs: Sequence[Relation], out: Relation, *,
                      eps: float = 0.0, scale: float = 0.0, causal: bool = False, residual: Relation | None = None,
                      store: int = 0, gqa_group: int = 0, seq_ends=None, stream=None) -> int:
    """Plan a join-agg configuration (first call: allocate the plan, run the
    GPU join, wait for it) and return the workspace bytes its runs need."""
    handles = _handles(inputs)
    prm, _ends = _params(eps, scale, causal, store, residual, gqa_group, seq_ends)
    n = ctypes.c_int64()
    _check(lib().ea_joinagg_workspace(spec.encode(), join_op, agg_op, len(inputs), handles, out.handle,
                                      ctypes.byref(prm), ctypes.byref(n), _stream(stream)))
    return int(n.value)


def joinagg(spec: str, join_op: int, agg_op: int, inputs: Sequence[Relation], out: Relation, *,
            eps: float = 0.0, scale: float = 0.0, causal: bool = False, residual: Relation | None = None,
            store: int = 0, gqa_group: int = 0, seq_ends=None, stream=None,
            workspace: torch.Tensor | None = None) -> None:
    """Run one GPU's share of a join-agg: join the input relations' blocks,
    run the per-tuple kernel, aggregate by output key, store into ``out``.
    ``store``: STORE_CACHED (default) or STORE_STREAM (non-temporal output
    stores, for an output nothing reads soon).  Attention: ``gqa_group``
    query heads per key-value head, ``seq_ends`` the ends of packed
    sequences.  The configuration is planned on first use (see
    joinagg_workspace).  ``workspace``: a device buffer from new_workspace
    for key-split partials; by default one buffer per stream, held by the
    binding."""
    handles = _handles(inputs)
    prm, _ends = _params(eps, scale, causal, store, residual, gqa_group, seq_ends)
    s = _stream(stream)
    spec_b, prm_p, n_in = spec.encode(), ctypes.byref(prm), len(inputs)
    # A planned configuration whose workspace fits runs at once.  Where the
    # plan is missing, or the workspace (EA_ERR_ARG without one) or its size,
    # all of which are found before anything is enqueued, it is planned, the
    # workspace grown, and the call made again; any other error is raised: after
    # EA_ERR_HIP the kernels may be queued already.
    buf = workspace
    if buf is None and _WS:
        buf = _WS.get((torch.cuda.current_device(), s or 0))
    if buf is None:
        ws, nbytes = None, 0
    else:
        ws, nbytes = buf.data_ptr(), buf.numel() * buf.element_size()
    rc = lib().ea_joinagg(spec_b, join_op, agg_op, n_in, handles, out._h, prm_p, ws, nbytes, s)
    if rc == OK:
        return
    if rc not in (ERR_NOPLAN, ERR_CAPACITY) and not (rc == ERR_ARG and ws is None):
        _check(rc)
    need = ctypes.c_int64()
    _check(lib().ea_joinagg_workspace(spec_b, join_op, agg_op, n_in, handles, out._h, prm_p, ctypes.byref(need), s))
    ws, nbytes = None, 0
    if need.value:
        buf = workspace if workspace is not None else _stream_workspace(need.value, s)
        ws, nbytes = buf.data_ptr(), buf.numel() * buf.element_size()
    _check(lib().ea_joinagg(spec_b, join_op, agg_op, n_in, handles, out._h, prm_p, ws, nbytes, s))


def joinagg_noalloc(spec: str, join_op: int, agg_op: int, inputs: Sequence[Relation], out: Relation, *,
                    eps: float = 0.0, scale: float = 0.0, causal: bool = False, residual: Relation | None = None,
                    store: int = 0, gqa_group: int = 0, seq_ends=None, stream=None) -> None:
    """ea_joinagg_noalloc: run a join-agg planned earlier (joinagg_workspace)
    with the library's own per-device workspace array; allocates nothing.
    Calls that may overlap in time on one GPU race on that array."""
    handles = _handles(inputs)
    prm, _ends = _params(eps, scale, causal, store, residual, gqa_group, seq_ends)
    _check(lib().ea_joinagg_noalloc(spec.encode(), join_op, agg_op, len(inputs), handles, out.handle,
                                    ctypes.byref(prm), _stream(stream)))


def repartition_plan(src: Relation, dst: Relation, stream=None) -> None:
    """Plan the repartition of ``src``'s partition into ``dst``'s (first call:
    build and upload its overlay boxes, wait)."""
    _check(lib().ea_repartition_plan(src.handle, dst.handle, _stream(stream)))


def repartition(src: Relation, dst: Relation, stream=None, *, store: int = 0) -> None:
    """Write ``src``'s dense tensor into ``dst`` under ``dst``'s partition
    (``store`` as for joinagg); planned on first use."""
    s = _stream(stream)
    rc = lib().ea_repartition_ex(src._h, dst._h, int(store), s)
    if rc == OK:
        return
    if rc != ERR_NOPLAN:
        _check(rc)
    _check(lib().ea_repartition_plan(src._h, dst._h, s))
    _check(lib().ea_repartition_ex(src._h, dst._h, int(store), s))


def join_tuples(spec: str, join_op: int, inputs: Sequence[Relation], out: Relation, *, causal: bool = False,
                scale: float = 1.0, eps: float = 1e-6, gqa_group: int = 0, seq_ends=None, stream=None):
    """The GPU-built tuple table and CSR group offsets of a join (synchronous)."""
    handles = _handles(inputs)
    prm, _ends = _params(eps, scale, causal, 0, None, gqa_group, seq_ends)
    n_t, n_g = ctypes.c_int64(), ctypes.c_int64()
    dev = out.data.device if out.data is not None else torch.device("cuda")
    # first call sizes the tables (it fails with EA_ERR_CAPACITY but reports the counts)
    rc = lib().ea_join_tuples(spec.encode(), join_op, len(inputs), handles, out.handle, ctypes.byref(prm), None, 0,
                              None, 0, ctypes.byref(n_t), ctypes.byref(n_g), _stream(stream))
    if rc not in (OK, -1, -4):
        _check(rc)
    tuples = torch.zeros((max(n_t.value, 1), len(inputs) + 1), dtype=torch.int32, device=dev)
    goff = torch.zeros(n_g.value + 1, dtype=torch.int64, device=dev)
    _check(lib().ea_join_tuples(spec.encode(), join_op, len(inputs), handles, out.handle, ctypes.byref(prm),
                                ctypes.c_void_p(tuples.data_ptr()), tuples.shape[0], ctypes.c_void_p(goff.data_ptr()),
                                goff.numel(), ctypes.byref(n_t), ctypes.byref(n_g), _stream(stream)))
    return tuples[:n_t.value], goff


# ---- decoding: head rows, attention over a paged cache, the page table -------
PAGES_OK, PAGES_NONE_FREE, PAGES_TOO_LONG = 0, 1, 2  # status[0] of the page calls (EA_PAGES_*)
PAGED_MAX_SEQ = 2048  # EA_PAGED_MAX_SEQ


_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device_array(t, name: str, shape, dtype=torch.int32, optional: bool = False):
    """The address of a small device array, checked: type, shape (None: any
    extent), rows without gaps, on the current device."""
    if t is None and optional:
        return None
    # the usual case in five cheap questions; what is wrong is found below
    if isinstance(t, torch.Tensor) and t.dtype is dtype and 0 <= t.get_device() == _get_device() and t.is_contiguous() \
            and (t.shape == shape or len(t.shape) == len(shape) == 1 and shape[0] is None):
        return t.data_ptr()
    if t is None:
        raise EAError(ERR_ARG, f"{name} is missing")
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        raise EAError(ERR_ARG, f"{name} is no {dtype} tensor")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise EAError(ERR_ARG, f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous():
        raise EAError(ERR_ARG, f"{name} is not contiguous")
    raise EAError(ERR_ARG, f"{name} is on {t.device}, not on the current GPU")


def _on_device(*rels):
    """Relations whose data torch holds lie on the current device."""
    dev = None
    for r in rels:
        if r is not None and r.data is not None:
            if dev is None:
                dev = _get_device() if r._device >= 0 else -2
            if r._device != dev:
                raise EAError(ERR_ARG, f"a relation is on {r.data.device}, not on the current GPU")


def _h(r):
    return None if r is None else r._h


def _workspace(need: int, workspace, stream):
    """Address and size of a call's workspace: the caller's, or the stream's."""
    if need == 0:
        return None, 0
    if workspace is None:
        workspace = _stream_workspace(need, stream)
    elif not 0 <= workspace.get_device() == _get_device() or not workspace.is_contiguous():
        raise EAError(ERR_ARG, f"the workspace is on {workspace.device}, not on the current GPU, or has gaps")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _heads_params(rows, d_head, eps, inv_freq, interleaved, positions, slots):
    freq = _device_array(inv_freq, "inv_freq", (None,), torch.float32, optional=True)
    return _HeadsParams(int(d_head), float(eps), 2 * inv_freq.numel() if freq else 0, int(interleaved), freq,
                        _device_array(positions, "positions", (rows,), optional=True),
                        _device_array(slots, "slots", (rows,), optional=True))


def heads(qkv: Relation, q: Relation, k: Relation, v: Relation, *, d_head: int, wq: Relation | None = None,
          wk: Relation | None = None, eps: float = 0.0, inv_freq: torch.Tensor | None = None,
          interleaved: bool = False, positions: torch.Tensor | None = None, slots: torch.Tensor | None = None,
          stream=None) -> None:
    """The head rows of a QKV activation [T, (Hq + 2 Hkv) d_head] to where
    attention reads them: queries and keys normed with ``wq`` and ``wk`` (None:
    not), their first 2 * len(inv_freq) elements rotated by positions[t] *
    inv_freq (``interleaved``: pairs of neighbours, else of halves; positions
    None: the row's index), values moved along.  ``q``, ``k``, ``v``:
    token-major [T, H d_head] or head-major [.., H, T, d_head]; with ``slots``
    k and v are the pages [pages, Hkv, page_size, d_head] of a cache and row t
    goes to slot slots[t] (-1: to none)."""
    _on_device(qkv, q, k, v, wq, wk)
    prm = _heads_params(qkv.shape[0], d_head, eps, inv_freq, interleaved, positions, slots)
    _check(lib().ea_heads(qkv._h, _h(wq), _h(wk), q._h, k._h, v._h, ctypes.byref(prm), _stream(stream)))


def heads_backward(qkv: Relation, dq: Relation, dk: Relation, dv: Relation, dqkv: Relation, *, d_head: int,
                   wq: Relation | None = None, wk: Relation | None = None, dwq: Relation | None = None,
                   dwk: Relation | None = None, eps: float = 0.0, inv_freq: torch.Tensor | None = None,
                   interleaved: bool = False, positions: torch.Tensor | None = None, stream=None,
                   workspace: torch.Tensor | None = None) -> None:
    """The gradient of ``heads`` (without slots): ``dqkv`` in qkv's layout and,
    where wanted, the norm weights' ``dwq`` and ``dwk`` ([d_head])."""
    _on_device(qkv, dq, dk, dv, dqkv, wq, wk, dwq, dwk)
    prm = _heads_params(qkv.shape[0], d_head, eps, inv_freq, interleaved, positions, None)
    s = _stream(stream)
    ws, n = None, 0
    if dwq is not None or dwk is not None:
        need = ctypes.c_int64()
        _check(lib().ea_heads_backward_workspace(int(d_head), ctypes.byref(need)))
        ws, n = _workspace(need.value, workspace, s)
    _check(lib().ea_heads_backward(qkv._h, _h(wq), _h(wk), dq._h, dk._h, dv._h, dqkv._h, _h(dwq), _h(dwk),
                                   ctypes.byref(prm), ws, n, s))


def _paged(scale, table, lengths, q_start, group_start, group_shared):
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise EAError(ERR_ARG, "table is no [sequences, pages] tensor")
    n, stride = table.shape
    if (group_start is None) != (group_shared is None):
        raise EAError(ERR_ARG, "group_start and group_shared: both or neither")
    n_group = 0 if group_shared is None else group_shared.numel()
    return _Paged(float(scale), n, _device_array(q_start, "q_start", (n + 1,), optional=True),
                  _device_array(lengths, "lengths", (n,)), _device_array(table, "table", (n, stride)), stride, n_group,
                  _device_array(group_start, "group_start", (n_group + 1,), optional=True),
                  _device_array(group_shared, "group_shared", (n_group,), optional=True))


def attention_paged_workspace(q: Relation, k: Relation, n_seq: int, n_group: int = 0) -> int:
    """Workspace bytes of attention_paged for these operands and counts."""
    n = ctypes.c_int64()
    b = _Paged(1.0, int(n_seq), None, None, None, 1, int(n_group), None, None)
    _check(lib().ea_attention_paged_workspace(q._h, k._h, ctypes.byref(b), ctypes.byref(n)))
    return int(n.value)


def attention_paged(q: Relation, k: Relation, v: Relation, out: Relation, *, scale: float, table: torch.Tensor,
                    lengths: torch.Tensor, q_start: torch.Tensor | None = None,
                    group_start: torch.Tensor | None = None, group_shared: torch.Tensor | None = None,
                    k_scale: Relation | None = None, v_scale: Relation | None = None, stream=None,
                    workspace: torch.Tensor | None = None) -> None:
    """Attention of each sequence's newest tokens over a paged cache: ``k`` and
    ``v`` [pages, Hkv, page_size, d], one block a page; sequence s has
    lengths[s] keys in the pages table[s]; its query rows are q_start[s] ..
    q_start[s + 1] - 1 of ``q`` (None: row s), the last of which sees all keys
    and each one before it one less.  Groups of sequences group_start[g] ..
    group_start[g + 1] - 1 share their first group_shared[g] keys, which are
    read once.  The arrays are read when the kernels run.  A cache in 8 bits
    ("e4m3", "e5m2", see pages_write) comes with its scales."""
    _on_device(q, k, v, out, k_scale, v_scale)
    if (k_scale is None) != (v_scale is None):
        raise EAError(ERR_ARG, "k_scale and v_scale: both or neither")
    b = _paged(scale, table, lengths, q_start, group_start, group_shared)
    s = _stream(stream)
    need = ctypes.c_int64()
    _check(lib().ea_attention_paged_workspace(q._h, k._h, ctypes.byref(b), ctypes.byref(need)))
    ws, n = _workspace(need.value, workspace, s)
    if k_scale is None:
        _check(lib().ea_attention_paged(q._h, k._h, v._h, out._h, ctypes.byref(b), ws, n, s))
    else:
        _check(lib().ea_attention_paged8(q._h, k._h, v._h, k_scale._h, v_scale._h, out._h, ctypes.byref(b), ws, n, s))


def _page_rows(x, table, lengths, q_start, slots):
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise EAError(ERR_ARG, "table is no [sequences, pages] tensor")
    n, stride = table.shape
    return _PageRows(n, stride, _device_array(q_start, "q_start", (n + 1,), optional=True),
                     _device_array(lengths, "lengths", (n,)), _device_array(table, "table", (n, stride)),
                     _device_array(slots, "slots", x.shape[-2:][:1], optional=True))


def pages_write(xk: Relation, xv: Relation, k: Relation, v: Relation, *, k_scale: Relation, v_scale: Relation,
                table: torch.Tensor, lengths: torch.Tensor, q_start: torch.Tensor | None = None,
                slots: torch.Tensor | None = None, stream=None) -> None:
    """Rows quantised into a cache in 8 bits.  Rows q_start[s] .. q_start[s + 1]
    - 1 (None: row s) of ``xk`` and ``xv`` ([T, Hkv d] or [.., Hkv, T, d]) are
    the last of sequence s's lengths[s] keys, which lie in the pages table[s] of
    ``k`` and ``v``: codes [pages, Hkv, page_size, d], "e4m3" or "e5m2", one
    block a page.  Every head and block of page_size / n rows has a scale, a
    power of two, in ``k_scale`` and ``v_scale`` ("f32" [pages, Hkv, n]): the
    least under which the largest new element has a code, or the one that the
    block has from earlier rows, if that is larger; where it grows those rows are
    rounded again.  A block whose first row is written is begun anew.  ``slots``
    [T]: the rows' slots from pages_extend; a sequence whose first row's is
    negative gets none (that call was not served).  The arrays are read when the
    kernel runs."""
    _on_device(xk, xv, k, v, k_scale, v_scale)
    rows = _page_rows(xk, table, lengths, q_start, slots)
    _check(lib().ea_pages_write(xk._h, xv._h, k._h, v._h, k_scale._h, v_scale._h, ctypes.byref(rows), _stream(stream)))


def pages_read(k: Relation, v: Relation, xk: Relation, xv: Relation, *, k_scale: Relation, v_scale: Relation,
               table: torch.Tensor, lengths: torch.Tensor, q_start: torch.Tensor | None = None,
               slots: torch.Tensor | None = None, stream=None) -> None:
    """The rows that pages_write puts into a cache, read back into ``xk`` and
    ``xv``: code times scale, rounded once (zeros where a row has no key)."""
    _on_device(xk, xv, k, v, k_scale, v_scale)
    rows = _page_rows(xk, table, lengths, q_start, slots)
    _check(lib().ea_pages_read(k._h, v._h, k_scale._h, v_scale._h, xk._h, xv._h, ctypes.byref(rows), _stream(stream)))


def _pages(table, lengths, refs, page_size, out_table, out_lengths, out_refs, status):
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise EAError(ERR_ARG, "table is no [sequences, pages] tensor")
    if not isinstance(refs, torch.Tensor):
        raise EAError(ERR_ARG, "refs is no tensor")
    n, stride = table.shape
    A = _device_array
    return _Pages(n, stride, refs.numel(), int(page_size), A(table, "table", (n, stride)),
                  A(lengths, "lengths", (n,)), A(refs, "refs", (None,)), A(out_table, "out_table", (n, stride)),
                  A(out_lengths, "out_lengths", (n,), optional=True), A(out_refs, "out_refs", (refs.numel(),)),
                  A(status, "status", (2,)))


def pages_extend(table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, add: torch.Tensor, *, page_size: int,
                 status: torch.Tensor, out_lengths: torch.Tensor | None = None, out_refs: torch.Tensor | None = None,
                 slots: torch.Tensor | None = None, positions: torch.Tensor | None = None, stream=None,
                 workspace: torch.Tensor | None = None) -> None:
    """Pages for add[s] more keys of every sequence, lowest free ones first:
    written into ``table``; ``lengths`` and ``refs`` are updated (in place
    unless outputs are given).  ``slots`` and ``positions`` receive the new
    tokens' places, sequence by sequence, -1 and 0 behind them.  status[0]:
    PAGES_OK or why nothing was done; status[1]: free pages left."""
    st = _pages(table, lengths, refs, page_size, table, lengths if out_lengths is None else out_lengths,
                refs if out_refs is None else out_refs, status)
    ps = _device_array(slots, "slots", (None,), optional=True)
    pp = _device_array(positions, "positions", (None if slots is None else slots.numel(),), optional=True)
    n = slots.numel() if ps else positions.numel() if pp else 0
    a = _device_array(add, "add", (table.shape[0],))
    s = _stream(stream)
    ws, nbytes = _pages_workspace(st, workspace, s)
    _check(lib().ea_pages_extend(ctypes.byref(st), a, ps, pp, n, ws, nbytes, s))


def _page_caches(caches, scales):
    caches = list(caches)
    scales = [None] * len(caches) if scales is None else list(scales)
    if len(scales) != len(caches):
        raise EAError(ERR_ARG, f"{len(scales)} scales for {len(caches)} caches")
    _on_device(*caches, *scales)
    given = (ctypes.c_void_p * max(1, len(scales)))(*[_h(r) for r in scales])
    return len(caches), _handles(caches), given, caches[0].shape[-2] if caches else None


def pages_workspace(sequences: int, pages: int) -> int:
    """Workspace bytes of the page table's calls."""
    need = ctypes.c_int64()
    _check(lib().ea_pages_workspace(sequences, pages, ctypes.byref(need)))
    return need.value


def _pages_workspace(st, workspace, s):
    return _workspace(pages_workspace(st.n_seq, st.n_pages), workspace, s)


def pages_select(caches: Sequence[Relation], parent: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                 refs: torch.Tensor, *, out_table: torch.Tensor, out_lengths: torch.Tensor, out_refs: torch.Tensor,
                 status: torch.Tensor, page_size: int | None = None, scales: Sequence[Relation | None] | None = None,
                 stream=None, workspace: torch.Tensor | None = None) -> None:
    """Sequence i of the new state is a copy of sequence parent[i] (-1: empty):
    forks, reorders and frees.  Whole pages are shared; a partly filled last
    page is copied for all children but the first, in every plane of the caches
    ([pages, Hkv, page_size, d] or [planes, pages, Hkv, page_size, d]).
    ``page_size`` is the caches' (needed where there are none).  ``scales``: those
    of caches in 8 bits ([pages, Hkv, n], or [planes, pages, Hkv, n] with one
    block a plane), which move along; None for the others."""
    n, handles, given, ps = _page_caches(caches, scales)
    st = _pages(table, lengths, refs, page_size or ps or 0, out_table, out_lengths, out_refs, status)
    s = _stream(stream)
    ws, nbytes = _pages_workspace(st, workspace, s)
    _check(lib().ea_pages_select_scaled(n, handles, given, ctypes.byref(st),
                                        _device_array(parent, "parent", (table.shape[0],)), ws, nbytes, s))


def pages_compact(caches: Sequence[Relation], table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, *,
                  status: torch.Tensor, out_table: torch.Tensor | None = None, out_refs: torch.Tensor | None = None,
                  page_size: int | None = None, scales: Sequence[Relation | None] | None = None, stream=None,
                  workspace: torch.Tensor | None = None) -> None:
    """Move the used pages to the first places of the cache (the k-th lowest
    one behind them to the k-th lowest hole) and rewrite the table and the
    counts, in place unless outputs are given (``scales`` as for pages_select)."""
    n, handles, given, ps = _page_caches(caches, scales)
    st = _pages(table, lengths, refs, page_size or ps or 0, table if out_table is None else out_table, None,
                refs if out_refs is None else out_refs, status)
    s = _stream(stream)
    ws, nbytes = _pages_workspace(st, workspace, s)
    _check(lib().ea_pages_compact_scaled(n, handles, given, ctypes.byref(st), ws, nbytes, s))


def plan_cache_size() -> int:
    return int(lib().ea_plan_cache_size())


def plan_cache_clear() -> None:
    _check(lib().ea_plan_cache_clear())


# ---- dense <-> relation through the library's own repartition ---------------
def whole_partition(shape):
    return [[0, int(n)] for n in shape]


def from_dense(dense: torch.Tensor, dtype: str, partition, stream=None) -> Relation:
    """A new relation holding ``dense`` (a contiguous device tensor whose bytes
    are the dtype's storage) under ``partition``; the re-blocking runs on the
    GPU (a one-block relation over the dense tensor, repartitioned)."""
    dense = dense.contiguous()
    raw = dense.view(torch.uint8).reshape(-1)
    src = Relation(dense.shape, dtype, whole_partition(dense.shape), data=raw)
    dst = Relation(dense.shape, dtype, partition, device=dense.device)
    repartition(src, dst, stream)
    return dst


def to_dense(rel: Relation, stream=None) -> torch.Tensor:
    """The relation's dense tensor as raw storage (uint8, then viewed by the
    caller), re-blocked on the GPU."""
    dst = Relation(rel.shape, rel.dtype, whole_partition(rel.shape), device=rel.data.device)
    repartition(rel, dst, stream)
    return dst.bytes()
