"""Python binding of the serving step's cache operators (include/hxkv.h).

One step of an instance's running batch over a paged 8-bit cache:

    step = map_step(held, add, block_table, ring, ring_state, n_tokens, block)   # where its tokens go
    cache.append(k, v, step.runs)                                                # their keys and values, in e4m3
    out = cache.attend(q, block_table, step.row_start, step.kv_len)              # what each token reads

Arguments are torch tensors on the current CUDA device; everything runs in the
library's kernels on torch's current stream (or `stream`), and there is no CPU
fallback.  The tensors must not be freed or reused on another stream before
the kernels are done, as for any asynchronous call.
"""
from __future__ import annotations

import ctypes
import threading
from dataclasses import dataclass
from typing import Optional

import torch

from . import hxsim as H

HX_BF16, HX_F16, HX_F32 = range(3)

_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class hx_kv_map_args(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_rows", "n_tokens", "block_tokens", "n_blocks", "table_width", "n_runs")] + \
               [("table_stride", _i64)] + \
               [(n, _vp) for n in ("held", "add", "block_table", "ring", "ring_state", "row_start", "kv_len", "slots",
                                   "runs", "counts", "ring_state_out")]


class hx_kv_cache(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("k", "v", "k_scale", "v_scale")] + \
               [(n, _i64) for n in ("block_stride", "scale_stride")] + \
               [(n, _i32) for n in ("n_blocks", "n_kv_heads", "block_tokens", "head_dim")]


class hx_kv_new(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("k", "v")] + \
               [(n, _i64) for n in ("k_token_stride", "k_head_stride", "v_token_stride", "v_head_stride")] + \
               [("n_tokens", _i32), ("dtype", _i32), ("runs", _vp), ("n_runs", _i32)]


class hx_kv_query(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("q", "out", "lse")] + \
               [(n, _i64) for n in ("q_token_stride", "q_head_stride", "out_token_stride", "out_head_stride")] + \
               [(n, _i32) for n in ("n_tokens", "n_heads", "dtype", "n_rows")] + \
               [(n, _vp) for n in ("row_start", "kv_len", "block_table")] + \
               [("table_stride", _i64)] + [(n, _i32) for n in ("table_width", "max_q", "causal", "window")] + \
               [("sm_scale", ctypes.c_float), ("workspace", _vp), ("workspace_bytes", _i64), ("status", _vp)]


_lib = None


def load():
    """The library with the prototypes of hxkv.h; raises if it has not been built."""
    global _lib
    if _lib is None:
        lib = H.load()
        lib.hx_kv_max_runs.restype = _i64
        lib.hx_kv_max_runs.argtypes = [_i32, _i32, _i32]
        for name, args in [("hx_kv_map", [_vp, _vp]), ("hx_kv_append", [_vp, _vp, _vp]),
                           ("hx_kv_attend_workspace", [_vp, _vp, _vp]), ("hx_kv_attend", [_vp, _vp, _vp])]:
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = lib
    return _lib


def _fail(msg: str):
    raise H.HxError(H.HX_ERR_INVALID, msg)


def _want(x, name: str, dtypes, ndim: int, device: int):
    """Check one tensor argument: type, dimensions, CUDA device (its index)."""
    if x.dtype not in dtypes:
        _fail(f"{name}: dtype {x.dtype} is not one of {[str(d) for d in dtypes]}")
    if x.dim() != ndim:
        _fail(f"{name} must have {ndim} dimensions")
    if x.get_device() != device or device < 0:
        _fail(f"{name} must be a CUDA tensor" if x.get_device() < 0 else f"{name} is not on cuda:{device}")


def _dense(x, name: str, dtypes, ndim: int, device: int):
    _want(x, name, dtypes, ndim, device)
    if not x.is_contiguous():
        _fail(f"{name} must be contiguous")


def _count(x: int, name: str, least: int = 0):
    """Check a whole number that goes into an int32: ctypes would cut off what does not fit."""
    if not least <= x < 1 << 31:
        _fail(f"{name} must be {least}..2^31-1")


class _On:
    """The device and stream of a call that names a stream, or tensors of another device than the
    current one: kernels go there, and so does what the binding allocates."""

    def __init__(self, device: int, stream):
        self.ctx = [torch.cuda.device(device)]
        if stream is not None:
            # a handle too: what is allocated for the call may be freed before its kernels run
            if isinstance(stream, int):
                s = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
            else:
                s = stream
            self.ctx.append(torch.cuda.stream(s))
        self.stream = stream

    def __enter__(self):
        for c in self.ctx:
            c.__enter__()
        return H._stream_handle(self.stream)

    def __exit__(self, *exc):
        for c in reversed(self.ctx):
            c.__exit__(*exc)


class _Current:
    """The usual case, torch's current device and stream.  (torch.cuda.current_stream() builds an object
    around the same handle, which takes longer than a small step's kernels.)"""

    def __init__(self, device: int):
        self.device = device

    def __enter__(self):
        return torch._C._cuda_getCurrentRawStream(self.device)

    def __exit__(self, *exc):
        pass


_current: dict = {}


def _on(device: int, stream):
    if stream is not None or device != torch._C._cuda_getDevice():
        return _On(device, stream)
    on = _current.get(device)
    if on is None:
        on = _current[device] = _Current(device)
    return on


def max_runs(n_rows: int, n_tokens: int, block_tokens: int) -> int:
    """The most blocks that a step of n_tokens of n_rows requests can write."""
    return min(n_tokens, n_tokens // block_tokens + 2 * n_rows)


@dataclass
class Step:
    """One step's tables (hx_kv_map_args): row_start [rows + 1], kv_len [rows], slots
    [tokens] int64, runs [max_runs, 4], counts [4] = (tokens, runs, refused rows, blocks
    taken), ring_state [2] int64 after the step."""
    row_start: object
    kv_len: object
    slots: object
    runs: object
    counts: object
    ring_state: object

    @staticmethod
    def empty(n_rows: int, n_tokens: int, block_tokens: int, device="cuda") -> "Step":
        runs = max_runs(n_rows, n_tokens, block_tokens)
        # six allocations take less time than one that is split: views are recorded
        i32, i64 = torch.int32, torch.int64
        return Step(torch.empty(n_rows + 1, dtype=i32, device=device), torch.empty(n_rows, dtype=i32, device=device),
                    torch.empty(n_tokens, dtype=i64, device=device), torch.empty((runs, 4), dtype=i32, device=device),
                    torch.empty(4, dtype=i32, device=device), torch.empty(2, dtype=i64, device=device))


def map_step(held, add, block_table, ring, ring_state, n_tokens: int, block_tokens: int, out: Optional[Step] = None,
             stream=None) -> Step:
    """Build one step's tables on the GPU (hx_kv_map).

    held, add   int32 [rows]: tokens that each request holds, and what the step gives it
                (0: nothing, -1: it has ended)
    block_table int32 [rows, width], updated in place (rows may be strided)
    ring, ring_state  int32 [blocks], int64 [2]: the free blocks and (first, count); ended rows' blocks are
                entered in the ring, the new state is in the result
    n_tokens    the step's tokens, sum(max(add, 0)), known to the scheduler
    out         a Step to write to instead of a new one (not the one whose ring_state or kv_len is passed in)
    """
    _count(n_tokens, "map: n_tokens")
    _count(block_tokens, "map: block_tokens", 1)
    i32, i64 = (torch.int32,), (torch.int64,)
    dev = held.get_device()
    _dense(held, "held", i32, 1, dev)
    _dense(add, "add", i32, 1, dev)
    _want(block_table, "block_table", i32, 2, dev)
    _dense(ring, "ring", i32, 1, dev)
    _dense(ring_state, "ring_state", i64, 1, dev)
    n = held.shape[0]
    if add.shape[0] != n or block_table.shape[0] != n or ring_state.shape[0] != 2:
        _fail("map: held, add and block_table must have one entry per row, ring_state two")
    if block_table.shape[1] > 1 and block_table.stride(1) != 1:
        _fail("map: block_table's rows must be contiguous")
    if n < 1:
        _fail("map: n_rows must be at least 1")
    lib = load()
    with _on(dev, stream) as handle:
        if out is None:
            out = Step.empty(n, n_tokens, block_tokens, held.device)
        else:
            for x, name, t, shape in ((out.row_start, "row_start", i32, (n + 1,)), (out.kv_len, "kv_len", i32, (n,)),
                                      (out.slots, "slots", i64, (n_tokens,)), (out.counts, "counts", i32, (4,)),
                                      (out.runs, "runs", i32, (max_runs(n, n_tokens, block_tokens), 4)),
                                      (out.ring_state, "ring_state", i64, (2,))):
                _dense(x, "out." + name, t, len(shape), dev)
                if tuple(x.shape) != shape:
                    _fail(f"out.{name} must have the shape {shape}")
        a = hx_kv_map_args(n, n_tokens, block_tokens, ring.shape[0], block_table.shape[1], out.runs.shape[0],
                           block_table.stride(0) if n > 1 else block_table.shape[1], held.data_ptr(), add.data_ptr(),
                           block_table.data_ptr(), ring.data_ptr(), ring_state.data_ptr(), out.row_start.data_ptr(),
                           out.kv_len.data_ptr(), out.slots.data_ptr(), out.runs.data_ptr(), out.counts.data_ptr(),
                           out.ring_state.data_ptr())
        H._check(lib, lib.hx_kv_map(ctypes.byref(a), handle))
    return out


class Cache:
    """A paged 8-bit cache on tensors that the caller owns (hx_kv_cache).

    k, v              float8_e4m3fn [blocks, kv heads, block tokens, head dim]; the blocks may be
                      strided (for instance k and v side by side), what is inside one is contiguous
    k_scale, v_scale  float32 [blocks, kv heads]
    """

    def __init__(self, k, v, k_scale, v_scale):
        f8, f32 = (torch.float8_e4m3fn,), (torch.float32,)
        dev = k.get_device()
        for x, name in ((k, "k"), (v, "v")):
            _want(x, name, f8, 4, dev)
        for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _want(x, name, f32, 2, dev)
        N, heads, block, dim = k.shape
        if v.shape != k.shape or tuple(k_scale.shape) != (N, heads) or tuple(v_scale.shape) != (N, heads):
            _fail("cache: k and v must have one shape, and the scales its first two dimensions")
        whole = heads * block * dim
        for x, name in ((k, "k"), (v, "v")):
            if not x[0].is_contiguous():
                _fail(f"cache: a block of {name} must be contiguous")
        for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if heads > 1 and x.stride(1) != 1:
                _fail(f"cache: a block's scales in {name} must be contiguous")
        if N > 1 and (k.stride(0) != v.stride(0) or k_scale.stride(0) != v_scale.stride(0)):
            _fail("cache: k and v must have the same block stride, and so must their scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device = dev
        self.struct = hx_kv_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                  k.stride(0) if N > 1 else whole, k_scale.stride(0) if N > 1 else heads, N, heads, block,
                                  dim)
        self._ref = ctypes.byref(self.struct)
        self._work = {}  # workspaces by stream: calls on one stream follow one another,
        self._turn = threading.Lock()  # and all launches of one call those of another, whatever threads they are from
        # in host memory that the kernels write to: it holds its zero without any stream's doing
        self._status = torch.zeros(1, dtype=torch.int32, pin_memory=True)
        self._status_at = self._status.data_ptr()
        self.lib = load()

    @staticmethod
    def empty(n_blocks: int, n_kv_heads: int, block_tokens: int, head_dim: int, device="cuda") -> "Cache":
        """A new cache; its contents are undefined until tokens are appended."""
        shape = (n_blocks, n_kv_heads, block_tokens, head_dim)
        k, v = (torch.empty(shape, dtype=torch.float8_e4m3fn, device=device) for _ in range(2))
        ks, vs = (torch.empty(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
        return Cache(k, v, ks, vs)

    def check(self) -> None:
        """Raise if a wait inside a kernel of an `attend` ran out, whose tokens then hold NaN.  Of calls whose work is
        done: synchronize with their stream first."""
        if self._status.item():
            raise H.HxError(H.HX_ERR_CUDA, "attend: a wait inside a kernel ran out; results hold NaN")

    def append(self, k, v, runs, stream=None) -> None:
        """Write a step's keys and values, [tokens, kv heads, head dim] in bf16, f16 or f32 (tokens and heads may be
        strided by multiples of 16 bytes), where `runs` (a Step's) says (hx_kv_append)."""
        kinds = (torch.bfloat16, torch.float16, torch.float32)
        _want(k, "k", kinds, 3, self.device)
        _want(v, "v", (k.dtype,), 3, self.device)
        _dense(runs, "runs", (torch.int32,), 2, self.device)
        T, heads, dim = k.shape
        if v.shape != k.shape or heads != self.struct.n_kv_heads or dim != self.struct.head_dim or runs.shape[1] != 4:
            _fail("append: k and v must be [tokens, kv heads, head dim] of the cache, runs [runs, 4]")
        if k.stride(2) != 1 or v.stride(2) != 1:
            _fail("append: a head's values must be contiguous")
        a = hx_kv_new(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), v.stride(0), v.stride(1), T,
                      kinds.index(k.dtype), runs.data_ptr(), runs.shape[0])
        with _on(self.device, stream) as handle:
            H._check(self.lib, self.lib.hx_kv_append(self._ref, ctypes.byref(a), handle))

    def attend(self, q, block_table, row_start, kv_len, *, max_q: int = 0, sm_scale: Optional[float] = None,
               causal: bool = True, window: int = 0, out=None, return_lse: bool = False, workspace=None, stream=None):
        """softmax(sm_scale * q k^T) v over what each token sees (hx_kv_attend).

        q           bf16 or f16 [tokens, heads, head dim] (tokens and heads may be strided by multiples of 8)
        block_table, row_start, kv_len   int32, as map_step leaves them
        max_q       the most tokens that a row has in this step, if the scheduler knows it (1: every row
                    decodes; fewer kernels run), 0 if not
        sm_scale    default head dim ** -0.5
        workspace   uint8 tensor to use instead of the one that the cache keeps for each stream (not by calls
                    on another cache at the same time)

        Returns out, or (out, lse) with lse float32 [tokens, heads].  There is no backward pass: no gradient flows
        from them to q.
        """
        _count(window, "attend: window")
        _count(max_q, "attend: max_q")
        kinds = (torch.bfloat16, torch.float16)
        dev = self.device
        _want(q, "q", kinds, 3, dev)
        _want(block_table, "block_table", (torch.int32,), 2, dev)
        _dense(row_start, "row_start", (torch.int32,), 1, dev)
        _dense(kv_len, "kv_len", (torch.int32,), 1, dev)
        T, heads, dim = q.shape
        n = kv_len.shape[0]
        if dim != self.struct.head_dim or q.stride(2) != 1:
            _fail("attend: q must be [tokens, heads, head dim] of the cache, a head's values contiguous")
        if row_start.shape[0] != n + 1 or block_table.shape[0] != n:
            _fail("attend: row_start must have one entry more than kv_len, block_table as many")
        if block_table.shape[1] > 1 and block_table.stride(1) != 1:
            _fail("attend: block_table's rows must be contiguous")
        with _on(dev, stream) as handle:
            if out is None:
                out = torch.empty((T, heads, dim), dtype=q.dtype, device=q.device)
            else:
                _want(out, "out", (q.dtype,), 3, dev)
                if out.shape != q.shape or out.stride(2) != 1:
                    _fail("attend: out must have q's shape, a head's values contiguous")
            lse = torch.empty((T, heads), dtype=torch.float32, device=q.device) if return_lse else None
            a = hx_kv_query(q.data_ptr(), out.data_ptr(), lse.data_ptr() if return_lse else None, q.stride(0),
                            q.stride(1), out.stride(0), out.stride(1), T, heads, kinds.index(q.dtype), n,
                            row_start.data_ptr(), kv_len.data_ptr(), block_table.data_ptr(),
                            block_table.stride(0) if n > 1 else block_table.shape[1], block_table.shape[1], max_q,
                            1 if causal else 0, window, dim ** -0.5 if sm_scale is None else sm_scale, None, 0, self._status_at)
            ref = ctypes.byref(a)
            if workspace is not None:
                _dense(workspace, "workspace", (torch.uint8,), 1, dev)
            with self._turn:
                if workspace is None:
                    need = ctypes.c_int64()
                    H._check(self.lib, self.lib.hx_kv_attend_workspace(self._ref, ref, ctypes.byref(need)))
                    graph = torch.cuda.is_current_stream_capturing()  # a graph has a workspace of its own
                    workspace = None if graph else self._work.pop(handle, None)
                    if workspace is None or workspace.numel() < need.value:
                        workspace = torch.empty(need.value, dtype=torch.uint8, device=q.device)
                    if not graph:  # the streams used last are the dict's last (what goes, goes back to its own stream's memory)
                        self._work[handle] = workspace
                        if len(self._work) > 16:
                            del self._work[next(iter(self._work))]
                a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
                H._check(self.lib, self.lib.hx_kv_attend(self._ref, ref, handle))
        return (out, lse) if return_lse else out
