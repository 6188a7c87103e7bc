"""Python binding of the serving step's cache operators (include/hxkv.h), and of the rotary positions
before them (include/hxstep.h).

One step of an instance's running batch over a paged 8-bit cache:

    step = map_step(held, add, block_table, ring, ring_state, n_tokens, block)   # where its tokens go
    q, k = rope.rotate(q, k, step.row_start, step.kv_len)                        # turned by their positions
    cache.append(k, v, step.runs)                                                # their keys and values, in e4m3
    out = cache.attend(q, block_table, step.row_start, step.kv_len)              # what each token reads

Arguments are torch tensors on the current CUDA device; everything runs in the
library's kernels on torch's current stream (or `stream`), and there is no CPU
fallback.  The tensors must not be freed or reused on another stream before
the kernels are done, as for any asynchronous call.
"""
from __future__ import annotations

import ctypes
import math
import threading
from dataclasses import dataclass
from fractions import Fraction
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


class hx_rotate_args(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("q", "k", "q_out", "k_out")] + \
               [(n, _i64) for n in ("q_token_stride", "q_head_stride", "k_token_stride", "k_head_stride", "q_out_token_stride",
                                    "q_out_head_stride", "k_out_token_stride", "k_out_head_stride")] + \
               [(n, _i32) for n in ("n_tokens", "n_heads", "n_kv_heads", "head_dim", "rotary_dim", "dtype", "interleaved",
                                    "inverse")] + \
               [("scale", ctypes.c_float), ("n_rows", _i32)] + \
               [(n, _vp) for n in ("turns", "positions", "row_start", "kv_len")]


_lib = None


def load():
    """The library with the prototypes of hxkv.h and hx_rotate; raises if it has not been built."""
    global _lib
    if _lib is None:
        lib = H.load()
        lib.hx_kv_max_runs.restype = _i64
        lib.hx_kv_max_runs.argtypes = [_i32, _i32, _i32]
        for name, args in [("hx_kv_map", [_vp, _vp]), ("hx_kv_append", [_vp, _vp, _vp]),
                           ("hx_kv_attend_workspace", [_vp, _vp, _vp]), ("hx_kv_attend", [_vp, _vp, _vp]),
                           ("hx_rotate", [_vp, _vp])]:
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


_PI = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


class Rope:
    """Rotary positions (hx_rotate): the table of a model's frequencies, on one device.

    frequencies   radians a position for each pair of values, in 64 bits; they set how much of a head is turned
                  (2 values for each; see Rope.frequencies)
    interleaved   pairs are values 2i and 2i + 1 of a head, not i and i + len(frequencies)
    scale         factor of what is turned
    """

    def __init__(self, frequencies, *, interleaved: bool = False, scale: float = 1.0, device="cuda"):
        f = torch.as_tensor(frequencies, dtype=torch.float64).cpu()
        if f.dim() != 1 or not 1 <= f.shape[0] <= 512 or not bool(torch.isfinite(f).all()):
            _fail("rope: frequencies must be 1 to 512 finite numbers")
        if not math.isfinite(scale):
            _fail("rope: scale is not finite")
        turns = [round(Fraction(x) / (2 * _PI) * (1 << 64)) % (1 << 64) for x in f.tolist()]
        self.turns = torch.tensor([t - (t >> 63 << 64) for t in turns], dtype=torch.int64).to(device)
        self.device = self.turns.get_device()
        self.rotary_dim, self.interleaved, self.scale = 2 * len(turns), bool(interleaved), float(scale)
        self.lib = load()

    @staticmethod
    def frequencies(rotary_dim: int, theta: float = 10000.0, *, scaling: str = "linear", factor: float = 1.0,
                    original: int = 0, low: float = 1.0, high: float = 32.0):
        """theta ** (-2i / rotary_dim) for the rotary_dim / 2 pairs, scaled for contexts `factor` times as long as trained:

        "linear"  every frequency / factor (Chen et al. 2023)
        "base"    theta * factor ** (rotary_dim / (rotary_dim - 2)): the slowest / factor, the fastest as they are
        "bands"   those that turn fewer than `low` times in the `original` tokens / factor, those that
                  turn more than `high` times as they are, the others between (Peng et al. 2023)
        """
        if rotary_dim < 2 or rotary_dim % 2 or not theta > 0 or not factor > 0:
            _fail("rope: rotary_dim must be even and at least 2, theta and factor above 0")
        if scaling == "base" and factor != 1:
            if rotary_dim == 2:
                _fail("rope: one pair alone has no base to scale")
            theta *= factor ** (rotary_dim / (rotary_dim - 2))
        f = theta ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / rotary_dim)
        if scaling == "linear":
            return f / factor
        if scaling == "base":
            return f
        if scaling != "bands" or original < 1 or not high > low:
            _fail("rope: scaling must be linear, base, or bands with original >= 1 and high above low")
        keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return keep * f + (1 - keep) * f / factor

    def rotate(self, q, k=None, row_start=None, kv_len=None, *, positions=None, out=None, inverse: bool = False, stream=None):
        """Turn a step's queries and keys by their positions (hx_rotate).

        q, k       bf16, f16 or f32 [tokens, heads, head dim] and [tokens, kv heads, head dim] (tokens and heads may
                   be strided: the projections' output with q, k and v side by side)
        row_start, kv_len   int32, as map_step leaves them; tokens behind the last row are left as they are, in
                   new outputs too, where they are then undefined
        positions  int32 [tokens] in their place
        out        (q's, k's) tensors to write to; (q, k) itself: in place
        inverse    turn the other way, times the same scale: the way back where that is 1 (with scale s, s * s times what was turned)

        Returns q's and k's, or q's alone where there is no k.  No backward pass is recorded: the gradient of what is turned is
        rotate(the gradient of the result, inverse=True), at every scale.
        """
        dev = self.device
        kinds = (torch.bfloat16, torch.float16, torch.float32)
        _want(q, "q", kinds, 3, dev)
        T, heads, dim = q.shape
        if q.stride(2) != 1 and dim > 1:
            _fail("rotate: a head's values must be contiguous")
        n = 0
        if positions is not None:
            if row_start is not None or kv_len is not None:
                _fail("rotate: either positions or row_start and kv_len")
            _dense(positions, "positions", (torch.int32,), 1, dev)
            if positions.shape[0] != T:
                _fail("rotate: positions must have one entry per token")
        else:
            if row_start is None or kv_len is None:
                _fail("rotate: either positions or row_start and kv_len")
            _dense(row_start, "row_start", (torch.int32,), 1, dev)
            _dense(kv_len, "kv_len", (torch.int32,), 1, dev)
            n = kv_len.shape[0]
            if row_start.shape[0] != n + 1:
                _fail("rotate: row_start must have one entry more than kv_len")
        kv_heads = 0
        if k is not None:
            _want(k, "k", (q.dtype,), 3, dev)
            kv_heads = k.shape[1]
            if k.shape[0] != T or k.shape[2] != dim or (k.stride(2) != 1 and dim > 1):
                _fail("rotate: k must be [tokens, kv heads, head dim] with q's tokens and head dim, a head's values contiguous")
            if kv_heads < 1:
                _fail("rotate: k has no heads")
        with _on(dev, stream) as handle:
            if out is None:
                q_out = torch.empty((T, heads, dim), dtype=q.dtype, device=q.device)
                k_out = None if k is None else torch.empty((T, kv_heads, dim), dtype=q.dtype, device=q.device)
            else:
                q_out, k_out = (out, None) if k is None else out
                for x, like, name in ((q_out, q, "q"), (k_out, k, "k")):
                    if like is not None:
                        _want(x, f"out: {name}'s", (q.dtype,), 3, dev)
                        if x.shape != like.shape or (x.stride(2) != 1 and dim > 1):
                            _fail(f"rotate: out must have {name}'s shape, a head's values contiguous")
            none = k is None
            a = hx_rotate_args(
                q.data_ptr(), None if none else k.data_ptr(), q_out.data_ptr(), None if none else k_out.data_ptr(),
                q.stride(0), q.stride(1), 0 if none else k.stride(0), 0 if none else k.stride(1), q_out.stride(0), q_out.stride(1),
                0 if none else k_out.stride(0), 0 if none else k_out.stride(1), T, heads, kv_heads, dim, self.rotary_dim,
                kinds.index(q.dtype), self.interleaved, 1 if inverse else 0, self.scale, n, self.turns.data_ptr(),
                None if positions is None else positions.data_ptr(), None if n == 0 else row_start.data_ptr(),
                None if n == 0 else kv_len.data_ptr())
            H._check(self.lib, self.lib.hx_rotate(ctypes.byref(a), handle))
        return q_out if none else (q_out, k_out)


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
