"""Python binding of what follows a serving step's last product (include/hxstep.h): from logits to tokens.

    rules = Rules(history=h, length=n, prompt_len=m, repetition=r, mask=bits, mask_row=state)   # what holds for the requests
    token, logprob = sample(logits, noise, temperature=t, top_p=0.9, rules=rules)               # the next token of each
    logits = adjust(logits, rules)                                                              # or the adjusted logits

Arguments are torch tensors on one CUDA device; everything runs in the library's kernels on torch's
current stream (or `stream`), and there is no CPU fallback.  The tensors must not be freed or reused on another
stream before the kernels are done, as for any asynchronous call.  There is no backward pass.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import hxsim as H
from . import kvcache as KV
from .kvcache import _dense, _fail, _on, _want

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float

MAX_VOCAB = 393216
MAX_HISTORY = 524287
MAX_BIAS = 4095

_KINDS = (torch.bfloat16, torch.float16, torch.float32)  # by hxkv.h's numbers


class hx_rules(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("history_width", _i32), ("history", _vp), ("history_stride", _i64)] + \
               [(n, _vp) for n in ("length", "prompt_len", "repetition", "presence", "frequency", "bias_start", "bias_token",
                                   "bias_value", "mask", "mask_row")] + \
               [("mask_stride", _i64)] + [(n, _i32) for n in ("n_bias", "n_masks", "mask_width")]


class hx_logits(ctypes.Structure):
    _fields_ = [("x", _vp), ("stride", _i64)] + [(n, _i32) for n in ("n_rows", "n_vocab", "dtype")]


class hx_pick(ctypes.Structure):
    _fields_ = [("noise", _vp), ("noise_stride", _i64)] + [(n, _vp) for n in ("temperature", "top_k", "top_p", "min_p")] + \
               [(n, _f32) for n in ("all_temperature", "all_top_p", "all_min_p")] + [("all_top_k", _i32)] + \
               [(n, _vp) for n in ("token", "logprob", "workspace")] + [("workspace_bytes", _i64)]


_lib = None


def load():
    """The library with the prototypes of hxstep.h; raises if it has not been built."""
    global _lib
    if _lib is None:
        lib = KV.load()
        for name, args in [("hx_adjust", [_vp, _vp, _vp, _i64, _i32, _vp]), ("hx_sample", [_vp, _vp, _vp, _vp])]:
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        lib.hx_sample_workspace.restype = _i64
        lib.hx_sample_workspace.argtypes = [_vp, _vp, _vp]
        _lib = lib
    return _lib


class Rules:
    """What holds for the rows of a step's logits (hx_rules), on tensors that the caller owns and may write to between calls.
    Each is optional:

    history     int32 [rows, width], rows may be strided: a request's tokens, the first length[r] of them; what is no token
                of the vocabulary is passed over
    length      int32 [rows]
    prompt_len  int32 [rows]: so many of them are its prompt, the others were written (default: all were written)
    repetition, presence, frequency   float32 [rows]: logits of tokens in the history are divided by `repetition` where they
                are above 0 and multiplied by it elsewhere; those of tokens that were written are lowered by
                presence + frequency * times
    bias        (start int32 [rows + 1], token int32 [entries], value float32 [entries]): row r's entries are start[r] to
                start[r + 1], at most MAX_BIAS; of several for one token the last counts
    mask        int32 [masks, words], rows may be strided: bit t % 32 of word t / 32 allows token t
    mask_row    int32 [rows]: which mask holds for a row, out of range (-1): none (default: row r's is mask r)
    """

    def __init__(self, *, history=None, length=None, prompt_len=None, repetition=None, presence=None, frequency=None,
                 bias=None, mask=None, mask_row=None):
        i32, f32 = (torch.int32,), (torch.float32,)
        start, token, value = (None, None, None) if bias is None else bias
        whole = [("length", length), ("prompt_len", prompt_len), ("mask_row", mask_row)]
        real = [("repetition", repetition), ("presence", presence), ("frequency", frequency)]
        some = [x for x in (history, length, start, mask, mask_row) if x is not None]
        self.device = some[0].get_device() if some else None
        self.rows: Optional[int] = None
        if history is None and any(x is not None for _, x in whole[:2] + real):
            _fail("rules: length, prompt_len, repetition, presence and frequency need a history")
        if history is not None and length is None:
            _fail("rules: a history needs length")
        if mask is None and mask_row is not None:
            _fail("rules: mask_row needs a mask")
        if history is not None:
            _want(history, "history", i32, 2, self.device)
            if history.shape[1] > 1 and history.stride(1) != 1:
                _fail("rules: history's rows must be contiguous")
            if history.shape[1] > MAX_HISTORY:
                _fail(f"rules: a row of history has more than {MAX_HISTORY} entries")
            self._rows(history.shape[0], "history")
        for kinds, names in ((i32, whole), (f32, real)):
            for name, x in names:
                if x is not None:
                    _dense(x, name, kinds, 1, self.device)
                    self._rows(x.shape[0], name)
        if bias is not None:
            _dense(start, "bias: start", i32, 1, self.device)
            _dense(token, "bias: token", i32, 1, self.device)
            _dense(value, "bias: value", f32, 1, self.device)
            self._rows(start.shape[0] - 1, "bias: start")
            if token.shape != value.shape:
                _fail("rules: bias must have one value for each token")
        if mask is not None:
            _want(mask, "mask", i32, 2, self.device)
            if mask.shape[1] > 1 and mask.stride(1) != 1:
                _fail("rules: a mask's words must be contiguous")
            if mask.shape[0] and not mask.shape[1]:  # its address would say that there is none
                _fail("rules: a mask has no words")
            if mask_row is None:
                self._rows(mask.shape[0], "mask")
        p = lambda x: None if x is None else x.data_ptr()
        stride = lambda x: 0 if x is None else x.stride(0) if x.shape[0] > 1 else x.shape[1]
        self.tensors = (history, length, prompt_len, repetition, presence, frequency, start, token, value, mask, mask_row)
        # an empty tensor has no address: a list of no entries, or a history of no columns, is none
        if bias is not None and token.shape[0] == 0:
            start = token = value = None
        if history is not None and history.numel() == 0:
            history = length = prompt_len = repetition = presence = frequency = None
        self.struct = hx_rules(self.rows or 0, 0 if history is None else history.shape[1], p(history), stride(history), p(length),
                               p(prompt_len), p(repetition), p(presence), p(frequency), p(start), p(token), p(value), p(mask),
                               p(mask_row), stride(mask), 0 if token is None else token.shape[0],
                               0 if mask is None else mask.shape[0], 0 if mask is None else mask.shape[1])
        self._ref = ctypes.byref(self.struct)

    def _rows(self, n: int, name: str):
        if self.rows is None:
            self.rows = n
        if n != self.rows:
            _fail(f"rules: {name} has {n} rows, not {self.rows}")

    def _for(self, x):
        """A reference to the struct for these logits."""
        if self.rows is None:  # nothing holds: for any number of rows
            return ctypes.byref(hx_rules(x.shape[0]))
        if self.device != x.get_device():
            _fail(f"rules are on cuda:{self.device}, the logits are not")
        if self.rows != x.shape[0]:
            _fail(f"rules are for {self.rows} rows, the logits have {x.shape[0]}")
        return self._ref


def _logits(x) -> hx_logits:
    _want(x, "logits", _KINDS, 2, x.get_device())
    n, vocab = x.shape
    if not 1 <= vocab <= MAX_VOCAB:
        _fail(f"logits: the vocabulary must be 1..{MAX_VOCAB}")
    if vocab > 1 and x.stride(1) != 1:
        _fail("logits: a row must be contiguous")
    return hx_logits(x.data_ptr(), x.stride(0) if n > 1 else vocab, n, vocab, _KINDS.index(x.dtype))


def adjust(logits, rules: Rules, *, out=None, dtype=None, stream=None):
    """Logits [rows, vocabulary] in bf16, f16 or f32 (rows may be strided), as the rules adjust them (hx_adjust): what a mask does
    not allow is -infinity.

    out    a tensor to write to; `logits` itself: in place
    dtype  of a new one: the logits' (default) or float32
    """
    a = _logits(logits)
    n, vocab = logits.shape
    ref = rules._for(logits)
    kinds = (logits.dtype, torch.float32)
    if out is not None:
        _want(out, "out", kinds, 2, logits.get_device())
        if out.shape != logits.shape or (vocab > 1 and out.stride(1) != 1) or dtype not in (None, out.dtype):
            _fail("adjust: out must have the logits' shape and the dtype asked for, a row contiguous")
    elif dtype is not None and dtype not in kinds:
        _fail("adjust: dtype must be the logits' or float32")
    lib = load()
    with _on(logits.get_device(), stream) as handle:
        if out is None:
            out = torch.empty((n, vocab), dtype=dtype or logits.dtype, device=logits.device)
        H._check(lib, lib.hx_adjust(ctypes.byref(a), ref, out.data_ptr(), out.stride(0) if n > 1 else vocab,
                                    _KINDS.index(out.dtype), handle))
    return out


def sample(logits, noise=None, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, rules: Optional[Rules] = None, out=None,
           stream=None):
    """The next token of each row of logits [rows, vocabulary] in bf16, f16 or f32 (hx_sample; rows may be strided).

    noise        float32 [rows, vocabulary], random numbers of the exponential distribution (Tensor.exponential_), rows may be
                 strided; None: the likeliest token of every row
    temperature, top_p, min_p   float32 [rows] or a number
    top_k        int32 [rows] or a number
                 (temperature 0 or below: the likeliest token; top_k 0 or below, top_p 1, min_p 0: no tokens left out)
    rules        how the logits are adjusted before
    out          (token int32 [rows], logprob float32 [rows]) to write to

    Returns (token, logprob): -1 and -infinity where the rules leave no token; logprob is the token's share of
    all that the rules leave, at the row's temperature, before tokens are left out for being unlikely.
    """
    a = _logits(logits)
    dev = logits.get_device()
    n, vocab = logits.shape
    ref = None if rules is None else rules._for(logits)
    p = hx_pick()
    if noise is not None:
        _want(noise, "noise", (torch.float32,), 2, dev)
        if noise.shape != logits.shape or (vocab > 1 and noise.stride(1) != 1):
            _fail("sample: noise must have the logits' shape, a row contiguous")
        p.noise, p.noise_stride = noise.data_ptr(), noise.stride(0) if n > 1 else vocab
    for x, name, kind in ((temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
                          (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
        if isinstance(x, torch.Tensor):
            _dense(x, name, (kind,), 1, dev)
            if x.shape[0] != n:
                _fail(f"sample: {name} must have one entry per row")
            setattr(p, name, x.data_ptr())
        else:
            if kind == torch.int32 and (not -1 << 31 <= x < 1 << 31 or x != int(x)):
                _fail(f"sample: {name} must be a whole number of 32 bits")
            setattr(p, "all_" + name, int(x) if kind == torch.int32 else float(x))
    lib = load()
    with _on(dev, stream) as handle:
        if out is None:
            token = torch.empty(n, dtype=torch.int32, device=logits.device)
            logprob = torch.empty(n, dtype=torch.float32, device=logits.device)
        else:
            token, logprob = out
            _dense(token, "out: token", (torch.int32,), 1, dev)
            _dense(logprob, "out: logprob", (torch.float32,), 1, dev)
            if token.shape[0] != n or logprob.shape[0] != n:
                _fail("sample: out must have one entry per row")
        p.token, p.logprob = token.data_ptr(), logprob.data_ptr()
        x, p_ref = ctypes.byref(a), ctypes.byref(p)
        p.workspace_bytes = lib.hx_sample_workspace(x, ref, p_ref)
        work = torch.empty(p.workspace_bytes, dtype=torch.uint8, device=logits.device)  # its stream's, or its graph's
        p.workspace = work.data_ptr()
        H._check(lib, lib.hx_sample(x, ref, p_ref, handle))
    return token, logprob
