"""The operators on either side of the cache without a GPU: struct layouts and refusals before any launch."""
import ctypes
import itertools
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import kvcache as KV
from paper_2505_05286_gb300 import logits as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = [KV.hx_rotate_args, L.hx_rules, L.hx_logits] + ([L.hx_pick] if hasattr(L, "hx_pick") else [])
FAKE = 1 << 30  # an aligned address; nothing is launched with it


@pytest.fixture(scope="module")
def lib():
    B_.build()
    return L.load()


def test_both_builds_export_what_the_header_declares(lib):
    text = open(os.path.join(ROOT, "include", "hxstep.h")).read()
    names = sorted(set(re.findall(r"^\s*(?:int|int64_t)\s+(hx_\w+)\s*\(", text, re.M)))
    assert {"hx_rotate", "hx_adjust"} <= set(names)
    for n in names:
        assert hasattr(lib, n) and hasattr(H.load_checked(), n)


def test_struct_layout_matches_binding(tmp_path):
    lines = "".join(f'printf("{s.__name__} %zu\\n", sizeof({s.__name__}));\n' + "".join(
        f'printf("{s.__name__}.{f} %zu\\n", offsetof({s.__name__}, {f}));\n' for f, _ in s._fields_) for s in STRUCTS)
    src = tmp_path / "probe.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "hxstep.h"\nint main(void) {\n' + lines +
                   'printf("limits %d\\n", HX_MAX_VOCAB + HX_MAX_HISTORY + HX_MAX_BIAS);\nreturn 0;\n}\n')
    exe = tmp_path / "probe"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    by = {s.__name__: s for s in STRUCTS}
    for line in subprocess.check_output([str(exe)], text=True).splitlines():
        name, size = line.split()
        if name == "limits":
            assert int(size) == L.MAX_VOCAB + L.MAX_HISTORY + L.MAX_BIAS
            continue
        s, _, f = name.partition(".")
        assert (getattr(by[s], f).offset if f else ctypes.sizeof(by[s])) == int(size), name


def _set(struct, **kw):
    s = type(struct)()
    ctypes.pointer(s)[0] = struct
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _refused(lib, rc, msg):
    err = lib.hx_last_error().decode()
    assert rc == H.HX_ERR_INVALID and msg in err, (rc, err)


# ---------------------------------------------------------------- rotate

MB = 1 << 20


def _rotate(**kw):
    """q [10, 4, 64] and k [10, 2, 64] of bf16, everything at a place of its own."""
    a = KV.hx_rotate_args(FAKE, FAKE + MB, FAKE + 2 * MB, FAKE + 3 * MB, 256, 64, 128, 64, 256, 64, 128, 64, 10, 4, 2, 64, 64,
                          KV.HX_BF16, 0, 0, 1.0, 3, FAKE + 4 * MB, None, FAKE + 5 * MB, FAKE + 6 * MB)
    return _set(a, **kw)


def test_rotate_refusals(lib):
    for kw, msg in [(dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=2 ** 30 + 1), "n_tokens"), (dict(n_heads=0), "n_heads"),
                    (dict(n_heads=2049), "n_heads"), (dict(n_kv_heads=-1), "n_kv_heads"), (dict(n_kv_heads=2049), "n_kv_heads"),
                    (dict(n_kv_heads=0), "k must be NULL"), (dict(k=None), "k must be NULL"), (dict(head_dim=1), "head_dim"),
                    (dict(head_dim=1025), "head_dim"), (dict(rotary_dim=0), "rotary_dim"), (dict(rotary_dim=66), "rotary_dim"),
                    (dict(rotary_dim=7), "rotary_dim"), (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"),
                    (dict(interleaved=2), "interleaved"), (dict(inverse=-1), "inverse"), (dict(scale=math.inf), "scale"),
                    (dict(scale=math.nan), "scale"), (dict(n_rows=0), "n_rows"), (dict(n_rows=65537), "n_rows"),
                    (dict(positions=FAKE + 7 * MB), "positions"), (dict(row_start=None), "NULL"), (dict(kv_len=None), "NULL"),
                    (dict(turns=None), "NULL"), (dict(q=None), "NULL"), (dict(k_out=None), "NULL"), (dict(q=FAKE + 1), "aligned"),
                    (dict(k_out=FAKE + 3 * MB + 1), "aligned"), (dict(turns=FAKE + 4 * MB + 4), "aligned"),
                    (dict(row_start=FAKE + 5 * MB + 2), "aligned"), (dict(kv_len=FAKE + 6 * MB + 2), "aligned"),
                    (dict(q_token_stride=-256), "strides"), (dict(n_tokens=2 ** 30, q_token_stride=2 ** 37), "2^44"), (dict(k_head_stride=2 ** 38), "strides"),
                    (dict(q_out_token_stride=255), "one place"), (dict(q_out_head_stride=63), "one place"),
                    (dict(k_out_token_stride=0), "one place"), (dict(q_out=FAKE + 2), "overlaps q"),
                    (dict(q_out=FAKE, q_out_head_stride=128, q_out_token_stride=512), "other strides"),
                    (dict(k_out=FAKE + MB + 2), "overlaps k"), (dict(k_out=FAKE), "overlaps the other"),
                    (dict(k_out=FAKE + 2 * MB + 4096), "overlaps the other"), (dict(q_out=FAKE + 5 * MB), "row_start"),
                    (dict(k_out=FAKE + 4 * MB - 8), "turns")]:
        _refused(lib, lib.hx_rotate(ctypes.byref(_rotate(**kw)), None), msg)
    _refused(lib, lib.hx_rotate(None, None), "NULL")
    assert lib.hx_rotate(ctypes.byref(_rotate(n_tokens=0, q=None, k=None, row_start=None)), None) == H.HX_OK


def _bytes(base, T, ts, heads, hs, D, size):
    return {base + (t * ts + h * hs + d) * size + b for t in range(T) for h in range(heads) for d in range(D) for b in range(size)}


@pytest.mark.skipif(torch.cuda.is_available(), reason="what passes the checks would be launched, at addresses that are none")
def test_rotate_finds_every_overlap(lib):
    """Against all bytes of small arrays: what shares one is refused, q and k side by side in one buffer are not."""
    rng = np.random.default_rng(0)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        T, H_, K, D = (int(v) for v in rng.integers(1, 4, 4))
        D = 2 * D
        kind = rng.integers(0, 4)
        if kind == 0:  # side by side
            ts, hs = (H_ + K) * D + int(rng.integers(0, 3)), D
        elif kind == 1:  # heads between one another
            ts, hs = (H_ + K) * 2 * D, 2 * D
        elif kind == 2:  # heads outermost
            ts, hs = 2 * D, 2 * D * T + int(rng.integers(0, 3))
        else:
            ts, hs = H_ * D, D
        q, qo = 5000, 5000 + int(rng.integers(-60, 60))
        ko, k = qo + int(rng.integers(-120, 120)), 50000
        a = _rotate(q=2 * q, q_out=2 * qo, k=2 * k, k_out=2 * ko, n_tokens=T, n_heads=H_, n_kv_heads=K, head_dim=D, rotary_dim=2,
                    q_token_stride=ts, q_head_stride=hs, q_out_token_stride=ts, q_out_head_stride=hs, k_out_token_stride=ts,
                    k_out_head_stride=hs, k_token_stride=K * D, k_head_stride=D)
        b = {n: _bytes(2 * at, T, ts, h, hs, D, 2) for n, at, h in (("q", q, H_), ("qo", qo, H_), ("ko", ko, K))}
        inside = len(b["qo"]) == T * H_ * D * 2 and len(b["ko"]) == T * K * D * 2
        shared = (q != qo and b["q"] & b["qo"]) or b["q"] & b["ko"] or b["qo"] & b["ko"] or not inside
        rc = lib.hx_rotate(ctypes.byref(a), None)
        if shared:
            assert rc == H.HX_ERR_INVALID, (T, H_, K, D, ts, hs, q, qo, ko)
        seen[bool(shared)] += rc == H.HX_ERR_INVALID
    # the usual layouts pass the checks (what then fails is the launch: there is no device here)
    D = 64
    for ts, hs, ko in ((6 * D, D, 4 * D), (2 * 6 * D, D, 4 * D), (12 * D, 2 * D, D)):  # in place, side by side or by turns
        a = _rotate(q=FAKE, q_out=FAKE, k=FAKE + 2 * ko, k_out=FAKE + 2 * ko, q_token_stride=ts, q_head_stride=hs,
                    q_out_token_stride=ts, q_out_head_stride=hs, k_token_stride=ts, k_head_stride=hs, k_out_token_stride=ts,
                    k_out_head_stride=hs)
        assert lib.hx_rotate(ctypes.byref(a), None) == H.HX_ERR_CUDA
    assert lib.hx_rotate(ctypes.byref(_rotate()), None) == H.HX_ERR_CUDA
    assert seen[True] > 500


def test_frequencies():
    f = KV.Rope.frequencies(128, 10000.0)
    assert f.dtype == torch.float64 and f[0] == 1 and abs(float(f[1]) - 10000 ** (-2 / 128)) < 1e-15
    assert torch.equal(KV.Rope.frequencies(64, factor=4.0), KV.Rope.frequencies(64) / 4)
    base = KV.Rope.frequencies(64, scaling="base", factor=8.0)
    plain = KV.Rope.frequencies(64)
    assert base[0] == plain[0] and abs(float(base[-1] * 8 / plain[-1]) - 1) < 1e-12
    bands = KV.Rope.frequencies(128, scaling="bands", factor=8.0, original=8192)
    plain = KV.Rope.frequencies(128)
    turns = 8192 * plain / (2 * math.pi)
    assert torch.equal(bands[turns > 32], plain[turns > 32])
    assert torch.allclose(bands[turns < 1], plain[turns < 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert bool((bands[mid] < plain[mid]).all()) and bool((bands[mid] > plain[mid] / 8).all())
    for kw in (dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=4, theta=0.0), dict(rotary_dim=4, factor=-1.0),
               dict(rotary_dim=4, scaling="other"), dict(rotary_dim=4, scaling="bands"), dict(rotary_dim=2, scaling="base", factor=2.0),
               dict(rotary_dim=4, scaling="bands", original=10, low=3.0, high=3.0)):
        with pytest.raises(H.HxError) as e:
            KV.Rope.frequencies(**kw)
        assert e.value.code == H.HX_ERR_INVALID


def test_turns_are_exact_fractions(lib):
    """Frequencies as 64-bit fractions of a turn, rounded to the nearest, of any sign and size."""
    f = [1.0, 0.5, 1e-9, 0.0, -1.0, 100.0, 2 * math.pi]
    rope = KV.Rope(f, device="cpu")
    got = [int(t) & (1 << 64) - 1 for t in rope.turns.tolist()]
    want = [round(x / (2 * math.pi) % 1.0 * 2 ** 64) % 2 ** 64 for x in f]
    for g, w in zip(got, want):
        assert min((g - w) % 2 ** 64, (w - g) % 2 ** 64) < 2 ** 16  # what a double's turn has lost
    assert got[3] == 0 and got[0] + got[4] == 2 ** 64 and got[0] == 2935890503282001226
    for bad in ([], [math.nan], [math.inf], [1.0] * 513, [[1.0]]):
        with pytest.raises(H.HxError):
            KV.Rope(bad, device="cpu")
    with pytest.raises(H.HxError):
        KV.Rope([1.0], scale=math.inf, device="cpu")


# ---------------------------------------------------------------- logits

def _logits(**kw):
    return _set(L.hx_logits(FAKE, 100, 3, 100, KV.HX_BF16), **kw)


def _rules(**kw):
    at = [FAKE + MB * i for i in range(1, 12)]
    a = L.hx_rules(3, 20, at[0], 20, at[1], at[2], at[3], at[4], at[5], at[6], at[7], at[8], at[9], at[10], 4, 9, 3, 4)
    return _set(a, **kw)


LOGITS_BAD = [(dict(n_rows=-1), "n_rows"), (dict(n_rows=65537), "n_rows"), (dict(n_vocab=0), "n_vocab"),
              (dict(n_vocab=393217, stride=1 << 20), "n_vocab"), (dict(dtype=3), "dtype"), (dict(stride=99), "stride"),
              (dict(stride=2 ** 38), "stride"), (dict(x=None), "NULL"), (dict(x=FAKE + 1), "aligned")]
RULES_BAD = [(dict(n_rows=2), "n_rows"), (dict(history_width=-1), "history_width"), (dict(history_width=524288), "history_width"),
             (dict(history_stride=19), "history_stride"), (dict(length=None), "length"), (dict(n_bias=-1), "n_bias"),
             (dict(bias_token=None), "biases"), (dict(bias_value=None), "biases"), (dict(n_masks=0), "n_masks"),
             (dict(mask_row=None, n_masks=2), "mask_row"), (dict(mask_width=3), "fewer bits"), (dict(mask_stride=3), "mask_stride")] + \
            [({name: FAKE + 2}, "aligned") for name in ("history", "length", "prompt_len", "repetition", "presence", "frequency",
                                                        "bias_start", "bias_token", "bias_value", "mask", "mask_row")]
OUT = FAKE + 40 * MB


def test_adjust_refusals(lib):
    adjust = lambda x, r, out=OUT, stride=100, dtype=KV.HX_BF16: lib.hx_adjust(
        None if x is None else ctypes.byref(x), None if r is None else ctypes.byref(r), out, stride, dtype, None)
    _refused(lib, adjust(None, _rules()), "NULL")
    _refused(lib, adjust(_logits(), None), "NULL")
    for kw, msg in LOGITS_BAD:
        _refused(lib, adjust(_logits(**kw), _rules()), msg)
    for kw, msg in RULES_BAD:
        _refused(lib, adjust(_logits(), _rules(**kw)), msg)
    for kw, msg in [(dict(dtype=KV.HX_F16), "type"), (dict(stride=99), "out_stride"), (dict(out=None), "NULL"),
                    (dict(out=OUT + 1), "aligned"), (dict(out=FAKE + 2), "overlaps the logits"),
                    (dict(out=FAKE, stride=101), "overlaps the logits"), (dict(out=FAKE, dtype=KV.HX_F32), "overlaps the logits")]:
        _refused(lib, adjust(_logits(), _rules(), **kw), msg)
    for name in ("history", "length", "repetition", "bias_start", "bias_value", "mask", "mask_row"):
        _refused(lib, adjust(_logits(), _rules(), out=getattr(_rules(), name)), "overlaps the rules")
    assert adjust(_logits(n_rows=0, x=None), _rules(n_rows=0)) == H.HX_OK


def _pick(**kw):
    at = [FAKE + MB * i for i in range(50, 58)]
    return _set(L.hx_pick(at[0], 100, at[1], at[2], at[3], at[4], 1.0, 1.0, 0.0, 0, at[5], at[6], FAKE + 100 * MB, 1 << 30), **kw)


def test_sample_refusals(lib):
    sample = lambda x, r, p: lib.hx_sample(*(None if v is None else ctypes.byref(v) for v in (x, r, p)), None)
    _refused(lib, sample(None, _rules(), _pick()), "NULL")
    _refused(lib, sample(_logits(), _rules(), None), "NULL")
    for kw, msg in LOGITS_BAD:
        _refused(lib, sample(_logits(**kw), _rules(), _pick()), msg)
    for kw, msg in RULES_BAD:
        _refused(lib, sample(_logits(), _rules(**kw), _pick()), msg)
    for kw, msg in [(dict(noise_stride=99), "noise_stride"), (dict(noise_stride=2 ** 38), "noise_stride"), (dict(token=None), "NULL"),
                    (dict(workspace=None), "too small"), (dict(workspace_bytes=0), "too small"), (dict(workspace=FAKE + 100 * MB + 8), "16-byte"),
                    (dict(workspace=_pick().noise), "workspace overlaps"), (dict(workspace=_pick().token - 16), "workspace overlaps"),
                    (dict(workspace=_rules().mask), "workspace overlaps"), (dict(logprob=_pick().token + 4), "token and logprob"),
                    (dict(token=FAKE + 4), "overlaps what is read"), (dict(logprob=_pick().temperature), "overlaps what is read"),
                    (dict(token=_rules().history + 40), "overlaps the rules")] + \
            [({name: FAKE + 50 * MB + 2}, "aligned") for name in ("noise", "temperature", "top_k", "top_p", "min_p", "token", "logprob")]:
        _refused(lib, sample(_logits(), _rules(), _pick(**kw)), msg)
    assert sample(_logits(n_rows=0, x=None), None, _pick(workspace=None)) == H.HX_OK
    size = lambda x, r, p: lib.hx_sample_workspace(*(None if v is None else ctypes.byref(v) for v in (x, r, p)))
    need = size(_logits(), _rules(), _pick())
    _refused(lib, sample(_logits(), _rules(), _pick(workspace_bytes=need - 1)), "too small")
    assert need == size(_logits(), None, _pick()) > size(_logits(), None, _pick(noise=None)) > 0
    assert size(None, None, _pick()) == 0 and size(_logits(), None, None) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 5))
    for call in (lambda: L.adjust(x, L.Rules()), lambda: L.sample(x), lambda: L.Rules(history=torch.zeros((2, 3), dtype=torch.int32),
                                                                  length=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(H.HxError) as e:
            call()
        assert e.value.code == H.HX_ERR_INVALID and "CUDA" in str(e.value)
