"""The cache operators without a GPU: struct layouts, refusals before any launch,
and the tests' own plain implementations."""
import ctypes
import os
import re
import subprocess
import threading

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import kvcache as KV
from tests import kv_cases as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = (KV.hx_kv_map_args, KV.hx_kv_cache, KV.hx_kv_new, KV.hx_kv_query)


@pytest.fixture(scope="module")
def lib():
    B_.build()
    return KV.load()


def test_both_builds_export_what_the_header_declares(lib):
    text = open(os.path.join(ROOT, "include", "hxkv.h")).read()
    names = sorted(set(re.findall(r"^\s*(?:int|int64_t)\s+(hx_kv_\w+)\s*\(", text, re.M)))
    assert names == ["hx_kv_append", "hx_kv_attend", "hx_kv_attend_workspace", "hx_kv_map", "hx_kv_max_runs"]
    for n in names:
        assert hasattr(lib, n) and hasattr(H.load_checked(), n)


def test_struct_layout_matches_binding(tmp_path):
    lines = "".join(f'printf("{s.__name__} %zu\\n", sizeof({s.__name__}));\n' + "".join(
        f'printf("{s.__name__}.{f} %zu\\n", offsetof({s.__name__}, {f}));\n' for f, _ in s._fields_) for s in STRUCTS)
    src = tmp_path / "probe.c"
    src.write_text('#include <stdio.h>\n#include "hxkv.h"\nint main(void) {\n' + lines + "return 0;\n}\n")
    exe = tmp_path / "probe"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    by = {s.__name__: s for s in STRUCTS}
    for line in subprocess.check_output([str(exe)], text=True).splitlines():
        name, size = line.split()
        s, _, f = name.partition(".")
        assert (getattr(by[s], f).offset if f else ctypes.sizeof(by[s])) == int(size), name


def _set(struct, **kw):
    s = type(struct)()
    ctypes.pointer(s)[0] = struct
    for k, v in kw.items():
        setattr(s, k, v)
    return s


FAKE = 1 << 20  # an aligned address; nothing is launched with it


def _cache(**kw):
    return _set(KV.hx_kv_cache(FAKE, FAKE, FAKE, FAKE, 4 * 32 * 64, 4, 10, 4, 32, 64), **kw)


def _refused(lib, rc, msg):
    err = lib.hx_last_error().decode()
    assert rc == H.HX_ERR_INVALID and msg in err, (rc, err)


CACHE_BAD = [(dict(k=None), "NULL"), (dict(v_scale=None), "NULL"), (dict(n_blocks=0), "n_blocks"),
             (dict(n_kv_heads=0), "n_kv_heads"), (dict(block_tokens=48), "block_tokens"), (dict(head_dim=96), "head_dim"),
             (dict(k=FAKE + 8), "aligned"), (dict(k_scale=FAKE + 2), "aligned"), (dict(block_stride=4 * 32 * 64 - 16), "block_stride"),
             (dict(block_stride=4 * 32 * 64 + 8), "block_stride"), (dict(scale_stride=3), "scale_stride")]


def test_map_refusals(lib):
    good = KV.hx_kv_map_args(3, 10, 32, 8, 4, 6, 4, *[FAKE] * 10, FAKE + 64)
    for kw, msg in [(dict(n_rows=0), "n_rows"), (dict(n_rows=65537), "n_rows"), (dict(n_tokens=-1), "n_tokens"),
                    (dict(n_tokens=2 ** 30 + 1), "n_tokens"), (dict(block_tokens=0), "block_tokens"),
                    (dict(n_blocks=0), "n_blocks"), (dict(table_width=0), "table_width"),
                    (dict(table_width=2 ** 23 + 1, table_stride=2 ** 24), "table_width"),
                    (dict(table_stride=3), "table_stride"), (dict(n_runs=5), "n_runs"), (dict(held=None), "NULL"),
                    (dict(slots=None), "NULL"), (dict(ring_state_out=FAKE), "ring_state_out"),
                    (dict(runs=FAKE + 4), "aligned")]:
        a = _set(good, **kw)
        _refused(lib, lib.hx_kv_map(ctypes.byref(a), None), msg)
    _refused(lib, lib.hx_kv_map(None, None), "NULL")


def test_append_refusals(lib):
    good = KV.hx_kv_new(FAKE, FAKE, 256, 64, 256, 64, 10, KV.HX_BF16, FAKE, 3)
    for kw, msg in CACHE_BAD:
        c = _cache(**kw)
        _refused(lib, lib.hx_kv_append(ctypes.byref(c), ctypes.byref(good), None), msg)
    c = _cache()
    for kw, msg in [(dict(n_tokens=-1), "n_tokens"), (dict(n_runs=-1), "n_runs"), (dict(dtype=3), "dtype"),
                    (dict(k=None), "NULL"), (dict(runs=None), "NULL"), (dict(v=FAKE + 2), "aligned"),
                    (dict(k_token_stride=260), "strides"), (dict(v_head_stride=4), "strides"),
                    (dict(dtype=KV.HX_F32, v_head_stride=2), "strides"), (dict(n_runs=2 ** 28), "n_runs")]:
        a = _set(good, **kw)
        _refused(lib, lib.hx_kv_append(ctypes.byref(c), ctypes.byref(a), None), msg)
    _refused(lib, lib.hx_kv_append(None, ctypes.byref(good), None), "NULL")
    _refused(lib, lib.hx_kv_append(ctypes.byref(c), None, None), "NULL")
    for kw in (dict(n_tokens=0), dict(n_runs=0)):  # nothing to do
        a = _set(good, **kw)
        assert lib.hx_kv_append(ctypes.byref(c), ctypes.byref(a), None) == H.HX_OK


def test_attend_refusals(lib):
    good = KV.hx_kv_query(FAKE, FAKE, None, 512, 64, 512, 64, 10, 8, KV.HX_F16, 3, FAKE, FAKE, FAKE, 4, 4, 1, 1, 0, 0.125,
                          FAKE, 1 << 40)
    for kw, msg in CACHE_BAD:
        c = _cache(**kw)
        _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(good), None), msg)
    c = _cache()
    for kw, msg in [(dict(n_tokens=-1), "n_tokens"), (dict(n_rows=0), "n_rows"), (dict(n_rows=65537), "n_rows"),
                    (dict(n_heads=6), "n_heads"), (dict(n_heads=0), "n_heads"), (dict(n_heads=4 * 129), "n_heads"),
                    (dict(dtype=KV.HX_F32), "dtype"), (dict(max_q=-1), "max_q"), (dict(causal=2), "causal"),
                    (dict(window=-1), "window"), (dict(sm_scale=float("nan")), "sm_scale"), (dict(q=None), "NULL"),
                    (dict(kv_len=None), "NULL"), (dict(block_table=None), "NULL"), (dict(table_width=0), "table_width"),
                    (dict(table_stride=3), "table_stride"), (dict(q=FAKE + 2), "aligned"), (dict(out=FAKE + 8), "aligned"),
                    (dict(q_head_stride=4), "strides"), (dict(out_token_stride=514), "strides")]:
        a = _set(good, **kw)
        _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(a), None), msg)
    need = ctypes.c_int64()
    assert lib.hx_kv_attend_workspace(ctypes.byref(c), ctypes.byref(good), ctypes.byref(need)) == H.HX_OK
    if need.value:
        a = _set(good, workspace_bytes=need.value - 1)
        _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(a), None), "workspace")
        a = _set(good, workspace=None)
        _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(a), None), "workspace")
    a = _set(good, n_tokens=0)
    assert lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(a), None) == H.HX_OK


def test_limits_refused(lib):
    a = KV.hx_kv_map_args(3, 10, 32, 8, 4, 6, 4, *[FAKE] * 10, FAKE + 64)
    _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, counts=FAKE + 8)), None), "aligned")
    c = _cache()
    q = KV.hx_kv_query(FAKE, FAKE, None, 512, 64, 512, 64, 10, 8, KV.HX_F16, 3, FAKE, FAKE, FAKE, 4, 4, 1, 1, 0, 0.125,
                       FAKE, 1 << 40)
    for kw, msg in [(dict(n_tokens=2 ** 29 + 1), "2^30"), (dict(workspace=FAKE + 16), "32-byte"), (dict(q_token_stride=-512), "2^38"),
                    (dict(q_head_stride=2 ** 38 + 8), "2^38"), (dict(table_width=2 ** 23 + 1, table_stride=2 ** 24), "table_width")]:
        _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(_set(q, **kw)), None), msg)


def test_binding_refuses_host_tensors():
    z = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(H.HxError) as e:
        KV.map_step(z, z, z[None], z, z.long(), 1, 16)
    assert e.value.code == H.HX_ERR_INVALID and "CUDA" in str(e.value)
    f = torch.zeros((2, 1, 16, 64), dtype=torch.uint8)
    with pytest.raises(H.HxError):
        KV.Cache(f.view(torch.float8_e4m3fn), f.view(torch.float8_e4m3fn), torch.ones(2, 1), torch.ones(2, 1))


def test_max_runs_agrees(lib):
    for n, t, b in ((1, 0, 16), (1, 1, 16), (5, 3, 64), (3, 1000, 32), (65536, 1 << 30, 16)):
        assert lib.hx_kv_max_runs(n, t, b) == KV.max_runs(n, t, b)


def test_plain_e4m3_agrees_with_the_type():
    bits = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(bits).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(P.GRID, want, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).normal(0, 2.0 ** e, 4000) for e in range(-12, 9)])
    mid = (P._POS[1:] + P._POS[:-1]) / 2
    x = np.concatenate([x, mid, -mid, P._POS]).astype(np.float32)
    t = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(P.to_e4m3(x), t)


def test_attend_status_refused_where_it_cannot_be_written(lib):
    c = _cache()
    q = KV.hx_kv_query(FAKE, FAKE, None, 512, 64, 512, 64, 10, 8, KV.HX_F16, 3, FAKE, FAKE, FAKE, 4, 4, 1, 1, 0, 0.125,
                       FAKE, 1 << 40)
    _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(_set(q, status=FAKE + 2)), None), "status")


class _Interleaved:
    """Stands in for the library: notes which workspaces are in use by calls that have not returned."""

    def __init__(self):
        self.gate, self.busy, self.clash = threading.Barrier(2), [], False

    def hx_kv_attend_workspace(self, cache, query, need):
        need._obj.value = 64
        return H.HX_OK

    def hx_kv_attend(self, cache, query, stream):
        work = query._obj.workspace
        self.clash |= work in self.busy
        self.busy.append(work)
        try:  # the launches of one call take a while; the other thread comes in here if nothing holds it
            self.gate.wait(0.5)
        except threading.BrokenBarrierError:
            pass
        self.busy.remove(work)
        return H.HX_OK


def test_calls_of_two_threads_do_not_share_a_workspace_at_a_time(monkeypatch):
    """A call's kernels hand partial results on through its workspace: launches of two calls on one stream must not
    alternate."""
    class On:
        def __enter__(self):
            return 0

        def __exit__(self, *exc):
            pass

    monkeypatch.setattr(KV, "_want", lambda *a: None)
    monkeypatch.setattr(KV, "_dense", lambda *a: None)
    monkeypatch.setattr(KV, "_on", lambda *a: On())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    fake = _Interleaved()
    monkeypatch.setattr(KV, "load", lambda: fake)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, **{k: v for k, v in kw.items() if k != "device"}))
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, **kw: zeros(*a, **{k: v for k, v in kw.items() if k != "pin_memory"}))
    f = empty((2, 1, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    cache = KV.Cache(f, f.clone(), torch.ones(2, 1), torch.ones(2, 1))
    q, i32 = empty((1, 2, 64), dtype=torch.float16), torch.int32
    args = (q, zeros((1, 2), dtype=i32), zeros(2, dtype=i32), zeros(1, dtype=i32))
    threads = [threading.Thread(target=cache.attend, args=args) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fake.clash


def _map_args(**kw):
    """Arguments of a map call with every array at an address of its own."""
    a = KV.hx_kv_map_args(3, 10, 32, 8, 4, 6, 4, *[FAKE + 4096 * i for i in range(11)])
    return _set(a, **kw)


def test_map_refuses_runs_without_an_array(lib):
    """Runs are cleared up to their length even where the step has no tokens."""
    for kw in (dict(n_tokens=0, runs=None), dict(n_tokens=0, n_runs=1, runs=None, slots=None), dict(runs=None)):
        _refused(lib, lib.hx_kv_map(ctypes.byref(_map_args(**kw)), None), "NULL")


@pytest.mark.parametrize("name", ["held", "add", "block_table", "ring", "row_start", "kv_len"])
def test_map_refuses_misaligned_ints(lib, name):
    a = _map_args()
    _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, **{name: getattr(a, name) + 2})), None), "aligned")


@pytest.mark.parametrize("name", ["ring_state", "ring_state_out", "slots"])
def test_map_refuses_misaligned_long_ints(lib, name):
    a = _map_args()
    _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, **{name: getattr(a, name) + 4})), None), "aligned")


@pytest.mark.parametrize("name", ["lse", "row_start", "kv_len", "block_table"])
def test_attend_refuses_misaligned_arrays(lib, name):
    q = KV.hx_kv_query(FAKE, FAKE, None, 512, 64, 512, 64, 10, 8, KV.HX_F16, 3, FAKE, FAKE, FAKE, 4, 4, 1, 1, 0, 0.125,
                       FAKE, 1 << 40)
    c = _cache()
    _refused(lib, lib.hx_kv_attend(ctypes.byref(c), ctypes.byref(_set(q, **{name: FAKE + 2})), None), "aligned")


@pytest.mark.parametrize("out,into", [("kv_len", "held"), ("kv_len", "add"), ("row_start", "held"), ("slots", "add"),
                                      ("runs", "ring"), ("counts", "ring_state"), ("ring_state_out", "held"),
                                      ("kv_len", "block_table")])
def test_map_refuses_to_write_over_what_it_reads(lib, out, into):
    """Blocks of threads read all lengths while others already write theirs."""
    a = _map_args()
    _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, **{out: getattr(a, into)})), None), "overlap")
    if (out, into) == ("kv_len", "held"):  # its last entry only
        _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, kv_len=a.held + 8)), None), "overlap")
        _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, kv_len=a.held - 8)), None), "overlap")


def test_map_lets_outputs_lie_between_the_rows_of_a_table(lib):
    """A strided table's rows are what may not be written over, not what lies between them."""
    a = _map_args(table_stride=64)
    gap = a.block_table + 4 * 16
    row = a.block_table + 4 * 64
    _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, counts=gap, kv_len=row + 12)), None), "overlap")
    _refused(lib, lib.hx_kv_map(ctypes.byref(_set(a, row_start=row + 16, kv_len=a.held)), None), "held")


@pytest.mark.parametrize("value", [2 ** 32, 2 ** 32 + 5, -2 ** 32 + 3, 2 ** 31])
def test_binding_refuses_whole_numbers_past_32_bits(value):
    """ctypes would cut them off: a window of 2^32 + 5 would be one of 5."""
    cache = object.__new__(KV.Cache)
    for kw in (dict(window=value), dict(max_q=value)):
        with pytest.raises(H.HxError) as e:
            cache.attend(None, None, None, None, **kw)
        assert e.value.code == H.HX_ERR_INVALID and list(kw)[0] in str(e.value)
    z = torch.zeros(3, dtype=torch.int32)
    for args, name in (((value, 16), "n_tokens"), ((1, value), "block_tokens"), ((1, 0), "block_tokens")):
        with pytest.raises(H.HxError) as e:
            KV.map_step(z, z, z[None], z, z.long(), *args)
        assert e.value.code == H.HX_ERR_INVALID and name in str(e.value)


def test_workspaces_of_streams_gone_by_are_given_back(monkeypatch):
    """The cache keeps one for each of the streams used last, not for every stream that there ever was."""
    class On:
        def __init__(self, device, stream):
            self.stream = stream

        def __enter__(self):
            return self.stream

        def __exit__(self, *exc):
            pass

    class Lib:
        used = []

        def hx_kv_attend_workspace(self, cache, query, need):
            need._obj.value = 64
            return H.HX_OK

        def hx_kv_attend(self, cache, query, stream):
            self.used.append(query._obj.workspace)
            return H.HX_OK

    lib = Lib()
    monkeypatch.setattr(KV, "_want", lambda *a: None)
    monkeypatch.setattr(KV, "_dense", lambda *a: None)
    monkeypatch.setattr(KV, "_on", On)
    monkeypatch.setattr(KV, "load", lambda: lib)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, **kw: zeros(*a, **{k: v for k, v in kw.items() if k != "pin_memory"}))
    f = torch.empty((2, 1, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    cache = KV.Cache(f, f.clone(), torch.ones(2, 1), torch.ones(2, 1))
    q, i32 = torch.empty((1, 2, 64), dtype=torch.float16), torch.int32
    args = (q, zeros((1, 2), dtype=i32), zeros(2, dtype=i32), zeros(1, dtype=i32))
    for handle in range(100):
        cache.attend(*args, stream=7)
        cache.attend(*args, stream=1000 + handle)
    assert len(cache._work) <= 16 and len(set(lib.used[::2])) == 1
