"""Waits that run out: the attention's kernels built so that no wait waits.  A block gives up at its first one, what
it had left to compute is NaN, the status says so, and the GPU goes on."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import kvcache as KV
from tests import kv_cases as P
from tests.test_gpu_kvcache import _near, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def impatient(tmp_path_factory):
    B_.build()
    out = str(tmp_path_factory.mktemp("waits") / "libhxsim_impatient.so")
    lib = ctypes.CDLL(B_.build(out=out, extra=("-DHX_KV_WAIT_CYCLES=0",), checked=False))
    lib.hx_last_error.restype = ctypes.c_char_p
    for name in ("hx_kv_attend_workspace", "hx_kv_attend"):
        getattr(lib, name).argtypes = [ctypes.c_void_p] * 3
    return lib


@pytest.mark.parametrize("D,B", [(64, 16), (128, 64)])
@pytest.mark.parametrize("q_len,kv_len,group,max_q", [([1, 1, 1], [3000, 0, 70], 4, 1),            # few rows
                                                      ([1, 1, 1], [3000, 0, 70], 12, 1),
                                                      ([300, 1, 90], [700, 20, 5000], 4, 0),       # many rows
                                                      ([30, 1, 9], [700, 20, 5000], 4, 30)])       # by turns
def test_a_wait_that_runs_out_leaves_nan_and_a_status(impatient, D, B, q_len, kv_len, group, max_q):
    g, H_ = gen(D), 2
    table, N = P.paged(g, kv_len, B)
    k, v, ks, vs = P.random_cache(g, N, H_, B, D)
    cache = KV.Cache(k, v, ks, vs)
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    q = torch.randn((int(start[-1]), H_ * group, D), generator=g, device="cuda").half()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    want, wlse, tol, ltol = P.attend_plain(q, k, v, ks, vs, table, start, kv_len, D ** -0.5, True, 0)
    args = (q, table, i32(start), i32(kv_len))
    cache.check()
    patient, cache.lib = cache.lib, impatient
    got, lse = cache.attend(*args, max_q=max_q, return_lse=True)
    torch.cuda.synchronize()
    with pytest.raises(H.HxError, match="ran out"):
        cache.check()
    lost = torch.isnan(got).any(2)
    assert bool(lost.any()) and torch.equal(lost, torch.isnan(got).all(2)) and torch.equal(lost, torch.isnan(lse))
    sees = wlse > -float("inf")
    assert not bool((lost & ~sees).any())
    kept = ~lost
    _near(got[kept], lse[kept], want[kept], wlse[kept], tol[kept], ltol[kept])
    cache.lib = patient
    cache._status.zero_()
    got, lse = cache.attend(*args, max_q=max_q, return_lse=True)
    _near(got, lse, want, wlse, tol, ltol)
    torch.cuda.synchronize()
    cache.check()
