"""Layouts and calls of the cache operators beside the usual ones."""
import math

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import kvcache as KV
from tests import kv_cases as P
from tests.test_gpu_kvcache import _near, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B_.build()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("q_len,max_q", [([1, 1], (1, 0)), ([9, 30], (30, 0, 200))])
@pytest.mark.parametrize("group", [1, 4])
def test_tokens_before_the_first_row_get_zeros(q_len, max_q, group):
    """A caller that attends to some rows of a step passes the rest of its row_start with the whole q."""
    g, H, D = gen(7), 2, 64
    kv, lead, tail = [30, 50], 5, 3
    table, N = P.paged(g, kv, 16)
    k, v, ks, vs = P.random_cache(g, N, H, 16, D)
    start = [lead, lead + q_len[0], lead + sum(q_len)]
    q = torch.randn((start[-1] + tail, H * group, D), generator=g, device="cuda").half()
    want = P.attend_plain(q, k, v, ks, vs, table, start, kv, D ** -0.5, True, 0)
    for mq in max_q:
        out = torch.full_like(q, math.nan)
        got, lse = KV.Cache(k, v, ks, vs).attend(q, table, i32(start), i32(kv), max_q=mq, out=out, return_lse=True)
        _near(got, lse, *want)
        for part in (slice(0, lead), slice(start[-1], None)):
            assert bool((got[part] == 0).all()) and bool((lse[part] == -math.inf).all())


def test_no_row_owns_anything():
    g = gen(3)
    table, N = P.paged(g, [30], 16)
    k, v, ks, vs = P.random_cache(g, N, 2, 16, 64)
    q = torch.randn((700, 4, 64), generator=g, device="cuda").half()
    for start in ([700, 700], [0, 0], [900, 900], [-5, -3], [300, 300]):
        out = torch.full_like(q, math.nan)
        got, lse = KV.Cache(k, v, ks, vs).attend(q, table, i32(start), i32([30]), out=out, return_lse=True)
        assert bool((got == 0).all()) and bool((lse == -math.inf).all())
