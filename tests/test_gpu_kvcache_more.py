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


@pytest.mark.parametrize("group,chunk", [(4, 5), (4, 32), (16, 8), (3, 42), (1, 100)])
@pytest.mark.parametrize("where", [0.5, 0.95])
def test_nan_with_a_bound_on_the_tokens(group, chunk, where):
    """A NaN in the cache reaches the tokens that see it and no others, where max_q says that no request has more tokens than
    a half of an item: also one that the half which does not write the result has taken."""
    D, B = 64, 16
    for which in (0, 1):
        for kv0 in (chunk + 45, chunk + 300):
            g = gen(6)
            kv = [kv0, 80]
            table, N = P.paged(g, kv, B)
            k, v, ks, vs = P.random_cache(g, N, 2, B, D)
            p = kv0 - max(1, int(chunk * (1 - where)))
            far = kv0 // 3  # on another head
            (k, v)[which].view(torch.uint8)[table[0, p // B].long(), 1, p % B, 9] = 0x7f
            (k, v)[which].view(torch.uint8)[table[0, far // B].long(), 0, far % B, 11] = 0xff
            q = torch.randn((chunk + 1, 2 * group, D), generator=g, device="cuda").half()
            got, lse = KV.Cache(k, v, ks, vs).attend(q, table, i32([0, chunk, chunk + 1]), i32(kv), max_q=chunk, return_lse=True)
            sees = torch.zeros((chunk + 1, 2 * group), dtype=torch.bool, device="cuda")
            sees[p - (kv0 - chunk):chunk, group:] = True
            sees[max(0, far - (kv0 - chunk)):chunk, :group] = True
            assert torch.equal(torch.isnan(got).any(2), sees)
            assert torch.equal(torch.isnan(lse), sees & (which == 0))
            if which == 1:
                cols = torch.zeros_like(got, dtype=torch.bool)
                cols[:, group:, 9], cols[:, :group, 11] = sees[:, group:], sees[:, :group]
                assert torch.equal(torch.isnan(got), cols)
            else:
                assert torch.equal(torch.isnan(got).all(2), sees)


@pytest.mark.parametrize("positions", [12, 40])
def test_more_nan_than_the_list_holds(positions):
    """NaN at many positions of one item, seen by some rows each."""
    g, B, D, n = gen(13), 16, 64, 30
    kv = [400]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, 1, B, D)
    p = torch.randperm(400, generator=g, device="cuda")[:positions]
    col = torch.randint(0, D, (positions,), generator=g, device="cuda")
    v.view(torch.uint8)[table[0, p // B].long(), 0, p % B, col] = 0x7f
    q = torch.randn((n, 4, D), generator=g, device="cuda").half()
    for mq in (n, 0):
        got = KV.Cache(k, v, ks, vs).attend(q, table, i32([0, n]), i32(kv), max_q=mq)
        want = torch.zeros((n, D), dtype=torch.bool, device="cuda")
        for i in range(n):
            want[i, col[p <= 400 - n + i]] = True
        assert torch.equal(torch.isnan(got), want[:, None].expand(n, 4, D))


LAYOUTS = [([1, 1, 1], (1, 0)), ([4, 2, 3], (4, 0)), ([40, 1, 70], (70, 0)), ([20, 6, 30], (30, 0))]


@pytest.mark.parametrize("q_len,max_q", LAYOUTS)
@pytest.mark.parametrize("D,B,group", [(64, 16, 4), (128, 64, 3), (64, 128, 1)])
@pytest.mark.parametrize("layout", ["interleaved", "heads outermost", "both"])
def test_attend_over_other_layouts(q_len, max_q, D, B, group, layout):
    """k and v side by side in one tensor, with their scales; q (and out) with heads outermost."""
    g, H, dtype = gen(D + B), 2, torch.bfloat16
    kv = [200, 77, 310]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, H, B, D)
    cache = KV.Cache(k, v, ks, vs)
    if layout != "heads outermost":
        both = torch.empty((N, 2, H, B, D), dtype=torch.uint8, device="cuda")
        both[:, 0], both[:, 1] = k.view(torch.uint8), v.view(torch.uint8)
        both = both.view(torch.float8_e4m3fn)
        scales = torch.stack([ks, vs], 1)
        cache = KV.Cache(both[:, 0], both[:, 1], scales[:, 0], scales[:, 1])
    T = sum(q_len)
    q = torch.randn((T, H * group, D), generator=g, device="cuda").to(dtype)
    out = None
    if layout != "interleaved":
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
        out = torch.full((H * group, T, D), math.nan, dtype=dtype, device="cuda").transpose(0, 1)
        assert q.stride(0) < q.stride(1) or T == 1
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    want = P.attend_plain(q, k, v, ks, vs, table, start, kv, D ** -0.5, True, 0)
    for mq in max_q:
        got, lse = cache.attend(q, table, i32(start), i32(kv), max_q=mq, out=out, return_lse=True)
        _near(got, lse, *want)


@pytest.mark.parametrize("q_len,max_q", LAYOUTS)
def test_attend_with_one_q_for_all_tokens_or_heads(q_len, max_q):
    """Strides of zero: a q that is broadcast over the tokens or over the heads."""
    g, H, group, D, B = gen(5), 2, 3, 64, 32
    kv = [200, 77, 310]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, H, B, D)
    T = sum(q_len)
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    for q in (torch.randn((1, H * group, D), generator=g, device="cuda").half().expand(T, -1, -1),
              torch.randn((T, 1, D), generator=g, device="cuda").half().expand(-1, H * group, -1)):
        want = P.attend_plain(q, k, v, ks, vs, table, start, kv, D ** -0.5, True, 0)
        for mq in max_q:
            got, lse = KV.Cache(k, v, ks, vs).attend(q, table, i32(start), i32(kv), max_q=mq, return_lse=True)
            _near(got, lse, *want)
