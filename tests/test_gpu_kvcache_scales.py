"""Attention over the paged cache where scales, weights and lengths leave the ordinary range, on
both of its kernels, against the plain 64-bit implementation."""
import math

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import kvcache as KV
from tests import kv_cases as P
from tests.test_gpu_kvcache import gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B_.build()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def near(got, lse, want, wlse, tol, ltol):
    """Within the bounds where the 64-bit result is a number, not a finite number where it is not."""
    num = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), num), "which results are numbers"
    e = torch.where(num, (got.double() - want).abs(), 0)
    tol = torch.where(num, tol, 0)
    assert bool((e <= tol).all()), f"out: {float((e / tol.clamp(min=1e-300)).max())} of the bound"
    empty = wlse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    e = torch.where(empty, 0, (lse.double() - wlse).abs())
    assert bool((e <= torch.where(empty, 0, ltol)).all()), f"lse: {float((e / ltol.clamp(min=1e-300)).max())} of the bound"


def check(q, cache, table, q_len, kv_len, sm, causal=True, window=0, max_q=(0,)):
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    want = P.attend_plain(q, cache.k, cache.v, cache.k_scale, cache.v_scale, table, start, kv_len, sm, causal, window)
    for mq in max_q:
        out = torch.full_like(q, math.nan)
        got, lse = cache.attend(q, table, i32(start), i32(kv_len), sm_scale=sm, causal=causal, window=window, max_q=mq,
                                out=out, return_lse=True)
        near(got, lse, *want)


# ---- blocks that no token sees, or not all tokens

FORMS = [([1, 1, 1], 2, (1, 0)), ([1, 1, 1], 12, (1,)), ([4, 3, 1], 2, (4, 0)), ([4, 2, 4], 4, (4, 0)), ([40, 1, 21], 3, (40, 0, 100))]


@pytest.mark.parametrize("scale", [math.nan, math.inf, 2.0 ** 100])
@pytest.mark.parametrize("D,B", [(64, 16), (64, 32), (128, 16), (64, 64), (128, 64)])
@pytest.mark.parametrize("q_len,group,max_q", FORMS)
def test_scales_before_the_window_take_no_part(scale, D, B, q_len, group, max_q):
    """Table entries wholly before what any token of the request sees name blocks of any contents."""
    g = gen(B + D)
    window, kv_len = 70, [300, 171, 209]
    table, N = P.paged(g, kv_len, B)
    k, v, ks, vs = P.random_cache(g, N, 2, B, D)
    for r, (n, kv) in enumerate(zip(q_len, kv_len)):
        gone = table[r, :max(0, kv - n - window + 1) // B].long()
        assert len(gone) > 0
        ks[gone], vs[gone] = scale, scale
        k.view(torch.uint8)[gone, :, ::3], v.view(torch.uint8)[gone, :, ::5] = 0x7f, 0x7f
    q = torch.randn((sum(q_len), 2 * group, D), generator=g, device="cuda").bfloat16()
    check(q, KV.Cache(k, v, ks, vs), table, q_len, kv_len, D ** -0.5, window=window, max_q=max_q)


def _one_block(scale, D, n, group, max_q, edge):
    """One block is seen by the first token of a chunk only (through the window), or by the last only: a scale that is
    no number there makes that token's result none, one far above the others' costs the other tokens nothing."""
    g, B, window = gen(D + n), 16, 20
    if edge == "first":
        kv = 16 * 3 + window + n - 2  # token 0 sees from the last position of block 2 on
        block = 2
    else:
        kv, block = 16 * 4 + 1, 4
    table, N = P.paged(g, [kv], B)
    k, v, ks, vs = P.random_cache(g, N, 2, B, D)
    b = v.view(torch.uint8)
    b[(b & 0x7f) == 0] = 0x38  # an infinite scale times zero is no number either, but times one it is infinite
    vs[table[0, block].long()] = scale
    q = torch.randn((n, 2 * group, D), generator=g, device="cuda").bfloat16()
    check(q, KV.Cache(k, v, ks, vs), table, [n], [kv], D ** -0.5, window=window, max_q=max_q)


@pytest.mark.parametrize("scale", [math.nan, math.inf, 2.0 ** 100])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group,max_q", [(4, 2, (4, 0)), (4, 4, (4,))])
@pytest.mark.parametrize("edge", ["first", "last"])
def test_a_value_scale_reaches_the_few_rows_that_see_its_block(scale, D, n, group, max_q, edge):
    _one_block(scale, D, n, group, max_q, edge)


# ---- weights that are rescaled

def one_column_cache(scores, values, D, B, k_scale=1.0, v_scale=None):
    """A cache of one request and head in which token p's score is scores[p] powers of two for a q of ones in
    its first two columns (sums of two e4m3 numbers) and whose value is values[p] in every column."""
    n = len(scores)
    blocks = -(-n // B)
    k = torch.zeros((blocks * B, D))
    hi = torch.tensor(scores, dtype=torch.float32).to(torch.float8_e4m3fn).float()
    k[:n, 0], k[:n, 1] = hi, torch.tensor(scores, dtype=torch.float32) - hi
    v = torch.zeros((blocks * B, D))
    v[:n] = torch.tensor(values, dtype=torch.float32)[:, None]
    f8 = lambda x: x.view(blocks, 1, B, D).to(torch.float8_e4m3fn).cuda()
    assert torch.equal(f8(k).float().cpu().view(-1, D), k)
    vs = torch.ones((blocks, 1)) if v_scale is None else torch.tensor(v_scale, dtype=torch.float32).view(blocks, 1)
    return KV.Cache(f8(k), f8(v), torch.full((blocks, 1), k_scale, device="cuda"), vs.cuda()), i32([list(range(blocks))])


def two_columns(n, heads, D, dtype):
    q = torch.zeros((n, heads, D), dtype=dtype, device="cuda")
    q[:, :, :2] = 1
    return q


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (130, (0, 130))])
@pytest.mark.parametrize("jump", [11.875, 20.875, 24.875, 26.875, 29.875])
def test_weights_keep_their_bits_when_the_maximum_moves(D, n, max_q, jump):
    """64 tokens at 2^9.875 above the first 32 of their tile, then one far above those: each of the 64 counts little,
    but their values are all that there is."""
    scores = [0.0] * 32 + [9.875] * 64 + [jump] + [0.0] * 31
    values = [0.0] * 32 + [1.0] * 64 + [0.0] * 32
    cache, table = one_column_cache(scores, values, D, 16)
    check(two_columns(n, 1, D, torch.float16), cache, table, [n], [128], math.log(2), causal=False, max_q=max_q)


# ---- sums of weights under scales far apart

def _far(first, other, shift, D, blocks=64, B=16):
    """`blocks` blocks of values zero, as hx_kv_append leaves them (scale 2^-100), and one token of values one
    under the scale `other` whose score is `shift` powers of two above theirs; it comes first or last."""
    n = blocks * B
    scores, values, vs = [0.0] * n, [0.0] * n, [2.0 ** -100] * blocks
    own = [shift] + [-100.0] * (B - 1)
    val = [1.0] * B
    if first:
        return one_column_cache(own + scores, val + values, D, B, v_scale=[other] + vs)
    return one_column_cache(scores + own, values + val, D, B, v_scale=vs + [other])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (150, (0, 150))])
@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("other,shift", [(1.0, 7.0), (2.0 ** 20, 7.0), (2.0 ** 20, -3.0), (2.0 ** 60, 9.0), (2.0 ** 110, 0.0), (2.0 ** 110, 26.0)])
def test_tokens_of_zeros_count_under_any_scale(D, n, max_q, first, other, shift):
    cache, table = _far(first, other, shift, D)
    q = two_columns(n, 1, D, torch.bfloat16)
    check(q, cache, table, [n], [65 * 16], math.log(2), causal=False, max_q=max_q)


@pytest.mark.parametrize("n,max_q", [(1, (1,)), (20, (0, 20)), (150, (0,))])
def test_long_requests_with_scales_far_apart_are_joined(n, max_q):
    """The same over many blocks of the grid, whose partial results are joined: 20000 tokens of zeros, then values
    under 2^20 and under 2^-60, and in the middle."""
    B, D, blocks = 16, 64, 1250
    rng = np.random.default_rng(n)
    scores, values = [0.0] * (blocks * B), [0.0] * (blocks * B)
    vs = [2.0 ** -100] * blocks
    for b, s, x in ((3, 2.0 ** -60, 9.0), (600, 2.0 ** 20, 7.0), (601, 2.0 ** -100, 11.0), (1249, 2.0 ** 30, -4.0)):
        vs[b] = s
        scores[b * B], values[b * B:(b + 1) * B] = x, rng.choice([-1.5, 1.0, 2.0], B).tolist()
    cache, table = one_column_cache(scores, values, D, B, v_scale=vs)
    check(two_columns(n, 2, D, torch.bfloat16), cache, table, [n], [blocks * B], math.log(2), causal=False, max_q=max_q)


@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (150, (0, 150))])
def test_scales_of_every_size_side_by_side(n, max_q):
    """Every block and head under a power of two from 2^-100 to 2^100, rows that see different ones of them."""
    g, B, H, D = gen(n), 16, 2, 64
    kv = [700, 333]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, H, B, D)
    vs.copy_(torch.exp2(torch.randint(-100, 101, vs.shape, generator=g, device="cuda").float()))
    ks.fill_(2.0 ** -9)
    q = torch.randn((2 * n, 2 * H, D), generator=g, device="cuda").bfloat16()
    for window in (0, 40):
        check(q, KV.Cache(k, v, ks, vs), table, [n, n], kv, D ** -0.5, window=window, max_q=max_q)


# ---- scales that are small, zero or no numbers

@pytest.mark.parametrize("scale", [math.nan, math.inf, 2.0 ** 100])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group,max_q", [(4, 4, (0,)), (20, 3, (20, 0, 100))])
@pytest.mark.parametrize("edge", ["first", "last"])
def test_a_value_scale_reaches_the_many_rows_that_see_its_block(scale, D, n, group, max_q, edge):
    _one_block(scale, D, n, group, max_q, edge)


@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (150, (0, 150))])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -110, 3 * 2.0 ** -108, 2.0 ** -101])
def test_small_value_scales_are_followed(n, max_q, scale):
    """The whole cache under one small scale, and one block under it beside ordinary ones."""
    g, B, D = gen(n), 16, 64
    kv = [260]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, 1, B, D)
    q = torch.randn((n, 3, D), generator=g, device="cuda").bfloat16()
    one = vs.clone()
    one[table[0, 4].long()] = scale
    for s in (torch.full_like(vs, scale), one):
        check(q, KV.Cache(k, v, ks, s), table, [n], kv, D ** -0.5, max_q=max_q)


@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (150, (0, 150))])
@pytest.mark.parametrize("scale", [math.nan, math.inf])
def test_a_request_whose_scales_are_all_no_numbers(n, max_q, scale):
    g, B, D = gen(n), 16, 64
    kv = [100]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, 1, B, D)
    b = v.view(torch.uint8)
    b[(b & 0x7f) == 0] = 0x38
    q = torch.randn((n, 3, D), generator=g, device="cuda").bfloat16()
    check(q, KV.Cache(k, v, ks, torch.full_like(vs, scale)), table, [n], kv, D ** -0.5, max_q=max_q)


# ---- infinite scores

@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (90, (0, 90))])
@pytest.mark.parametrize("kv", [100, 300, 5000])
def test_infinite_scores_give_no_number(n, max_q, kv):
    """exp(inf - inf) is no number: not zeros, which is what a token that sees nothing gets."""
    D, B = 64, 16
    cache, table = one_column_cache([1.0] * kv, [1.0] * kv, D, B)
    q = torch.zeros((n, 4, D), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1
    q[n // 2, 1, 0] = math.inf
    for mq in max_q:
        got, lse = cache.attend(q, table, i32([0, n]), i32([kv]), max_q=mq, return_lse=True)
        want = torch.zeros_like(got, dtype=torch.bool)
        want[n // 2, 1] = True
        assert torch.equal(torch.isnan(got), want)
        assert not bool(torch.isfinite(lse[n // 2, 1])) and int((~torch.isfinite(lse)).sum()) == 1


@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (150, (0, 150))])
@pytest.mark.parametrize("scale", [2.0 ** 100, 2.0 ** -100, 3 * 2.0 ** 60])
@pytest.mark.parametrize("window", [0, 1, 2])
def test_sums_are_no_worse_under_large_or_small_scales(n, max_q, scale, window):
    """The values' scale is no part of the softmax, and must not cost its sum any bits either."""
    g, B, D = gen(n), 16, 64
    kv = [300]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, 2, B, D)
    q = torch.randn((n, 48, D), generator=g, device="cuda").bfloat16()
    check(q, KV.Cache(k, v, ks, torch.full_like(vs, scale)), table, [n], kv, 1e-5, window=window, max_q=max_q)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20)), (150, (0,))])
@pytest.mark.parametrize("tokens", [100, 1000000])
def test_sums_of_large_values_stay_in_range(D, n, max_q, tokens):
    """Before they are divided, sums are larger than results by as many tokens as there are and by what the maximum lags."""
    B = 16
    blocks = -(-tokens // B)
    cache, table = one_column_cache([0.0] * 16 + [7.875] * (tokens - 16), [448.0] * tokens, D, B, v_scale=[2.0 ** 100] * blocks)
    check(two_columns(n, 1, D, torch.bfloat16), cache, table, [n], [tokens], math.log(2), causal=False, max_q=max_q)


@pytest.mark.parametrize("n,max_q", [(1, (1, 0)), (20, (0, 20, 200)), (150, (0, 150))])
@pytest.mark.parametrize("one,other", [(3 * 2.0 ** 97, 3 * 2.0 ** 97), (1.0, 3 * 2.0 ** 37), (5 * 2.0 ** -105, 3 * 2.0 ** -69)])
@pytest.mark.parametrize("window", [0, 1, 2])
def test_sums_are_no_worse_under_scales_that_differ(n, max_q, one, other, window):
    """Nor under scales that are no powers of two, or that differ from block to block."""
    g, B, D = gen(n), 16, 64
    kv = [300]
    table, N = P.paged(g, kv, B)
    k, v, ks, vs = P.random_cache(g, N, 2, B, D)
    vs.fill_(one)
    vs[table[0, 1:18:2].long()] = other
    q = torch.randn((n, 48, D), generator=g, device="cuda").bfloat16()
    check(q, KV.Cache(k, v, ks, vs), table, [n], kv, 1e-5, window=window, max_q=max_q)
