"""Sampling on the GPU where filters meet: calls whose rows leave fewer tokens than they ask for, against the plain
64-bit implementation."""
import math

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import logits as L
from tests import step_cases as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B_.build()


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# A weight within its bin is rounded to 2^-18 of that of the bin's middle, so by 2^-19, and is at least exp(-1/32) of it: 2^-18.95 of the
# weight; its series and its bin's factor are off by 2^-22 together.  The sum up to the border and the sum that top_p is of: twice that,
# below 2^-17 of top_p.
SHARE = 2.0 ** -17


def _check(x, noise, T, k, p, allowed=None):
    """Rows of x [n, V] with numbers T, k, p for each; allowed [n, V]: the mask's tokens."""
    n, V = x.shape
    rules, z = None, x
    if allowed is not None:
        words = (V + 31) // 32
        bits = np.zeros((n, words * 32), bool)
        bits[:, :V] = allowed
        w = (bits.reshape(n, words, 32) * (1 << np.arange(32, dtype=np.int64))).sum(-1).astype(np.uint32).view(np.int32)
        rules, z = L.Rules(mask=_cuda(w)), np.where(allowed, x, -np.inf)
    token, logprob = L.sample(_cuda(x), _cuda(noise), temperature=_cuda(T), top_k=_cuda(k), top_p=_cuda(p), rules=rules)
    token, logprob = token.cpu().numpy(), logprob.cpu().numpy()
    wrong = []
    for r in range(n):
        args = z[r], noise[r], float(T[r]), int(k[r])
        if P.sample_plain(*args, float(p[r]), 0.0)[0] == token[r]:
            continue
        if token[r] not in [P.sample_plain(*args, float(p[r]) * (1 + d), 0.0)[0] for d in (-SHARE, SHARE)]:
            wrong.append(r)
    assert not wrong, (len(wrong), n, wrong[:5], token[wrong[:5]], k[wrong[:5]], p[wrong[:5]])
    for r in range(0, n, 7):
        t, lp, tol = P.sample_plain(z[r], noise[r], float(T[r]), int(k[r]), float(p[r]), 0.0)
        assert token[r] != t or abs(logprob[r] - lp) <= tol


def _rows(rng, n, V, k):
    x = (3 * rng.standard_normal((n, V))).astype(np.float32)
    noise = rng.exponential(size=(n, V)).astype(np.float32)
    return (x, noise, rng.choice([0.5, 1.0, 1.5], n).astype(np.float32), np.full(n, k, np.int32) if np.isscalar(k) else k,
            rng.uniform(0.3, 0.95, n).astype(np.float32))


@pytest.mark.parametrize("V", [3, 8, 12, 40, 100])
@pytest.mark.parametrize("more", [0, 1, 38, 5000])
def test_top_k_above_a_small_vocabulary_with_top_p(V, more):
    """top_k of all tokens or more leaves them all, whatever top_p does then."""
    rng = np.random.default_rng(V + more)
    _check(*_rows(rng, 600, V, V + more))


@pytest.mark.parametrize("V", [50, 5003, 40000])
def test_top_k_above_what_a_mask_leaves_with_top_p(V):
    """Grammar masks that allow 1 to 40 tokens, top_k below and above that."""
    rng = np.random.default_rng(V)
    n = 1500 if V < 10000 else 300
    allowed = np.zeros((n, V), bool)
    for r in range(n):
        allowed[r, rng.choice(V, int(rng.integers(1, 41)), replace=False)] = True
    k = rng.choice([1, 5, 20, 50, 50, 200, V + 9], n).astype(np.int32)
    _check(*_rows(rng, n, V, k), allowed=allowed)


def test_top_k_above_what_is_left_where_the_last_bin_is_not_empty():
    """Some tokens so far down that a filter's bins hold them no more: with and without a token there, the sums are the same."""
    rng = np.random.default_rng(1)
    x, noise, T, k, p = _rows(rng, 900, 30, 64)
    x[::2, ::5] -= 200
    x[::3, 7] = -math.inf
    _check(x, noise, T, k, p)


# ---------------------------------------------------------------- without a race

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("V", [1, 40, 9000, 50021])
def test_without_noise_the_share_is_at_the_row_s_temperature(dtype, V):
    """No noise picks the likeliest token; its log-probability is of exp(x / T) all the same, by number or by row, with filters
    that it passes anyway, with rules and without."""
    rng = np.random.default_rng(V)
    n = 8
    x = torch.from_numpy((3 * rng.standard_normal((n, V))).astype(np.float32)).to(dtype)
    T = np.array([0.3, 2.0, 1.0, 0.0, -1.0, math.nan, 0.01, 50.0], np.float32)
    rules = P.random_rules(rng, n, V, history=50, bias=4, mask=0.6)
    for r in (None, rules):
        z = x.float().numpy() if r is None else P.adjust_plain(x.float().numpy(), r, np.float32)[0]
        on_gpu = None if r is None else P.rules_on_gpu(r)
        for kw in ({}, dict(top_k=3), dict(top_p=0.5, min_p=0.1)):
            results = [L.sample(x.cuda(), temperature=_cuda(T), rules=on_gpu, **kw)]
            if r is None:
                for t in T:
                    token, logprob = L.sample(x.cuda(), temperature=float(t), **kw)
                    results.append((token, logprob, float(t)))
            for token, logprob, *t in results:
                for i in range(n):
                    want, lp, tol = P.sample_plain(z[i], None, t[0] if t else float(T[i]), 0, 1.0, 0.0)
                    got = float(logprob[i])
                    assert int(token[i]) == want and (got == lp or abs(got - lp) <= tol), (i, got, lp, tol)


# ---------------------------------------------------------------- far scores

def _scored(rng, n):
    """Rows of two segments far below the first token, whose tokens' noise makes up for it: token A wins by 1e-6 to 4e-5 of log 2.
    (rows, noise, A's place, B's place)"""
    V, log2 = 4 * 512, math.log(2)
    x = np.full((n, V), -400.0, np.float32)
    e = np.ones((n, V), np.float32)
    x[:, 0], e[:, 0] = 0.0, 2.0 ** 20
    a, b = 512 + 4 * rng.integers(0, 32, n), 1024 + 384 + 4 * rng.integers(0, 32, n) + 3  # the first and last of a thread's logits
    i, ulp = np.arange(n), 2.0 ** -17  # of numbers from 64 to 128
    for r in range(n):
        far = rng.uniform(70, 120)
        x[r, a[r]] = -far * log2
        # the scores within their segments, which are -log2 of the noise: A's last five bits about 31, B's about 0
        fa = (np.floor(rng.uniform(far - 1, far + 1) / ulp / 32) * 32 + rng.choice([28, 29, 30, 31])) * ulp
        e[r, a[r]] = 2.0 ** -fa
        want = float(x[r, a[r]]) / log2 - math.log2(float(e[r, a[r]])) - rng.uniform(1e-6, 4e-5)  # B's score
        fb = (np.floor(fa / ulp / 32) * 32 + 32 * rng.integers(-3, 4) + rng.choice([0, 1, 2])) * ulp
        x[r, b[r]] = (want - fb) * log2
        e[r, b[r]] = 2.0 ** -(want - float(x[r, b[r]]) / log2)
    return x, e, a, b


def test_scores_of_far_segments_with_tiny_noise():
    """Noise down to 2^-121: what a segment's winner scores is large beside what is left of it below the first token, and so
    are its roundings."""
    n = 4000
    x, e, a, b = _scored(np.random.default_rng(12), n)
    i = np.arange(n)
    score = lambda at: x[i, at].astype(np.float64) - np.log(e[i, at].astype(np.float64))
    assert (np.abs(score(a) - score(b)) < 1e-4).all() and (np.maximum(score(a), score(b)) > -2).all()
    want = np.where(score(a) > score(b), a, b)  # (equal ones would go to the lower, which is a)
    want = np.where(score(a) == score(b), a, want)
    one = np.float32(1)
    for T in (1.0, 0.5):
        token, _ = L.sample(_cuda(x * one * np.float32(T)), _cuda(e), temperature=T)
        wrong = np.flatnonzero(token.cpu().numpy() != want)
        assert not len(wrong), (len(wrong), T)


def test_top_k_as_a_number_means_what_it_means_by_row():
    """Numbers below 0 leave none out, those that are not whole or do not fit are refused."""
    rng = np.random.default_rng(4)
    n, V = 64, 300
    x, e = _cuda((3 * rng.standard_normal((n, V))).astype(np.float32)), _cuda(rng.exponential(size=(n, V)).astype(np.float32))
    for k in (-1, -2 ** 31, 0, 7, 7.0, np.int64(7), 2 ** 31 - 1):
        a = L.sample(x, e, top_k=k, top_p=0.9)
        b = L.sample(x, e, top_k=torch.full((n,), int(k), dtype=torch.int32, device="cuda"), top_p=0.9)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for k in (2.7, 0.5, -1.5, math.nan, math.inf, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(H.HxError) as err:
            L.sample(x, e, top_k=k)
        assert err.value.code == H.HX_ERR_INVALID and "top_k" in str(err.value)
