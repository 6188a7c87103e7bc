"""Sampling on the GPU against the plain 64-bit implementation."""
import math

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import logits as L
from tests import step_cases as P

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def built():
    B_.build()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _rows(rng, n, V, dtype):
    x = (3 * rng.standard_normal((n, V))).astype(np.float32)
    return torch.from_numpy(x).cuda().to(dtype)


def _noise(rng, n, V):
    return torch.from_numpy(rng.exponential(size=(n, V)).astype(np.float32)).cuda()


def _check_sample(x, noise, temperature, top_k, top_p, min_p, rules=None, **kw):
    n, V = x.shape
    full = lambda v, t: np.broadcast_to(np.asarray(v, t), (n,)).copy()
    T, k, p, m = full(temperature, np.float32), full(top_k, np.int32), full(top_p, np.float32), full(min_p, np.float32)
    d = lambda a: torch.from_numpy(a).cuda()
    token, logprob = L.sample(x, noise, temperature=d(T), top_k=d(k), top_p=d(p), min_p=d(m),
                              rules=P.rules_on_gpu(rules) if rules is not None else None, **kw)
    xs = x.float().cpu().numpy()
    if rules is not None:
        xs = P.adjust_plain(xs, rules, np.float32)[0]
    e = None if noise is None else noise.cpu().numpy()
    token, logprob = token.cpu().numpy(), logprob.cpu().numpy()
    for r in range(n):
        t, lp, tol = P.sample_plain(xs[r], None if e is None else e[r], float(T[r]), int(k[r]), float(p[r]), float(m[r]))
        assert token[r] == t, (r, token[r], t, T[r], k[r], p[r], m[r])
        assert (math.isnan(lp) and math.isnan(logprob[r])) or logprob[r] == lp or abs(logprob[r] - lp) <= tol, (r, logprob[r], lp, tol)
    return token, logprob


SIZES = [(5, 1), (5, 2), (5, 31), (6, 32), (6, 33), (9, 500), (7, 4096), (7, 4097), (6, 32000), (5, 50021), (5, 131072),
         (2, 262145), (2, 393216)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V", SIZES)
def test_sample(dtype, n, V):
    rng = np.random.default_rng(n * 7 + V)
    x = _rows(rng, n, V, dtype)
    e = _noise(rng, n, V)
    _check_sample(x, e, 1.0, 0, 1.0, 0.0)
    _check_sample(x, e, 0.7, 0, 0.9, 0.0)
    _check_sample(x, e, 1.3, 40, 1.0, 0.0)
    _check_sample(x, e, rng.choice([0.0, 0.3, 1.0, 4.0], n), rng.choice([0, 1, 2, 50, 700, V, V + 5], n),
                  rng.choice([0.0, 0.1, 0.5, 0.99, 0.99999, 1.0, 2.0], n), rng.choice([0.0, 0.001, 0.2, 1.0, 3.0], n))
    _check_sample(x, None, 1.0, 0, 1.0, 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V", [(6, 33), (8, 5003), (5, 50021), (4, 131072)])
def test_sample_with_rules(dtype, n, V):
    rng = np.random.default_rng(n * 5 + V)
    x, e = _rows(rng, n, V, dtype), _noise(rng, n, V)
    for kw in (dict(history=500), dict(bias=30), dict(mask=0.02), dict(history=200, bias=10, mask=0.3)):
        rules = P.random_rules(rng, n, V, **kw)
        _check_sample(x, e, rng.choice([0.0, 0.6, 1.0], n), rng.choice([0, 20, 300], n), rng.choice([0.3, 0.95, 1.0], n),
                      rng.choice([0.0, 0.05], n), rules)


@pytest.mark.parametrize("V", [600, 1024, 5003, 131072, 393216])
def test_sample_where_many_are_alike(V):
    """Equal logits, a few values, clusters far closer than a bin, far spread ones: cuts fall between equals, by their
    number."""
    rng = np.random.default_rng(V)
    flat = np.zeros(V, np.float32)
    some = rng.integers(0, 3, V).astype(np.float32)
    close = (5 + rng.random(V) * 1e-4).astype(np.float32)
    spread = (rng.standard_normal(V) * 1e30).astype(np.float32)
    two = np.where(rng.random(V) < 0.5, np.float32(-0.0), np.float32(0.0))
    x = torch.from_numpy(np.stack([flat, some, close, spread, two, -np.abs(spread)])).cuda()
    e = _noise(rng, 6, V)
    for k, p in ((V // 2 + 1, 1.0), (0, 0.5), (V // 3, 0.25), (513, 0.999), (0, 1e-6)):
        _check_sample(x, e, 1.0, k, p, 0.0)
    _check_sample(x, e, 1e30, V // 2, 0.5, 0.0)


def test_sample_special_values():
    """Infinities, NaN, nothing allowed, every noise unfit, temperatures of all kinds."""
    rng = np.random.default_rng(3)
    V = 700
    x = _rows(rng, 12, V, torch.float32)
    x[0] = -math.inf
    x[1] = math.nan
    x[2, 5], x[2, 9] = math.inf, math.inf
    x[3, 100:] = -math.inf
    x[4, 7] = math.nan
    x[5] = torch.finfo(torch.float32).min
    x[6, :] = -math.inf
    x[6, 699] = -3.0
    x[7, 3] = math.inf
    x[8] = torch.finfo(torch.float32).max
    x[9, ::2] = -torch.finfo(torch.float32).max
    e = _noise(rng, 12, V)
    for T in (1.0, 0.0, -1.0, math.nan, math.inf, 1e-30, 1e-40, 1e30):
        for k, p, m in ((0, 1.0, 0.0), (3, 1.0, 0.0), (0, 0.5, 0.0), (10, 0.9, 0.1), (0, math.nan, math.nan), (-1, -1.0, -1.0)):
            _check_sample(x, e, T, k, p, m)
    for v in (0.0, math.inf, -1.0, math.nan):  # the first of the order is picked
        _check_sample(x, torch.full((12, V), v, device="cuda"), 1.0, 0, 0.9, 0.0)
    e[:, ::3] = math.nan
    e[:, 1::3] = 0
    _check_sample(x, e, 1.0, 0, 1.0, 0.0)


@pytest.mark.parametrize("at", [-3.9e6, -4e6, -4.1e6, 3.9e6, 4e6, -1e7, 1e20])
def test_sample_far_from_zero(at):
    """Logits so far from zero that the grid of bins ends between one part of the vocabulary and another: x / T * 16 about `at`."""
    rng = np.random.default_rng(6)
    V = 40000
    x = torch.from_numpy((at / 16 + rng.standard_normal((3, V)) * max(3.0, abs(at) * 2e-8)).astype(np.float32)).cuda()
    e = _noise(rng, 3, V)
    for k, p in ((0, 0.9), (300, 1.0), (300, 0.7), (30000, 0.999)):
        _check_sample(x, e, 1.0, k, p, 0.0)


def test_sample_scores_next_to_each_other():
    """Scores that 32 bits cannot tell apart are told apart in 64, equal ones go to the lowest token."""
    rng = np.random.default_rng(5)
    V = 20000
    x = torch.zeros((4, V), device="cuda")
    e = torch.ones((4, V), device="cuda")
    up = np.nextafter(np.float32(1), np.float32(0))
    e[0, 17777] = float(up)
    e[1] = 1 + torch.from_numpy(rng.integers(0, 50, V).astype(np.float32) * 2.0 ** -23).cuda()
    x[2] = torch.from_numpy(rng.integers(0, 9, V).astype(np.float32) * 2.0 ** -24).cuda()
    token, _ = _check_sample(x, e, 1.0, 0, 1.0, 0.0)
    assert token[0] == 17777 and token[3] == 0
    token, _ = _check_sample(x, e, 1.0, 0, 0.75, 0.0)
    assert token[3] == 0


def test_sample_follows_the_weights():
    """Of many draws each token has about its share: 40000 of eight weights, six standard deviations."""
    n, V = 40000, 8
    w = torch.tensor([0.3, 0.25, 0.2, 0.1, 0.08, 0.04, 0.02, 0.01], dtype=torch.float64)
    x = torch.log(w).float().cuda().expand(n, V).contiguous()
    e = torch.empty((n, V), device="cuda").exponential_(generator=gen(9))
    for p, kept in ((1.0, 8), (0.74, 3)):
        token, _ = L.sample(x, e, top_p=p)
        share = torch.bincount(token.cpu().long(), minlength=V).double() / n
        want = torch.where(torch.arange(V) < kept, w, 0) / w[:kept].sum()
        assert bool(((share - want).abs() <= 6 * torch.sqrt(want * (1 - want) / n)).all())


def test_sample_strided_misaligned_and_out():
    rng = np.random.default_rng(14)
    for dtype in TYPES:
        for off, stride, nstride in ((0, 1040, 1009), (1, 1033, 1031), (5, 1011, 1200)):
            buf = torch.zeros(9 * 1040, dtype=dtype, device="cuda")
            x = buf[off:off + 7 * stride].view(7, stride)[:, :1009]
            x.copy_(_rows(rng, 7, 1009, dtype))
            e = torch.full((7 * nstride + off,), math.nan, device="cuda")[off:].view(7, nstride)[:, :1009]
            e.copy_(_noise(rng, 7, 1009))
            out = (torch.full((7,), -9, dtype=torch.int32, device="cuda"), torch.zeros(7, device="cuda"))
            a = _check_sample(x, e, 0.9, 0, 0.8, 0.0, P.random_rules(rng, 7, 1009, history=60, bias=5, mask=0.5), out=out)
            assert np.array_equal(a[0], out[0].cpu().numpy())


def test_sample_numbers_for_all_rows():
    rng = np.random.default_rng(15)
    x, e = _rows(rng, 6, 900, torch.bfloat16), _noise(rng, 6, 900)
    d = lambda v, t: torch.full((6,), v, dtype=t, device="cuda")
    f, i = torch.float32, torch.int32
    a = L.sample(x, e, temperature=0.8, top_k=30, top_p=0.7, min_p=0.05)
    b = L.sample(x, e, temperature=d(0.8, f), top_k=d(30, i), top_p=d(0.7, f), min_p=d(0.05, f))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert L.sample(x[:0], e[:0])[0].shape == (0,)


def test_sample_many_rows():
    n, V = 65536, 5
    x = randn(gen(1), n, V)
    token, logprob = L.sample(x)
    assert torch.equal(token.long(), x.argmax(1))
    want = torch.log_softmax(x.double(), 1).gather(1, token.long()[:, None])[:, 0]
    assert float((logprob.double() - want).abs().max()) <= 40 * P.U * 8


def test_sample_is_the_same_every_time_and_captured():
    rng = np.random.default_rng(16)
    n, V = 40, 60000
    x, e = _rows(rng, n, V, torch.bfloat16), _noise(rng, n, V)
    rules = P.rules_on_gpu(P.random_rules(rng, n, V, history=900, bias=30, mask=0.4))
    T = torch.rand(n, device="cuda", generator=gen(1))
    kw = dict(temperature=T, top_k=400, top_p=0.9, rules=rules)
    first = L.sample(x, e, **kw)
    for _ in range(20):
        again = L.sample(x, e, **kw)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1].view(torch.int32), again[1].view(torch.int32))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = L.sample(x, e, **kw)
        low = L.adjust(x, rules)
    x.copy_(x.flip(0))
    e.copy_(e.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    want = L.sample(x, e, **kw)
    assert torch.equal(out[0], want[0]) and torch.equal(low, L.adjust(x, rules))
    assert not torch.equal(out[0], first[0])
    for stream in (s, s.cuda_stream):
        other = L.sample(x, e, stream=stream, **kw)
        s.synchronize()
        assert torch.equal(other[0], want[0])


def test_sample_equals_adjust_then_sample():
    rng = np.random.default_rng(17)
    x, e = _rows(rng, 9, 40000, torch.float16), _noise(rng, 9, 40000)
    rules = P.rules_on_gpu(P.random_rules(rng, 9, 40000, history=900, bias=30, mask=0.4))
    a = L.sample(x, e, temperature=0.8, top_p=0.9, rules=rules)
    b = L.sample(L.adjust(x, rules, dtype=torch.float32), e, temperature=0.8, top_p=0.9)
    assert torch.equal(a[0], b[0])
    # the same weights, added up in another order: a sum takes at most 16 + 5 + 5 additions in a row on either side, of a
    # relative rounding each, and the result is rounded to 32 bits
    assert bool(((a[1] - b[1]).abs() <= P.U * (2 * 26 + 2 * a[1].abs())).all())



def test_sample_refusals_of_tensors():
    x = torch.zeros((2, 50), device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    for call, msg in [
            (lambda: L.sample(x.t(), x.t()), "contiguous"), (lambda: L.sample(x.double()), "dtype"),
            (lambda: L.sample(x, x[:1]), "shape"), (lambda: L.sample(x, x.half()), "dtype"),
            (lambda: L.sample(x, x.cpu()), "CUDA"), (lambda: L.sample(x, temperature=i), "dtype"),
            (lambda: L.sample(x, top_p=torch.ones(3, device="cuda")), "entry per row"), (lambda: L.sample(x, top_k=2 ** 31), "top_k"),
            (lambda: L.sample(x, x, out=(i, x[0, :2])), "overlaps"), (lambda: L.sample(x, out=(i, i.view(torch.float32))), "overlap"),
            (lambda: L.sample(x.expand(2, 50)[:, ::2]), "contiguous"), (lambda: L.sample(x[:1].expand(2, 50)), "stride")]:
        with pytest.raises(H.HxError) as e:
            call()
        assert e.value.code == H.HX_ERR_INVALID and msg in str(e.value), (msg, str(e.value))
