"""Rotary positions and adjusted logits on the GPU against the plain 64-bit implementations."""
import math

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import kvcache as KV
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


def near(got, want, tol):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:5], want[bad][:5], tol[bad][:5])


# ---------------------------------------------------------------- rotate

def _step(add, held):
    add, held = torch.tensor(add), torch.tensor(held)
    start = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(add, 0)])
    pos = torch.cat([h + torch.arange(int(a)) for a, h in zip(add, held)])
    return start.int().cuda(), (held + add).int().cuda(), pos


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (64, 32), (90, 30), (80, 20), (2, 2), (7, 4), (256, 256), (1024, 1022), (65, 2)])
def test_rotate(dtype, interleaved, dim, rotary):
    g = gen(dim + rotary)
    start, kv_len, pos = _step([3, 1, 0, 17, 1], [0, 70001, 9, 1 << 20, 250000000])
    T = len(pos)
    f = KV.Rope.frequencies(rotary, 10000.0)
    rope = KV.Rope(f, interleaved=interleaved, scale=1.25)
    q, k = randn(g, T, 6, dim, dtype=dtype), randn(g, T, 3, dim, dtype=dtype)
    for got in (rope.rotate(q, k, start, kv_len), rope.rotate(q, k, positions=pos.int().cuda())):
        for x, y in zip((q, k), got):
            want, tol = P.rotate_plain(x, pos, f, interleaved, 1.25)
            near(y, want, tol)
            assert torch.equal(y[..., rotary:], x[..., rotary:])
    near(rope.rotate(q, positions=pos.int().cuda(), inverse=True), *P.rotate_plain(q, pos, f, interleaved, 1.25, True))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (32, 8), (28, 4), (12, 12), (71, 1), (2048, 2048)])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 300])
def test_rotate_heads_and_lengths(heads, kv_heads, T):
    if heads == 2048 and T > 16:
        pytest.skip("slow on the host")
    g = gen(heads + T)
    f = KV.Rope.frequencies(64, 500000.0)
    rope = KV.Rope(f)
    q, k = randn(g, T, heads, 64, dtype=torch.bfloat16), randn(g, T, kv_heads, 64, dtype=torch.bfloat16)
    pos = torch.randint(0, 1 << 20, (T,), generator=g, device="cuda", dtype=torch.int32)
    for x, y in zip((q, k), rope.rotate(q, k, positions=pos)):
        near(y, *P.rotate_plain(x, pos, f, False, 1.0))


@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 1000, 4000, 65536])
def test_rotate_finds_rows(rows):
    """Rows of all lengths, empty ones at the ends and in between."""
    rng = np.random.default_rng(rows)
    add = rng.integers(0, 4, rows)
    add[0] = 0
    add[-1] = 0 if rows > 2 else 5
    held = rng.integers(0, 1000, rows)
    start, kv_len, pos = _step(add.tolist(), held.tolist())
    f = [1.0]
    x = torch.ones((len(pos), 1, 2), device="cuda")
    near(KV.Rope(f).rotate(x, None, start, kv_len), *P.rotate_plain(x, pos, f, False, 1.0))


@pytest.mark.parametrize("pos", [0, 1, 2 ** 31 - 1, -1, -2 ** 31])
def test_rotate_at_any_position(pos):
    f = KV.Rope.frequencies(64)
    x = randn(gen(1), 2, 3, 64)
    at = torch.full((2,), pos, dtype=torch.int32, device="cuda")
    near(KV.Rope(f).rotate(x, positions=at), *P.rotate_plain(x, at, f, False, 1.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [0, 1, 2, 4, 8])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_strided_and_in_place(dtype, offset, interleaved):
    """q, k and v of a token side by side at any alignment, heads outermost, outputs in place or elsewhere: what
    lies between stays."""
    g = gen(offset)
    T, H, K, D, R = 9, 4, 2, 64, 48
    f = KV.Rope.frequencies(R)
    rope = KV.Rope(f, interleaved=interleaved)
    pos = torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32)
    buf = randn(g, T * (H + 2 * K) * D + 16, dtype=dtype)
    x = buf[offset:offset + T * (H + 2 * K) * D].view(T, H + 2 * K, D)
    was = buf.clone()
    q, k = x[:, :H], x[:, H:H + K]
    want_q, want_k = P.rotate_plain(q, pos, f, interleaved, 1.0), P.rotate_plain(k, pos, f, interleaved, 1.0)
    # heads outermost, with gaps
    wide = torch.full((H, T + 1, D + 24), 7.0, dtype=dtype, device="cuda")
    q2 = wide[:, :T, 8:8 + D].permute(1, 0, 2)
    k2 = torch.empty((T, K, D), dtype=dtype, device="cuda")
    got = rope.rotate(q, k, positions=pos, out=(q2, k2))
    assert got[0] is q2 and torch.equal(buf, was)
    near(q2, *want_q)
    near(k2, *want_k)
    assert bool((wide[:, T:] == 7).all()) and bool((wide[:, :, :8] == 7).all()) and bool((wide[:, :, 8 + D:] == 7).all())
    rope.rotate(q, k, positions=pos, out=(q, k))
    near(q, *want_q)
    near(k, *want_k)
    y, z = buf[offset:offset + x.numel()].view(T, H + 2 * K, D), was[offset:offset + x.numel()].view(T, H + 2 * K, D)
    assert torch.equal(y[:, H + K:], z[:, H + K:]) and torch.equal(y[..., R:], z[..., R:])
    assert torch.equal(buf[:offset], was[:offset]) and torch.equal(buf[offset + x.numel():], was[offset + x.numel():])


def test_rotate_reads_broadcast_heads():
    g = gen(3)
    x = randn(g, 5, 1, 64, dtype=torch.float16).expand(5, 6, 64)
    f = KV.Rope.frequencies(64)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    near(KV.Rope(f).rotate(x, positions=pos), *P.rotate_plain(x, pos, f, False, 1.0))


def test_rotate_leaves_tokens_behind_the_last_row():
    f = KV.Rope.frequencies(32)
    start, kv_len, pos = _step([2, 3], [5, 9])
    q, k = randn(gen(2), 12, 2, 32), randn(gen(3), 12, 1, 32)
    out = (torch.full_like(q, 3.0), torch.full_like(k, 3.0))
    KV.Rope(f).rotate(q, k, start, kv_len, out=out)
    for x, y in zip((q, k), out):
        near(y[:5], *P.rotate_plain(x[:5], pos, f, False, 1.0))
        assert bool((y[5:] == 3).all())
    was = q.clone()
    KV.Rope(f).rotate(q, None, start, kv_len, out=q)
    assert torch.equal(q[5:], was[5:]) and not torch.equal(q[:5], was[:5])


def test_rotate_after_a_step_with_a_refused_row():
    """Rows that map_step refused hold nothing: their tokens are turned by positions below zero and hurt no other's."""
    i32 = dict(dtype=torch.int32, device="cuda")
    held, add = torch.tensor([3, 100, 7], **i32), torch.tensor([2, 40, 1], **i32)
    table, ring = torch.zeros((3, 3), **i32), torch.arange(1, 2, **i32)
    step = KV.map_step(held, add, table, ring, torch.tensor([0, 0], dtype=torch.int64, device="cuda"), 43, 64)  # no free block
    assert step.counts.tolist()[2] == 1
    f = KV.Rope.frequencies(32)
    q = randn(gen(2), 43, 2, 32)
    pos = torch.cat([torch.arange(3, 5), torch.arange(-40, 0), torch.arange(7, 8)])
    near(KV.Rope(f).rotate(q, None, step.row_start, step.kv_len), *P.rotate_plain(q, pos, f, False, 1.0))


def test_rotate_by_malformed_rows_stays_within_the_arrays():
    """Row starts in any order, lengths of any size: some angle, nothing outside."""
    start = torch.tensor([5, -3, 900, 2, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, 7, -1], dtype=torch.int32, device="cuda")
    buf = torch.ones(40, 1, 4, device="cuda")
    KV.Rope([1.0, 0.1]).rotate(buf[10:20], None, start, kv_len, out=buf[10:20])
    assert bool((buf[:10] == 1).all()) and bool((buf[20:] == 1).all())
    assert bool((buf.abs() <= 2).all())


def test_rotate_inverse_is_its_gradient():
    """Against differences: d/dx of sum(g * rotate(x)) is rotate of g, turned back."""
    f, g = KV.Rope.frequencies(8), gen(5)
    rope = KV.Rope(f, scale=1.0)
    pos = torch.tensor([3, 77], dtype=torch.int32, device="cuda")
    x, w = randn(g, 2, 1, 10), randn(g, 2, 1, 10)
    grad = rope.rotate(w, positions=pos, inverse=True).double().cpu()
    base = x.double().cpu()

    def value(z):
        return float((P.rotate_plain(z, pos, f, False, 1.0)[0] * w.double().cpu()).sum())

    for t in range(2):
        for d in range(10):
            a, b = base.clone(), base.clone()
            a[t, 0, d] += 0.5
            b[t, 0, d] -= 0.5
            # linear: the difference is exact but for 64 bits
            assert abs(value(a.float()) - value(b.float()) - float(grad[t, 0, d])) <= 64 * P.U * float(w.abs().max() + 1)
    near(rope.rotate(rope.rotate(x, positions=pos), positions=pos, inverse=True), base, torch.full_like(base, 16 * P.U * float(x.abs().max())))


def test_rotate_captured_on_other_streams_and_empty():
    f, g = KV.Rope.frequencies(64), gen(6)
    rope = KV.Rope(f)
    q, k = randn(g, 7, 4, 64, dtype=torch.bfloat16), randn(g, 7, 2, 64, dtype=torch.bfloat16)
    pos = torch.arange(7, dtype=torch.int32, device="cuda")
    out = (torch.empty_like(q), torch.empty_like(k))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        rope.rotate(q, k, positions=pos, out=out)
    q.mul_(2)
    pos.add_(11)
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip((q, k), out):
        near(y, *P.rotate_plain(x, pos, f, False, 1.0))
    for stream in (s, s.cuda_stream):
        a = rope.rotate(q, k, positions=pos, stream=stream)
        s.synchronize()
        assert torch.equal(a[0], out[0]) and torch.equal(a[1], out[1])
    e = rope.rotate(q[:0], k[:0], positions=pos[:0])
    assert e[0].shape == (0, 4, 64) and e[1].shape == (0, 2, 64)


def test_rotate_past_32_bits():
    """Values whose offsets pass 2^31."""
    T = 150000
    x = torch.zeros((T, 130, 128), dtype=torch.bfloat16, device="cuda")  # 2.5 billion values
    x[-1] = randn(gen(1), 130, 128, dtype=torch.bfloat16)
    f = KV.Rope.frequencies(128)
    start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    want = P.rotate_plain(x[-1:], torch.tensor([T - 1]), f, False, 1.0)
    KV.Rope(f).rotate(x, None, start, start[1:], out=x)
    near(x[-1:], *want)
    assert not bool(x[:-1].any())


# ---------------------------------------------------------------- adjust

CASES = [(1, 1), (3, 31), (5, 32), (4, 33), (9, 1000), (7, 8191), (7, 8192), (6, 8193), (2, 50021), (2, 131072)]


def _rows(rng, n, V, dtype):
    x = (3 * rng.standard_normal((n, V))).astype(np.float32)
    return torch.from_numpy(x).cuda().to(dtype)


def _check_adjust(x, rules, out_dtype=None, **kw):
    xs = x.float().cpu().numpy()
    got = L.adjust(x, P.rules_on_gpu(rules), dtype=out_dtype, **kw)
    as32, _ = P.adjust_plain(xs, rules, np.float32)
    want = torch.from_numpy(as32).to(got.dtype)
    assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
    assert torch.equal(got.cpu().nan_to_num(1.5), want.nan_to_num(1.5))  # every operation is defined, with its rounding
    as64, tol = P.adjust_plain(xs, rules)
    fine = np.isfinite(as64)
    assert np.array_equal(fine, np.isfinite(as32))
    eps = torch.finfo(got.dtype).eps / 2
    err = np.abs(got.double().cpu().numpy() - np.where(fine, as64, 0))[fine]
    assert (err <= (tol * (1 + eps) + eps * np.abs(np.where(fine, as64, 0)) + P.TINY[got.dtype])[fine]).all()
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V", CASES)
def test_adjust(dtype, n, V):
    rng = np.random.default_rng(n + V)
    x = _rows(rng, n, V, dtype)
    for kw in (dict(history=300), dict(bias=40), dict(mask=0.4), dict(history=77, bias=9, mask=0.7)):
        rules = P.random_rules(rng, n, V, **kw)
        _check_adjust(x, rules)
        if dtype != torch.float32:
            _check_adjust(x, rules, torch.float32)


@pytest.mark.parametrize("width", [1, 127, 4096, 30001])
def test_adjust_long_histories(width):
    rng = np.random.default_rng(width)
    rules = P.random_rules(rng, 5, 700, history=width)
    rules["length"][3:] = width
    rules["prompt_len"][4] = 0
    rules["history"][4, :] = 3  # one token all over again
    _check_adjust(_rows(rng, 5, 700, torch.float16), rules)


def test_adjust_the_longest_history():
    rng = np.random.default_rng(0)
    V, n = 40, L.MAX_HISTORY
    h = np.full((1, n), 7, np.int32)
    rules = dict(history=h, length=np.array([n], np.int32), frequency=np.array([2.0 ** -10], np.float32))
    x = _rows(rng, 1, V, torch.float32)
    got = L.adjust(x, P.rules_on_gpu(rules))
    want = x.clone()
    want[0, 7] = x[0, 7] - n * 2.0 ** -10
    assert torch.equal(got, want)


def test_adjust_parts_of_a_history_are_optional():
    rng = np.random.default_rng(4)
    full = P.random_rules(rng, 6, 500, history=90)
    x = _rows(rng, 6, 500, torch.float32)
    for names in ((), ("repetition",), ("presence",), ("frequency", "prompt_len"), ("prompt_len",)):
        _check_adjust(x, {k: v for k, v in full.items() if k in ("history", "length") + names})


@pytest.mark.parametrize("dtype", TYPES)
def test_adjust_special_values(dtype):
    """Infinities and NaN: behind a mask they are -infinity, elsewhere what arithmetic makes of them."""
    rng = np.random.default_rng(8)
    x = _rows(rng, 4, 200, dtype)
    x[:, 10], x[:, 11], x[:, 12], x[:, 13] = math.inf, -math.inf, math.nan, -30000.0
    x[:, 14], x[:, 15] = -0.0, 30000.0
    rules = P.random_rules(rng, 4, 200, history=100, mask=0.5, odd=False)
    rules["history"][:, :30] = np.arange(30) % 20
    rules["length"][:] = 100
    got = _check_adjust(x, rules)
    x[:, 13], x[:, 15] = torch.finfo(dtype).min, torch.finfo(dtype).max
    _check_adjust(x, P.random_rules(rng, 4, 200, mask=0.5))
    rules = dict(mask=np.zeros((1, 7), np.int32), mask_row=np.zeros(4, np.int32))
    assert bool((_check_adjust(x, rules) == -math.inf).all())
    assert got.shape == x.shape


def test_adjust_in_place_strided_and_misaligned():
    rng = np.random.default_rng(11)
    for dtype in TYPES:
        for off, stride in ((0, 1040), (1, 1033), (3, 1027), (8, 1029)):
            buf = torch.full((9 * 1040,), 5.0, dtype=dtype, device="cuda")
            x = buf[off:off + 7 * stride].view(7, stride)[:, :1009]
            x.copy_(_rows(rng, 7, 1009, dtype))
            was = buf.clone()
            rules = P.random_rules(rng, 7, 1009, history=60, bias=5, mask=0.5)
            want = _check_adjust(x, rules)
            assert torch.equal(buf, was)
            wide = torch.full((7, 1100), 9.0, device="cuda")
            got = _check_adjust(x, rules, out=wide[:, 33:33 + 1009])
            assert torch.equal(got.to(dtype), want) or dtype == torch.float32
            assert bool((wide[:, :33] == 9).all()) and bool((wide[:, 33 + 1009:] == 9).all())
            assert L.adjust(x, P.rules_on_gpu(rules), out=x) is x
            assert torch.equal(x, want)
            keep = torch.ones_like(buf, dtype=torch.bool)
            keep[off:off + 7 * stride].view(7, stride)[:, :1009] = False
            assert torch.equal(buf[keep], was[keep])


def test_adjust_masks_strided_or_one_a_row():
    rng = np.random.default_rng(12)
    x = _rows(rng, 5, 333, torch.float32)
    w = rng.integers(-2 ** 31, 2 ** 31, (5, 20)).astype(np.int32)
    big = torch.from_numpy(w).cuda()
    rules = L.Rules(mask=big[:, 2:14])
    want, _ = P.adjust_plain(x.cpu().numpy(), dict(mask=w[:, 2:14]), np.float32)
    assert torch.equal(L.adjust(x, rules).cpu(), torch.from_numpy(want))


def test_adjust_bias_lists():
    """Starts out of range or falling, and more entries than count."""
    rng = np.random.default_rng(13)
    V, n = 300, 6
    start = np.array([-5, 3, 2, 9, 9000, 4, 99999], np.int32)
    tok = rng.integers(0, V, 9000).astype(np.int32)
    rules = dict(bias_start=start, bias_token=tok, bias_value=rng.standard_normal(9000).astype(np.float32))
    _check_adjust(_rows(rng, n, V, torch.float32), rules)


def test_adjust_many_rows_and_none():
    x = randn(gen(1), 65536, 3)
    h = torch.arange(65536, dtype=torch.int32, device="cuda")[:, None] % 3
    r = L.Rules(history=h, length=torch.ones(65536, dtype=torch.int32, device="cuda"),
                presence=torch.full((65536,), 2.0, device="cuda"))
    want = x.clone()
    want.scatter_add_(1, h.long(), torch.full((65536, 1), -2.0, device="cuda"))
    assert torch.equal(L.adjust(x, r), want)
    assert L.adjust(x[:0], L.Rules()).shape == (0, 3)
    assert torch.equal(L.adjust(x, L.Rules()), x)


def test_refusals_of_tensors():
    x = torch.zeros((2, 50), device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    h = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    w = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    for call, msg in [
            (lambda: L.adjust(x, L.Rules(mask=w, mask_row=i)), "fewer bits"), (lambda: L.adjust(x, L.Rules(history=h[:1], length=i[:1])), "rows"),
            (lambda: L.adjust(x, L.Rules(history=h, length=i), out=x[:, :]), None),
            (lambda: L.adjust(x, L.Rules(history=h, length=i), dtype=torch.float16), "dtype"),
            (lambda: L.Rules(history=h), "length"), (lambda: L.Rules(length=i), "history"), (lambda: L.Rules(mask_row=i), "mask"),
            (lambda: L.Rules(history=h, length=i[:1]), "rows"), (lambda: L.Rules(history=h.t(), length=i), "contiguous"),
            (lambda: L.Rules(bias=(i, i, i)), "dtype"), (lambda: L.Rules(mask=w.cpu()), "CUDA")]:
        if msg is None:
            call()
            continue
        with pytest.raises(H.HxError) as e:
            call()
        assert e.value.code == H.HX_ERR_INVALID and msg in str(e.value), (msg, str(e.value))
    buf = torch.zeros(300, device="cuda")
    y = buf[:100].view(2, 50)
    with pytest.raises(H.HxError, match="overlaps the logits"):
        L.adjust(y, L.Rules(), out=buf[1:101].view(2, 50))
    z = torch.zeros((2, 50), dtype=torch.int32, device="cuda")
    with pytest.raises(H.HxError, match="overlaps the rules"):
        L.adjust(y, L.Rules(history=z, length=i), out=z.view(torch.float32))
    rope = KV.Rope([1.0, 0.5])
    q = torch.zeros((3, 2, 6), device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    flat = torch.zeros(200, device="cuda")
    for call, msg in [
            (lambda: rope.rotate(q), "either"), (lambda: rope.rotate(q, positions=pos[:2]), "positions"),
            (lambda: rope.rotate(q, positions=pos.long()), "dtype"), (lambda: rope.rotate(q[..., :3], positions=pos), "rotary_dim"),
            (lambda: rope.rotate(q, q.half(), positions=pos), "dtype"), (lambda: rope.rotate(q, q[:2], positions=pos), "k must be"),
            (lambda: rope.rotate(q, positions=pos, row_start=pos, kv_len=pos), "either"),
            (lambda: rope.rotate(q, None, pos, pos), "row_start"), (lambda: rope.rotate(q, positions=pos, out=q[:2]), "shape"),
            (lambda: rope.rotate(flat[:36].view(3, 2, 6), positions=pos, out=flat[1:37].view(3, 2, 6)), "overlaps q"),
            (lambda: rope.rotate(q, positions=pos, out=flat[:12].view(1, 2, 6).expand(3, 2, 6)), "one place"),
            (lambda: rope.rotate(q, q.clone(), positions=pos, out=(flat[:36].view(3, 2, 6), flat[30:66].view(3, 2, 6))), "other's"),
            (lambda: rope.rotate(q.cpu(), positions=pos), "CUDA")]:
        with pytest.raises(H.HxError) as e:
            call()
        assert e.value.code == H.HX_ERR_INVALID and msg in str(e.value), (msg, str(e.value))
