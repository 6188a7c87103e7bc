"""The cache operators on the GPU against the plain 64-bit implementations."""
import itertools
import math

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import kvcache as KV
from tests import kv_cases as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B_.build()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---------------------------------------------------------------- map

def _map_case(seed, n, B, kinds, free_share=1.0, over=0, width_cut=0):
    rng = np.random.default_rng(seed)
    held = rng.integers(0, 20 * B, n).astype(np.int32)
    add = np.ones(n, np.int32)
    u = rng.random(n)
    if "chunk" in kinds:
        add = np.where(u < 0.3, rng.integers(1, 9 * B, n), add).astype(np.int32)
    if "new" in kinds:
        held = np.where(u < 0.15, 0, held).astype(np.int32)
    if "idle" in kinds:
        add = np.where((u > 0.5) & (u < 0.7), 0, add).astype(np.int32)
    if "end" in kinds:
        add = np.where(u > 0.8, -1, add).astype(np.int32)
    if "edge" in kinds:
        held = (held // B * B + rng.integers(-1, 2, n)).clip(0).astype(np.int32)
    if "bad" in kinds:
        held = np.where(rng.random(n) < 0.1, -5, held).astype(np.int32)
        add = np.where(rng.random(n) < 0.1, -7, add).astype(np.int32)
    tok = np.maximum(add, 0).astype(np.int64)
    safe = np.maximum(held, 0).astype(np.int64)
    width = int(max(1, (-(-(safe + tok) // B)).max() + 1 - width_cut))
    have = -(-safe // B)
    need = int((-(-(safe + tok) // B) - have).sum())
    free = max(1, int(need * free_share))
    cap = int(have.sum()) + free
    ids = rng.permutation(cap).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    at = 0
    for r in range(n):
        m = min(int(have[r]), width)
        table[r, :m] = ids[at:at + m]
        at += m
    head = int(rng.integers(0, cap))
    ring = np.full(cap, -1, np.int32)
    ring[(head + np.arange(free)) % cap] = ids[cap - free:]
    n_tokens = max(0, int(tok.sum()) - over)
    return held, add, table, ring, np.array([head, free], np.int64), n_tokens


def _check_map(held, add, table, ring, state, n_tokens, B, strided=False):
    n = len(held)
    want_table, want_ring = table.copy(), ring.copy()
    most = KV.max_runs(n, n_tokens, B)
    want = P.map_plain(held, add, want_table, want_ring, state, n_tokens, B, max(most, 0))
    d = lambda x: torch.from_numpy(x).cuda()
    tb = d(table)
    if strided:
        wide = torch.full((n, table.shape[1] + 5), -9, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = tb
        tb = wide[:, :table.shape[1]]
    rg = d(ring)
    for _ in range(2):  # the second call starts from what the first one changed
        got = KV.map_step(d(held), d(add), tb, rg, d(state), n_tokens, B)
        for name, w in zip(("row_start", "kv_len", "slots", "runs", "counts", "ring_state"), want):
            g = getattr(got, name).cpu().numpy()
            assert np.array_equal(g, w), (name, np.argwhere(g != w)[:5])
        assert np.array_equal(tb.cpu().numpy(), want_table)
        assert np.array_equal(rg.cpu().numpy(), want_ring)
    if strided:
        assert bool((wide[:, table.shape[1]:] == -9).all())


@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 2, 33, 511, 513, 1500])
@pytest.mark.parametrize("kinds", ["", "chunk,new,idle,end", "edge,chunk"])
def test_map(B, n, kinds):
    _check_map(*_map_case(n * B, n, B, kinds), B, strided=n == 33)


@pytest.mark.parametrize("n", [5, 700])
@pytest.mark.parametrize("kw", [dict(free_share=0.5), dict(free_share=0.9), dict(over=1), dict(over=900),
                                dict(width_cut=3), dict(free_share=0.4, over=50, width_cut=2)])
def test_map_refuses_rows(n, kw):
    _check_map(*_map_case(7 * n, n, 32, "chunk,new,idle,end,bad", **kw), 32)


def test_map_one_long_row_between_short_ones():
    held = np.array([5, 0, 63], np.int32)
    add = np.array([1, 100003, 1], np.int32)
    n_blocks = 2 + 1 + 3200
    table = np.full((3, 3200), -1, np.int32)
    table[0, 0], table[2, 0:2] = 7, (9, 11)
    ring = np.random.default_rng(0).permutation(n_blocks).astype(np.int32)
    _check_map(held, add, table, ring, np.array([3, n_blocks], np.int64), 100005, 32)


def test_map_without_tokens():
    held, add = np.array([40, 0, 17, 3], np.int32), np.array([0, 0, -1, 0], np.int32)
    table = np.arange(16, dtype=np.int32).reshape(4, 4)
    ring = np.zeros(16, np.int32)
    _check_map(held, add, table, ring, np.array([14, 3], np.int64), 0, 16)


def test_map_steps_follow_one_another():
    """Requests that come, grow, end: no block is ever in two hands, and all come back."""
    rng = np.random.default_rng(5)
    n, B, cap, width = 40, 16, 400, 60
    held = torch.zeros(n, dtype=torch.int32, device="cuda")
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    ring = torch.arange(cap, dtype=torch.int32, device="cuda")
    state = torch.tensor([0, cap], dtype=torch.int64, device="cuda")
    steps = [KV.Step.empty(n, 0, B)]
    for _ in range(60):
        h = held.cpu().numpy()
        u = rng.random(n)
        add = np.where(h == 0, np.where(u < 0.5, rng.integers(1, 90, n), 0), np.where(u < 0.08, -1, 1)).astype(np.int32)
        T = int(np.maximum(add, 0).sum())
        step = KV.map_step(held, torch.from_numpy(add).cuda(), table, ring, state, T, B)
        kv = step.kv_len
        went_on = (kv > 0) | torch.from_numpy(add < 0).cuda()
        held = torch.where(went_on, kv, held)
        state = step.ring_state
        hold = held.cpu().numpy()
        used = np.concatenate([table[r, :-(-int(hold[r]) // B)].cpu().numpy() for r in range(n)])
        head, free = state.tolist()
        idle = ring.cpu().numpy()[(head + np.arange(free)) % cap]
        assert sorted(np.concatenate([used, idle]).tolist()) == list(range(cap))


# ---------------------------------------------------------------- append

def _append(x_k, x_v, cache, runs):
    kc, ks = cache.k.view(torch.uint8).cpu().numpy(), cache.k_scale.double().cpu().numpy()
    vc, vs = cache.v.view(torch.uint8).cpu().numpy(), cache.v_scale.double().cpu().numpy()
    P.append_plain(x_k.double().cpu().numpy(), kc, ks, runs.cpu().numpy())
    P.append_plain(x_v.double().cpu().numpy(), vc, vs, runs.cpu().numpy())
    for _ in range(2):  # appending the same tokens again changes nothing
        cache.append(x_k, x_v, runs)
        for got, want in ((cache.k.view(torch.uint8), kc), (cache.v.view(torch.uint8), vc)):
            g = got.cpu().numpy()
            assert np.array_equal(g, want), np.argwhere(g != want)[:5]
        assert np.array_equal(cache.k_scale.double().cpu().numpy(), ks)
        assert np.array_equal(cache.v_scale.double().cpu().numpy(), vs)


def _runs(rng, n_blocks, B, count):
    """Random runs on distinct blocks, tokens in order."""
    out, t = [], 0
    for b in rng.permutation(n_blocks)[:count]:
        off = int(rng.integers(0, B)) if rng.random() < 0.7 else 0
        n = int(rng.integers(1, B - off + 1)) if rng.random() < 0.6 else 1
        out.append((t, n, int(b), off))
        t += n
    return torch.tensor(out, dtype=torch.int32).cuda(), t


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("B,H,D", [(16, 3, 64), (32, 1, 128), (64, 8, 128), (128, 2, 64), (128, 1, 128)])
def test_append(dtype, B, H, D):
    g, rng = gen(B + H), np.random.default_rng(B * D)
    k, v, ks, vs = P.random_cache(g, 12, H, B, D, spread=3)
    runs, T = _runs(rng, 12, B, 9)
    big = torch.exp2(torch.randint(-6, 7, (T, H, 1), generator=g, device="cuda").float())  # some runs grow their scale
    x = [(torch.randn((T, H, D), generator=g, device="cuda") * big).to(dtype) for _ in range(2)]
    _append(x[0], x[1], KV.Cache(k, v, ks, vs), runs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_append_values_at_the_edges(dtype):
    """Ties, the largest and smallest values, zeros, infinities, NaN; blocks of zeros alone."""
    B, H, D = 16, 2, 64
    g = gen(3)
    k, v, ks, vs = P.random_cache(g, 6, H, B, D)
    top = torch.finfo(dtype).max
    vals = [0.0, -0.0, 448.0, 449.0, 464.0, 480.0, 1.0625, 1.1875, -1.0625, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10,
            torch.finfo(dtype).tiny, torch.finfo(dtype).smallest_normal, 17.0, 27.0]
    x = torch.zeros((24, H, D))
    x[0:4, 0, :16] = torch.tensor(vals)
    x[4:8, 1] = top
    x[5, 1, 3], x[5, 1, 4] = -top, 1.0
    x[8, 0, 5], x[9, 0, 6], x[10, 0, 7] = math.inf, -math.inf, math.nan
    x[8:11, 0, 8:] = 3.5
    x[12:16, 0] = 448.0
    x[12:16, 1] = 448.0 * 1.001 if dtype == torch.float32 else 450.0
    x[20, 0, :] = math.nan
    x[21, 1, :] = math.inf
    x = x.to(dtype).cuda()
    runs = torch.tensor([(0, 4, 2, 0), (4, 4, 0, 0), (8, 4, 5, 4), (12, 4, 1, 0), (16, 4, 3, 0), (20, 4, 4, 7)],
                        dtype=torch.int32).cuda()
    _append(x, x.flip(1).contiguous(), KV.Cache(k, v, ks, vs), runs)


def test_append_strided_heads_side_by_side_and_interleaved_blocks():
    g, rng = gen(9), np.random.default_rng(2)
    B, H, D, N = 32, 4, 64, 10
    both = torch.zeros((N, 2, H, B, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.ones((N, 2, H), device="cuda")
    runs, T = _runs(rng, N, B, 8)
    qkv = torch.randn((T, 12, D), generator=g, device="cuda").half()
    _append(qkv[:, 4:8], qkv[:, 8:], KV.Cache(both[:, 0], both[:, 1], scales[:, 0], scales[:, 1]), runs)
    x = torch.randn((H, T, D), generator=g, device="cuda").half().transpose(0, 1)  # heads outermost
    _append(x, x, KV.Cache(both[:, 0], both[:, 1], scales[:, 0], scales[:, 1]), runs)


def test_append_leaves_out_runs_that_do_not_fit():
    g = gen(4)
    k, v, ks, vs = P.random_cache(g, 5, 2, 16, 64)
    x = torch.randn((8, 2, 64), generator=g, device="cuda").half()
    runs = torch.tensor([(0, 2, 1, 0), (2, 0, 2, 0), (2, 2, 5, 0), (2, 2, -1, 0), (2, 7, 3, 0), (-1, 2, 3, 0),
                         (4, 2, 3, 15), (4, 2, 3, -1), (4, -3, 3, 2), (6, 2, 4, 3), (2 ** 31 - 1, 2, 0, 0)],
                        dtype=torch.int32).cuda()
    _append(x, x, KV.Cache(k, v, ks, vs), runs)


def test_map_append_fill_a_cache_that_reads_back():
    """Tokens that come in chunks and one by one are found at their slots, off by e4m3's rounding at most:
    2^-4 of a value once it is stored, the same again each time its block's scale has made it subnormal."""
    g, rng = gen(21), np.random.default_rng(8)
    n, B, H, D, width, cap = 6, 16, 2, 64, 16, 60
    held = torch.zeros(n, dtype=torch.int32, device="cuda")
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    ring = torch.arange(cap, dtype=torch.int32, device="cuda")
    state = torch.tensor([0, cap], dtype=torch.int64, device="cuda")
    cache = KV.Cache.empty(cap, H, B, D)
    seen = [[] for _ in range(n)]
    for i in range(20):
        add = torch.from_numpy(np.where(rng.random(n) < 0.3, rng.integers(1, 30, n), 1).astype(np.int32) if i < 4
                               else rng.integers(0, 2, n).astype(np.int32))
        T = int(add.sum())
        x = torch.randn((T, H, D), generator=g, device="cuda").half()
        step = KV.map_step(held, add.cuda(), table, ring, state, T, B)
        assert step.counts.tolist()[2] == 0
        cache.append(x, -x, step.runs)
        at = 0
        for r in range(n):
            seen[r].append(x[at:at + int(add[r])].double())
            at += int(add[r])
        held, state = step.kv_len, step.ring_state
    for r in range(n):
        want = torch.cat(seen[r])
        ids = table[r, :-(-len(want) // B)].long()
        for c, s, sign in ((cache.k, cache.k_scale, 1), (cache.v, cache.v_scale, -1)):
            sc = s[ids].double()[:, :, None, None]
            got = (c[ids].double() * sc).permute(0, 2, 1, 3).reshape(-1, H, D)[:len(want)]
            unit = (sc * 2.0 ** -9).expand(-1, -1, B, 1).permute(0, 2, 1, 3).reshape(-1, H, 1)[:len(want)]
            assert bool(((got - sign * want).abs() <= 2.0 ** -4 * want.abs() + 2 * unit).all())


# ---------------------------------------------------------------- attend

def _attend(q_len, kv_len, H, group, D, B, dtype, *, causal=True, window=0, seed=0, spread=2, max_q=None, strided=False,
            poison=True, sm_scale=None, scale_up=1.0):
    g = gen(seed)
    table, N = P.paged(g, kv_len, B)
    k, v, ks, vs = P.random_cache(g, N, H, B, D, spread)
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    T = int(start[-1])
    if poison:  # what no request holds: NaN, and blocks that no row uses with NaN scales
        live = torch.zeros((N, B), dtype=torch.bool, device="cuda")
        for r, n in enumerate(kv_len):
            for b in range(-(-n // B)):
                live[table[r, b].long(), :min(B, n - b * B)] = True
        for x in (k, v):
            x.view(torch.uint8).masked_fill_(~live[:, None, :, None], 0x7f)
        for s in (ks, vs):
            s.masked_fill_(~live.any(1)[:, None], math.nan)
    wide = torch.randn((T, H * group + 3, D), generator=g, device="cuda") * scale_up
    q = wide.to(dtype)[:, 1:1 + H * group] if strided else wide[:, :H * group].to(dtype).contiguous()
    out = None
    if strided:
        out = torch.full((T, 2 * H * group, D), 7.0, dtype=dtype, device="cuda")[:, ::2]
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    sm = D ** -0.5 if sm_scale is None else sm_scale
    cache = KV.Cache(k, v, ks, vs)
    args = (q, table, d(start), d(np.array(kv_len)))
    kw = dict(causal=causal, window=window, sm_scale=sm, max_q=max(q_len + [1]) if max_q is None else max_q)
    got, lse = cache.attend(*args, out=out, return_lse=True, **kw)
    want, wlse, tol, ltol = P.attend_plain(q, k, v, ks, vs, table, start, kv_len, sm, causal, window)
    _near(got, lse, want, wlse, tol, ltol)
    again, lse2 = cache.attend(*args, return_lse=True, **kw)
    assert torch.equal(again, got) and torch.equal(lse2, lse)
    return got, lse


def _near(got, lse, want, wlse, tol, ltol):
    e = (got.double() - want).abs()
    assert bool((e <= tol).all()), f"out: {float((e / tol.clamp(min=1e-300)).max())} of the bound"
    empty = wlse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    e = torch.where(empty, 0, (lse.double() - wlse).abs())
    assert bool((e[~empty] <= ltol[~empty]).all()), f"lse: {float((e / ltol.clamp(min=1e-300)).max())} of the bound"


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700]


@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,group", [(1, 1), (2, 4), (3, 7), (1, 16), (2, 24)])
def test_attend_single_tokens(B, D, dtype, H, group):
    _attend([1] * len(EDGES), EDGES, H, group, D, B, dtype, seed=B + D + group)


@pytest.mark.parametrize("group", [40, 100, 128])
def test_attend_many_heads_on_one(group):
    _attend([1, 1, 1], [5, 200, 333], 1, group, 64, 32, torch.bfloat16)
    _attend([1, 2, 3], [5, 200, 333], 2, group, 128, 16, torch.float16)


@pytest.mark.parametrize("B", [16, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 5, 64, 130])
def test_attend_several_tokens(B, D, causal, window):
    """Chunks of every size over lengths around the tiles; rows that hold fewer tokens than
    the step gives them, whose first tokens see nothing."""
    q_len = [1, 0, 3, 17, 130, 64, 2, 9, 40, 1]
    kv_len = [65, 100, 3, 200, 130, 300, 0, 4, 25, 513]
    _attend(q_len, kv_len, 2, 4, D, B, torch.float16, causal=causal, window=window, seed=window)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_chunks_of_groups(group, dtype):
    _attend([70, 257, 5, 33], [70, 400, 140, 34], 2, group, 128, 32, dtype, seed=group)


@pytest.mark.parametrize("H,group,D,B,n", [(1, 1, 128, 16, 20011), (2, 8, 128, 64, 9001), (8, 4, 64, 32, 12007),
                                           (1, 16, 64, 128, 30000)])
def test_attend_long_rows_are_joined(H, group, D, B, n):
    _attend([1, 1, 2], [n, 3, n // 2], H, group, D, B, torch.bfloat16, seed=n)


def test_attend_many_short_rows():
    rng = np.random.default_rng(1)
    kv = rng.integers(0, 90, 700).tolist()
    _attend([1] * 700, kv, 1, 2, 64, 16, torch.float16)
    _attend(rng.integers(0, 4, 300).tolist(), rng.integers(0, 90, 300).tolist(), 2, 3, 64, 16, torch.float16)


def test_attend_chunk_on_a_long_context():
    _attend([40, 1, 1], [6000, 3000, 10], 2, 4, 128, 64, torch.bfloat16)


@pytest.mark.parametrize("window", [1, 100, 1000])
def test_attend_window_on_long_rows(window):
    _attend([1, 1, 30], [5000, 900, 4000], 2, 4, 64, 16, torch.float16, window=window)


@pytest.mark.parametrize("spread", [0, 12, 30])
def test_attend_scales_far_apart(spread):
    """Blocks whose scales differ by up to 2^60: nothing is lost to a common one."""
    _attend([1, 1, 20], [100, 260, 300], 2, 4, 64, 16, torch.bfloat16, spread=spread, sm_scale=2.0 ** -(spread + 3))


def test_attend_large_scores():
    """Scores up to some thousands, where one position takes all the weight."""
    _attend([1, 50], [300, 400], 2, 4, 128, 32, torch.bfloat16, scale_up=100.0)


def test_attend_strided():
    _attend([1, 1, 1], [100, 50, 0], 2, 4, 128, 32, torch.bfloat16, strided=True)
    _attend([30, 1, 70], [100, 50, 90], 2, 4, 64, 32, torch.float16, strided=True)


@pytest.mark.parametrize("max_q", [0, 500])
def test_attend_without_a_tight_bound_on_the_tokens(max_q):
    _attend([1, 4, 90], [70, 60, 100], 2, 4, 64, 32, torch.float16, max_q=max_q)
    _attend([1, 1], [70, 60], 2, 4, 64, 32, torch.float16, max_q=max_q)


@pytest.mark.parametrize("q_len", [[1, 1, 1], [20, 3, 40]])
def test_attend_blocks_out_of_range_take_no_part(q_len):
    g = gen(2)
    kv = [200, 100, 170]
    table, N = P.paged(g, kv, 16)
    table[0, 3], table[0, 5], table[1, :7], table[2, 0] = -1, N, 1 << 29, -(1 << 31)
    k, v, ks, vs = P.random_cache(g, N, 2, 16, 64)
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    q = torch.randn((int(start[-1]), 6, 64), generator=g, device="cuda").half()
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got, lse = KV.Cache(k, v, ks, vs).attend(q, table, d(start), d(kv), return_lse=True)
    _near(got, lse, *P.attend_plain(q, k, v, ks, vs, table, start, kv, 0.125, True, 0))


@pytest.mark.parametrize("group,chunk", [(4, 3), (1, 16), (4, 60), (2, 200)])
def test_attend_nan_stays_where_it_is_seen(group, chunk):
    """A NaN in the cache reaches the tokens that see its position and no others, in K and in V."""
    for which in (0, 1):
        g = gen(6)
        kv = [chunk + 45, 80]
        table, N = P.paged(g, kv, 16)
        k, v, ks, vs = P.random_cache(g, N, 2, 16, 64)
        p = kv[0] - chunk // 2  # in the middle of the chunk
        (k, v)[which].view(torch.uint8)[table[0, p // 16].long(), 1, p % 16, 9] = 0x7f
        q = torch.randn((chunk + 1, 2 * group, 64), generator=g, device="cuda").half()
        d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        got, lse = KV.Cache(k, v, ks, vs).attend(q, table, d([0, chunk, chunk + 1]), d(kv), return_lse=True)
        sees = torch.zeros((chunk + 1, 2 * group), dtype=torch.bool, device="cuda")
        sees[p - 45:chunk, group:] = True
        assert torch.equal(torch.isnan(got).any(2), sees)
        assert torch.equal(torch.isnan(got).all(2), sees & (which == 0))
        if which == 1:
            assert torch.equal(torch.isnan(got[:, :, 9]), sees) and not bool(torch.isnan(got[:, :, :9]).any())
        assert torch.equal(torch.isnan(lse), sees & (which == 0))


def test_attend_tokens_that_no_row_owns_get_zeros():
    g = gen(7)
    table, N = P.paged(g, [30, 20], 16)
    k, v, ks, vs = P.random_cache(g, N, 2, 16, 64)
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for n, mq in (([1, 1], 1), ([9, 30], 30)):
        T = sum(n) + 5
        q = torch.randn((T, 4, 64), generator=g, device="cuda").half()
        out = torch.full_like(q, math.nan)
        got, lse = KV.Cache(k, v, ks, vs).attend(q, table, d([0, n[0], n[0] + n[1]]), d([30, 20]), max_q=mq, out=out,
                                                 return_lse=True)
        assert bool((got[T - 5:] == 0).all()) and bool((lse[T - 5:] == -math.inf).all())
        assert not bool(torch.isnan(got).any())


def test_attend_rows_above_max_q_get_zeros():
    g = gen(8)
    table, N = P.paged(g, [30, 60, 90], 16)
    k, v, ks, vs = P.random_cache(g, N, 1, 16, 64)
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q = torch.randn((31, 4, 64), generator=g, device="cuda").half()
    out = torch.full_like(q, math.nan)
    got, lse = KV.Cache(k, v, ks, vs).attend(q, table, d([0, 1, 30, 31]), d([30, 60, 90]), max_q=1, out=out, return_lse=True)
    assert bool((got[1:30] == 0).all()) and bool((lse[1:30] == -math.inf).all())
    assert not bool(torch.isnan(got).any()) and bool((got[0] != 0).any()) and bool((got[30] != 0).any())


def test_attend_offsets_past_32_bits():
    """Blocks that lie more than 2^32 bytes into k and v."""
    g = gen(10)
    B, H, D, N = 64, 8, 128, 70000  # 4.6 GB each
    shape = (N, H, B, D)
    k, v = (torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((N, H), device="cuda") for _ in range(2))
    last = [N - 1, N - 3, 3, 66000, N - 2]
    for x in (k, v):
        x[last] = (torch.randn((len(last), H, B, D), generator=g, device="cuda")).to(torch.float8_e4m3fn)
    x = torch.randn((3 + 40, H, D), generator=g, device="cuda").half()
    KV.Cache(k, v, ks, vs).append(x, -x, torch.tensor([(0, 3, N - 1, 2), (3, 40, N - 2, 0)], dtype=torch.int32).cuda())
    table = torch.tensor([last[:3] + [0], [last[3], last[4], 0, 0]], dtype=torch.int32, device="cuda")
    kv = [150, 100]
    sub = sorted(set(last))
    small = table.clone()
    for i, b in enumerate(sub):
        small[table == b] = i
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for q_len in ([1, 1], [90, 40]):
        start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
        q = torch.randn((int(start[-1]), 16, D), generator=g, device="cuda").half()
        got, lse = KV.Cache(k, v, ks, vs).attend(q, table, d(start), d(kv), return_lse=True)
        _near(got, lse, *P.attend_plain(q, k[sub], v[sub], ks[sub], vs[sub], small, start, kv, D ** -0.5, True, 0))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,heads,ctx,new", [(128, 8, [0] * 4, [4033, 4200, 4391, 4100]), (16, 2, [0] * 3, [3001, 2500, 2777]),
                                             (128, 1, list(range(40, 3000, 7)), [1] * 423), (32, 4, list(range(9, 2400, 40)), [5] * 60)])
def test_attend_takes_every_token_once(D, B, heads, ctx, new):
    """With q = 0 all tokens that a row sees weigh the same, and values that name their token's group of 16
    (and its 128) make the output count them: a tile that is read while the next one lands shows."""
    H, group, n = heads, 4, len(ctx)
    kv = torch.tensor(ctx) + torch.tensor(new)
    blocks = -(-kv // B)
    ids = torch.randperm(int(blocks.sum()), generator=torch.Generator().manual_seed(1))
    table, pos = torch.full((n, int(blocks.max())), -1, dtype=torch.int32), torch.empty(len(ids), dtype=torch.long)
    at = 0
    for r in range(n):
        m = int(blocks[r])
        table[r, :m] = ids[at:at + m].int()
        pos[ids[at:at + m]] = torch.arange(m) * B
        at += m
    half = D // 2
    tok = pos.cuda()[:, None] + torch.arange(B, device="cuda")
    v = torch.zeros((len(ids), B, D), device="cuda")
    v.scatter_(2, (tok // 16 % half)[..., None], 1.0)
    v.scatter_(2, (half + tok // 128 % half)[..., None], 1.0)
    v = v[:, None].expand(len(ids), H, B, D).to(torch.float8_e4m3fn).contiguous()
    scale = torch.ones((len(ids), H), device="cuda")
    cache = KV.Cache(torch.zeros_like(v.view(torch.uint8)).view(v.dtype), v, scale, scale.clone())
    start = torch.cumsum(torch.tensor([0] + new), 0).int().cuda()
    T = sum(new)
    q = torch.zeros((T, H * group, D), dtype=torch.bfloat16, device="cuda")
    # what row i of a request sees: tokens 0 .. ctx + i
    last = torch.cat([c + torch.arange(m) for c, m in zip(ctx, new)]).cuda()
    seen = torch.arange(int(kv.max()), device="cuda")
    code = torch.zeros((len(seen), D), dtype=torch.float64, device="cuda")
    code[seen, seen // 16 % half] = 1
    code[seen, half + seen // 128 % half] = 1
    want = torch.cumsum(code, 0)[last] / (last[:, None] + 1)
    for _ in range(12):
        out, lse = cache.attend(q, table.cuda(), start, kv.int().cuda(), max_q=max(new), return_lse=True)
        # a rounding to bf16 (2^-9), and those of the quotient in 32 bits
        far = (out.double() - want[:, None]).abs() > 2.0 ** -8 * want[:, None]
        assert not bool(far.any()), far.nonzero()[:4].tolist()
        # a log of a whole number in 32 bits, and its factor
        assert torch.allclose(lse.double(), torch.log((last + 1).double())[:, None].expand(T, H * group), rtol=0, atol=1e-5)


def test_operators_on_another_stream_and_in_a_graph():
    g = gen(11)
    n, B, H, D = 5, 16, 2, 64
    held = torch.tensor([30, 0, 16, 7, 64], dtype=torch.int32, device="cuda")
    add = torch.tensor([1, 40, 1, 1, 2], dtype=torch.int32, device="cuda")
    ids = torch.arange(40, dtype=torch.int32, device="cuda")
    table = torch.full((n, 8), -1, dtype=torch.int32, device="cuda")
    table[0, :2], table[2, :1], table[3, :1], table[4, :4] = ids[:2], ids[2:3], ids[3:4], ids[4:8]
    ring = ids.clone()
    state = torch.tensor([8, 32], dtype=torch.int64, device="cuda")
    k, v, ks, vs = P.random_cache(g, 40, H, B, D)
    start_k, start_v = k.clone(), v.clone()
    cache = KV.Cache(k, v, ks, vs)
    x = torch.randn((45, 4 * H, D), generator=g, device="cuda").half()
    step, out = KV.Step.empty(n, 45, B), torch.empty((45, 2 * H, D), dtype=torch.float16, device="cuda")
    work = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")

    def go(stream=None):
        KV.map_step(held, add, table, ring, state, 45, B, out=step, stream=stream)
        cache.append(x[:, 2 * H:3 * H], x[:, 3 * H:], step.runs, stream=stream)
        cache.attend(x[:, :2 * H], table, step.row_start, step.kv_len, max_q=40, out=out, workspace=work, stream=stream)

    go()
    torch.cuda.synchronize()
    want = out.clone()
    assert not bool(torch.isnan(want).any())
    side = torch.cuda.Stream()
    out.zero_()
    torch.cuda.synchronize()
    go(side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("handle", [False, True])
def test_a_named_stream_owns_what_a_call_allocates(handle):
    """Outputs and workspaces come from the call's stream, named by an object or by its handle."""
    side = torch.cuda.Stream()
    name = side.cuda_stream if handle else side
    with KV._on(torch.cuda.current_device(), name) as h:
        assert h == torch.cuda.current_stream().cuda_stream == side.cuda_stream
    with KV._on(torch.cuda.current_device(), 0) as h:
        assert h == torch.cuda.current_stream().cuda_stream == 0
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, ring, state = i(-1, -1).view(1, 2), i(1, 0, 2), torch.tensor([0, 3], device="cuda")
    torch.cuda.synchronize()
    step = KV.map_step(i(0), i(20), table, ring, state, 20, 16, stream=name)
    side.synchronize()
    assert step.slots.tolist() == list(range(16, 32)) + list(range(4)) and table.tolist() == [[1, 0]]


@pytest.mark.parametrize("B,D,group,most,dtype", [(16, 64, 4, 32, torch.float16), (64, 128, 8, 16, torch.bfloat16),
                                                  (128, 128, 16, 8, torch.float16), (32, 64, 3, 42, torch.bfloat16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 70), (True, 130), (True, 1000)])
def test_attend_chunks_of_half_an_item(B, D, group, most, dtype, causal, window):
    """No more tokens a request than a half of an item has: with a bound that says so and without one, over lengths of
    one tile, of few, and of more than a block's stretch."""
    q_len = [most, 0, 6, most - 1, 7, most, 6, 1, most, 5, most]
    kv_len = [most, 100, 6, 127, 129, 256, 0, 4, 3, 385, 9003]
    for max_q in (most, 0):
        _attend(q_len, kv_len, 2, group, D, B, dtype, causal=causal, window=window, seed=group + window, max_q=max_q)


@pytest.mark.parametrize("group,chunk", [(4, 5), (4, 32), (16, 8), (3, 42)])
def test_attend_nan_in_chunks_of_half_an_item(group, chunk):
    test_attend_nan_stays_where_it_is_seen(group, chunk)
