"""Plain 64-bit implementations of the cache operators, for their tests: loops
over requests, blocks and tokens on the host."""
from __future__ import annotations

import math

import numpy as np
import torch

E4M3_MAX = 448.0


def map_plain(held, add, table, ring, state, n_tokens, B, n_runs_len):
    """One step's tables as include/hxkv.h words them; table and ring are changed in place."""
    n, width, cap = len(held), table.shape[1], len(ring)
    head, free = int(state[0]), int(state[1])
    row_start, kv_len = np.zeros(n + 1, np.int32), np.zeros(n, np.int32)
    slots = np.full(n_tokens, -1, np.int64)
    runs = np.zeros((n_runs_len, 4), np.int32)
    t = asked = taken = refused = at_run = 0
    ended = []
    for r in range(n):
        h, a = int(held[r]), int(add[r])
        tok = max(a, 0)
        row_start[r] = min(t, n_tokens)
        bad = h < 0 or a < -1 or -(-(h + tok) // B) > width
        need = 0 if bad else -(-(h + tok) // B) - -(-h // B)
        mine = 0 if bad or tok == 0 else (h + tok - 1) // B - h // B + 1
        asked += need
        if bad or (tok and ((need and asked > free) or t + tok > n_tokens)):
            refused += 1
        elif tok:
            first = asked - need
            for j in range(need):
                table[r, -(-h // B) + j] = ring[(head + first + j) % cap]
            taken += need
            for i in range(tok):
                p = h + i
                slots[t + i] = int(table[r, p // B]) * B + p % B
                if i == 0 or p % B == 0:
                    runs[at_run + p // B - h // B] = (t + i, min(B - p % B, tok - i), table[r, p // B], p % B)
            kv_len[r] = h + tok
        elif a == 0:
            kv_len[r] = h
        else:
            ended += [int(b) for b in table[r, :-(-h // B)]]
        t += tok
        at_run += mine
    row_start[n] = min(t, n_tokens)
    for j, b in enumerate(ended):
        ring[(head + free + j) % cap] = b
    counts = np.array([min(t, n_tokens), at_run, refused, taken], np.int32)
    return row_start, kv_len, slots, runs, counts, np.array([(head + taken) % cap, free - taken + len(ended)], np.int64)


def e4m3_grid():
    """Every finite e4m3 value of either sign, by its byte."""
    out = np.full(256, np.nan)
    for b in range(256):
        s, e, m = b >> 7, (b >> 3) & 15, b & 7
        if e == 15 and m == 7:
            continue
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = -v if s else v
    return out


GRID = e4m3_grid()
_POS = GRID[:127]  # 0 .. 448, ascending


def to_e4m3(x):
    """Bytes of float64 values: nearest, ties to even, infinities and more than 448 to 448, NaN to 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), E4M3_MAX)
    hi = np.clip(np.searchsorted(_POS, a, "left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    pick = np.where(_POS[hi] == a, hi, pick)
    out = pick.astype(np.uint8) | (np.signbit(x).astype(np.uint8) << 7)
    return np.where(np.isnan(x), 0x7f, out).astype(np.uint8)


def scale_of(amax):
    e = -100
    if amax > 0:
        e = max(-100, math.frexp(amax)[1] - 12)
        while math.ldexp(448.0, e) < amax:
            e += 1
    return math.ldexp(1.0, e)


def append_plain(x, cache, scale, runs):
    """x [tokens, heads, dim] float64; cache uint8 [blocks, heads, B, dim] and scale float64 [blocks, heads], in place."""
    N, heads, B, D = cache.shape
    for t0, n, blk, off in runs.tolist():
        if n <= 0 or t0 < 0 or t0 + n > len(x) or off < 0 or off + n > B or not 0 <= blk < N:
            continue
        for h in range(heads):
            new = x[t0:t0 + n, h]
            size = np.abs(new[np.isfinite(new)])
            was = scale[blk, h] if off else 0.0
            now = max(was, scale_of(float(size.max()) if size.size else 0.0))
            if off and now > was:
                cache[blk, h, :off] = to_e4m3(GRID[cache[blk, h, :off]] * (was / now))
            cache[blk, h, off:off + n] = to_e4m3(new / now)
            scale[blk, h] = now


def attend_plain(q, k, v, k_scale, v_scale, table, row_start, kv_len, sm_scale, causal, window):
    """out, lse and bounds of their rounding errors, all float64 on q's device.

    The bounds: every score is a sum of dim products in 32 bits (each partial sum off by
    2^-24 of the sizes so far, twice that for the factors and the exponential's
    argument), a weight may be rounded to 16 bits (2^-11 of it, or 2^-25 near
    zero), sums of weights and of weighted values stay in 32 bits."""
    T, heads, D = q.shape
    H, B, N = k.shape[1], k.shape[2], k.shape[0]
    g = heads // H
    dev = q.device
    out = torch.zeros((T, heads, D), dtype=torch.float64, device=dev)
    lse = torch.full((T, heads), -math.inf, dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros((T, heads), dtype=torch.float64, device=dev)
    val = torch.tensor(GRID, device=dev)
    for r in range(len(kv_len)):
        a, b, n = int(row_start[r]), int(row_start[r + 1]), min(int(kv_len[r]), table.shape[1] * B)
        if a >= b or n <= 0:
            continue
        ids = table[r, :-(-n // B)].long()
        ok = ((ids >= 0) & (ids < N)).repeat_interleave(B)[:n]
        ids = ids.clamp(0, N - 1)
        for h in range(H):
            kk = (val[k.view(torch.uint8)[ids, h].long()] * k_scale[ids, h].double()[:, None, None]).reshape(-1, D)[:n]
            vv = (val[v.view(torch.uint8)[ids, h].long()] * v_scale[ids, h].double()[:, None, None]).reshape(-1, D)[:n]
            for i in range(a, b):
                p = n - (b - a) + i - a
                j = torch.arange(n, device=dev)
                see = ok & ((j <= p) if causal else (j < n))
                if window:
                    see = see & (j > p - window)
                if not bool(see.any()):
                    continue
                K, V = kk[see], vv[see]
                Q = q[i, h * g:(h + 1) * g].double()
                s = Q @ K.T * sm_scale
                size = (Q.abs() @ K.abs().T * abs(sm_scale)).amax(1, keepdim=True)
                ds = 2 * D * 2.0 ** -24 * size + 2.0 ** -22 * s.abs().amax(1, keepdim=True)
                top = s.amax(1, keepdim=True)
                w = torch.exp(s - top)
                total = w.sum(1, keepdim=True)
                o = w @ V / total
                hs = slice(h * g, (h + 1) * g)
                out[i, hs] = o
                lse[i, hs] = (top + torch.log(total))[:, 0]
                few = 2.0 ** -25 * V.abs().sum(0, keepdim=True) / total
                tol[i, hs] = (2.0 ** -10 + 4 * ds) * (w @ V.abs() / total) + 2 * few
                ltol[i, hs] = (2 * ds + 2.0 ** -19)[:, 0] + 2.0 ** -22 * lse[i, hs].abs()
    unit = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -11
    tiny = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    return out, lse, tol + unit * out.abs() + tiny, ltol


def random_cache(g, n_blocks, H, B, D, spread=2, dev="cuda"):
    """k, v, k_scale, v_scale with power-of-two scales over 2 * spread binades."""
    out = []
    for _ in range(2):
        x = (torch.randn((n_blocks, H, B, D), generator=g, device=dev) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        out += [x, torch.exp2(torch.randint(-7 - spread, -7 + spread + 1, (n_blocks, H), generator=g, device=dev).float())]
    return out[0], out[2], out[1], out[3]


def paged(g, kv_len, B, extra=2, spare=3, dev="cuda"):
    """(table, blocks): rows over a random permutation of blocks; what a row does not use is -1 or out of range."""
    need = [-(-max(n, 0) // B) for n in kv_len]
    n_blocks = sum(need) + spare
    ids = torch.randperm(n_blocks, generator=g, device=dev).int().cpu()
    table = torch.full((len(kv_len), max(need + [0]) + extra), -1, dtype=torch.int32)
    table[:, -1] = 1 << 30
    at = 0
    for r, m in enumerate(need):
        table[r, :m] = ids[at:at + m]
        at += m
    return table.to(dev), n_blocks
