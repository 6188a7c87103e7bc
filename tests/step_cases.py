"""Plain implementations in 64 bits of the operators on either side of the cache,
for their tests: loops over rows and tokens on the host."""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24  # a rounding in 32 bits, of a value
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # of what is below the normal numbers


def rotate_plain(x, positions, frequencies, interleaved, scale, inverse=False):
    """(result in 64 bits, its tolerance) for x [tokens, heads, dim]."""
    dt = x.dtype
    x = x.double().cpu()
    f = torch.as_tensor(frequencies, dtype=torch.float64)
    m = len(f)
    angle = positions.double().cpu()[:, None] * f[None] * (-1 if inverse else 1)
    c, s = torch.cos(angle)[:, None] * scale, torch.sin(angle)[:, None] * scale
    a, b = (x[..., 0:2 * m:2], x[..., 1:2 * m:2]) if interleaved else (x[..., :m], x[..., m:2 * m])
    p, q = a * c - b * s, a * s + b * c
    # cosine and sine: the angle converted to 32 bits (2^-25 of pi / 4 at most), the function's last place (2^-24), the
    # factor `scale` (2^-24); then a product and a product with its sum (2^-24 each, of the larger term): below 6
    # roundings of |a| + |b|; and what 64 bits lose themselves in a far angle
    far = angle.abs()[:, None] * 2.0 ** -52
    off = (6 * U + far) * abs(scale) * (a.abs() + b.abs())
    y, tol = x.clone(), torch.zeros_like(x)
    for part, err, where in ((p, off, 0), (q, off, 1)):
        at = slice(where, 2 * m, 2) if interleaved else slice(where * m, (where + 1) * m)
        y[..., at] = part
        tol[..., at] = err + (part.abs() + err) * torch.finfo(dt).eps / 2 + TINY[dt]
    return y, tol


def words_of(history, length, prompt_len, vocab):
    """Times written and whether seen, by token, of one row."""
    times, seen = np.zeros(vocab, np.int64), np.zeros(vocab, bool)
    for i in range(max(0, min(int(length), len(history)))):
        t = int(history[i])
        if 0 <= t < vocab:
            seen[t] = True
            if i >= prompt_len:
                times[t] += 1
    return times, seen


def adjust_plain(x, rules, dtype=np.float64):
    """(adjusted rows, tolerance) in `dtype`: float32 rounds as the definition does.  rules: dict of numpy arrays with the names
    of logits.Rules."""
    F = dtype
    n, V = x.shape
    out, tol = x.astype(F), np.zeros((n, V))
    for r in range(n):
        y, e = out[r], tol[r]
        if rules.get("history") is not None:
            m = rules["prompt_len"][r] if rules.get("prompt_len") is not None else 0
            times, seen = words_of(rules["history"][r], rules["length"][r], m, V)
            one = lambda name, default: F(rules[name][r]) if rules.get(name) is not None else F(default)
            rep, pres, freq = one("repetition", 1), one("presence", 0), one("frequency", 0)
            z = np.where(seen, np.where(y > 0, y / rep, y * rep), y)
            off = np.where(times > 0, freq * times.astype(F) + pres, F(0))
            y[:] = np.where(times > 0, z - off, z)
            with np.errstate(invalid="ignore"):
                e += np.where(seen, U * np.abs(z), 0) + np.where(times > 0, 2 * U * (abs(freq) * times + abs(pres)) + U * np.abs(y), 0)
        if rules.get("bias_start") is not None:
            a, b = (int(min(max(v, 0), len(rules["bias_token"]))) for v in rules["bias_start"][r:r + 2])
            last = {}
            for j in range(a, min(b, a + 4095)):
                if 0 <= rules["bias_token"][j] < V:
                    last[int(rules["bias_token"][j])] = j
            for t, j in last.items():
                y[t] = y[t] + F(rules["bias_value"][j])
                e[t] += U * abs(float(y[t]))
        if rules.get("mask") is not None:
            m = rules["mask_row"][r] if rules.get("mask_row") is not None else r
            if 0 <= m < len(rules["mask"]):
                w = rules["mask"][m].astype(np.int64) & 0xffffffff
                t = np.arange(V)
                y[((w[t // 32] >> (t % 32)) & 1) == 0] = -np.inf
    return out, tol


def sample_plain(x, noise, temperature, top_k, top_p, min_p):
    """One row: (token, logprob, tolerance of logprob) of adjusted logits x, float32 exact."""
    x = x.astype(np.float64)
    V = len(x)
    nan = bool(np.isnan(x).any())
    x = np.where(np.isnan(x), -np.inf, x)
    if not (x > -np.inf).any():
        return -1, math.nan if nan else -math.inf, 0.0
    T = np.float64(temperature) if temperature > 0 else np.float64(1)
    top = x.max()
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        z = np.where(x == top, 0.0, np.where(x > -np.inf, (x - top) / T, -np.inf))
    z = np.where(np.isnan(z), -np.inf, z)  # infinity less infinity: next to an infinite one the others weigh nothing
    w = np.where(x > -np.inf, np.exp(z), 0)
    order = np.lexsort((np.arange(V), -x))
    order = order[x[order] > -np.inf]
    total = w.sum()
    token = int(order[0])
    if temperature > 0 and noise is not None:
        kept = order[:top_k] if top_k > 0 else order
        if top_p < 1:
            mass = np.cumsum(w[kept])
            kept = kept[:max(1, int((mass - w[kept] < top_p * mass[-1]).sum()))]
        if min_p > 0:
            kept = kept[:max(1, int((w[kept] >= min_p).sum()))]
        e = noise[kept].astype(np.float64)
        fine = (e >= 2.0 ** -126) & (e < np.inf)
        score = np.where(fine, z[kept] - np.log(np.where(fine, e, 1)), -np.inf)
        if (score > -np.inf).any():
            token = int(kept[score == score.max()].min())
    lp = z[token] - math.log(total)
    # weights: five roundings of the exponent (difference, 1 / T, product, 1 / log 2, product) and exp2f's two last places (4
    # roundings' worth); at most 16 + 5 + 5 additions in a row; the result's own rounding
    y = float((np.where(w > 0, -z, 0) * w).sum() / total)
    tol = U * (5 * y + 4 + 26 + abs(lp))
    return token, (math.nan if nan else lp), tol


def random_rules(rng, n, V, history=0, bias=0, mask=0.0, odd=True):
    """Rules of all kinds as numpy arrays; odd: entries out of range, rows without anything."""
    r = {}
    if history:
        h = (V * rng.random((n, history)) ** 3).astype(np.int32)
        if odd:
            h[rng.random(h.shape) < 0.05] = -1
            h[rng.random(h.shape) < 0.02] = V
        length = rng.integers(0, history + 1, n)
        prompt = rng.integers(0, history + 1, n)
        if odd and n > 2:
            length[0], length[1], prompt[2] = 0, history + 9, -3
            length[2 % n] = -4 if n > 3 else history
        r.update(history=h, length=length.astype(np.int32), prompt_len=prompt.astype(np.int32),
                 repetition=(0.8 + rng.random(n)).astype(np.float32), presence=(rng.random(n) - 0.3).astype(np.float32),
                 frequency=(0.3 * rng.random(n)).astype(np.float32))
    if bias:
        per = rng.integers(0, bias + 1, n)
        start = np.concatenate([[0], np.cumsum(per)])
        tok = rng.integers(-1 if odd else 0, V + (1 if odd else 0), start[-1])
        tok[::3] = tok[:1] if len(tok) else 0
        r.update(bias_start=start.astype(np.int32), bias_token=tok.astype(np.int32),
                 bias_value=(4 * rng.standard_normal(start[-1])).astype(np.float32))
    if mask:
        m, words = max(1, n // 2), (V + 31) // 32
        bits = rng.random((m, words * 32)) < mask
        w = (bits.reshape(m, words, 32) * (1 << np.arange(32, dtype=np.int64))).sum(-1)
        row = rng.integers(0, m, n)
        if odd:
            row[::4] = -1
            row[1::7] = m
        r.update(mask=w.astype(np.uint32).view(np.int32), mask_row=row.astype(np.int32))
    return r


def rules_on_gpu(r):
    from paper_2505_05286_gb300 import logits
    d = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in r.items() if not k.startswith("bias")}
    bias = tuple(torch.from_numpy(r[k]).cuda() for k in ("bias_start", "bias_token", "bias_value")) if "bias_start" in r else None
    return logits.Rules(bias=bias, **d)
