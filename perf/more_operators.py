"""Cases of the operators on either side of the serving step's cache: rotary positions of
queries and keys before it, and from logits to tokens behind it.

  rotate   q and k of a step's tokens are turned by their positions.  Row r's tokens are row_start[r] to
           row_start[r + 1], the last of the kv_len[r] that it holds; or each token's position is given
  adjust   logits: penalties for the tokens that a request's history holds, biases, grammar masks
  sample   logits, adjusted too, to a token and its log-probability: temperature, top-k, top-p, min-p, and a race
           of exponential random numbers among the tokens that are left

A case is a dict of plain values:

  op        "rotate", "adjust" or "sample"
  rows      requests in the batch
  dtype     "bf16", "f16" or "f32"
  for rotate:
    ctx     what a request holds before the step: "prompt" (1500 to 6000 tokens) or "fixed:N" (N to N + 5 %)
    step    "decode" (one token), "spec:N" (1 to N), "chunk:N" (row 0 N tokens, the others one),
            "prefill" (all its tokens, so that nothing is held before), "given:N" (N tokens a row, each with a
            position of its own anywhere below 2^20)
    heads, kv_heads, dim, rotary (values of a head that are turned), interleaved, scaling (0, or the factor by which
    the context is longer than the trained one, by bands of frequencies)
  for adjust and sample:
    vocab   logits of a row
    history tokens of a request so far: "none", "prompt" (1500 to 6000 and up to 400 written) or "fixed:N"
    bias    entries of a row's list of biases
    mask    share of the vocabulary that a row's grammar state allows, 0: no mask
    pick    for sample: "greedy", "plain" (temperature alone), "top-p", "top-k" or "mixed" (each row its own)
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def _rotate(name, rows, ctx, step, heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False, scaling=0.0, dtype="bf16"):
    c = dict(op="rotate", rows=rows, ctx=ctx, step=step, heads=heads, kv_heads=kv_heads, dim=dim, rotary=rotary,
             interleaved=interleaved, scaling=scaling, dtype=dtype)
    return dict(c, name=name) if name else c


def _adjust(name, rows, vocab, history, bias=0, mask=0.0, dtype="bf16"):
    c = dict(op="adjust", rows=rows, vocab=vocab, history=history, bias=bias, mask=mask, dtype=dtype)
    return dict(c, name=name) if name else c


def _sample(name, rows, vocab, pick, history="none", bias=0, mask=0.0, dtype="bf16"):
    c = dict(op="sample", rows=rows, vocab=vocab, pick=pick, history=history, bias=bias, mask=mask, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one instance with 16 slots, every slot decoding: latency
        _rotate("rotate-16-decode", 16, "prompt", "decode"),
        # 500 requests with a few drafted tokens each, half of a small head turned, pairs side by side
        _rotate("rotate-500-spec", 500, "prompt", "spec:5", 28, 4, 64, 32, True, 0.0, "f16"),
        # odd head sizes in 32 bits, tokens with positions of their own far into a long context
        _rotate("rotate-9-given", 9, "fixed:100", "given:701", 12, 12, 90, 30, False, 0.0, "f32"),
        # eight whole prompts, frequencies scaled for a context eight times the trained one
        _rotate("rotate-8-prefill", 8, "fixed:5600", "prefill", 32, 8, 128, 128, False, 8.0),
        # one request alone with everything on: latency
        _adjust("adjust-1", 1, 32000, "prompt", 20, 0.3),
        # 16 slots, each in a state of its grammar, after long prompts
        _adjust("adjust-16-long", 16, 131072, "fixed:24001", 0, 0.05, "f32"),
        # 301 requests on a vocabulary of odd size, penalties and biases in half precision
        _adjust("adjust-301-odd", 301, 50021, "prompt", 100, 0.0, "f16"),
        # 256 requests, everything on
        _adjust("adjust-256-all", 256, 131072, "prompt", 30, 0.3),
        # one request alone picks its token among the likeliest
        _sample("sample-1-top-p", 1, 32000, "top-p"),
        # 16 slots, each with parameters of its own, penalties and grammar masks
        _sample("sample-16-mixed", 16, 131072, "mixed", "prompt", 20, 0.3),
        # candidates of 301 queries by temperature alone, on a vocabulary of odd size, in 32 bits
        _sample("sample-301-plain", 301, 50021, "plain", dtype="f32"),
        # 256 requests among the likeliest tokens of a large vocabulary
        _sample("sample-256-top-p", 256, 131072, "top-p"),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(("rotate", "adjust", "sample"))
    if op == "rotate":
        dtype = rng.choice(("bf16", "f16", "f32"))
        kv_heads = rng.choice((1, 2, 3, 4, 8, 12))
        heads = kv_heads * rng.choice((1, 2, 4, 7, 8))
        dim = rng.choice((64, 80, 96, 128, 128, 192, 256, 90))
        rotary = rng.choice((dim, dim, dim // 2, 2 * (dim // 6)))
        rotary -= rotary % 2
        most = 44800 * 40 * 128 * 2 // ((heads + kv_heads) * dim * SIZE[dtype])  # tokens of the largest listed case's bytes
        step = rng.choice(("decode", "spec", "chunk", "prefill", "given"))
        ctx = rng.choice(("prompt", "fixed:%d" % _log(rng, 1, 200000)))
        if step == "prefill":
            ctx = "fixed:%d" % _log(rng, 1, min(most // 2, 9000))
            rows = _log(rng, 1, max(1, min(16, most * 9 // (10 * (int(ctx[6:]) + 1)))))
        elif step in ("decode", "spec"):
            rows, step = _log(rng, 1, min(4000, most // 8)), step if step == "decode" else "spec:%d" % rng.randint(2, 8)
        else:
            rows, n = _log(rng, 1, 30), _log(rng, 2, 512)
            step = "%s:%d" % (step, max(2, min(n, most // rows - 1)))
        return _rotate(None, rows, ctx, step, heads, kv_heads, dim, rotary, rng.random() < 0.5, rng.choice((0.0, 0.0, 4.0, 32.0)),
                       dtype)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    vocab = _log(rng, 500, 260000)
    most = 256 * 131072 * 2 // (SIZE[dtype] * (2 if op == "sample" else 1))
    rows = _log(rng, 1, max(1, min(700, most // vocab)))
    history = rng.choice(("none", "prompt", "fixed:%d" % _log(rng, 1, 30000)))
    bias, mask = rng.choice((0, 0, 3, 50, 300)), rng.choice((0.0, 0.0, 0.01, 0.3, 0.9))
    if op == "adjust":
        history = "prompt" if history == "none" and not bias and not mask else history  # something to do
        return _adjust(None, rows, vocab, history, bias, mask, dtype)
    return _sample(None, rows, vocab, rng.choice(("greedy", "plain", "top-p", "top-k", "mixed", "mixed")), history, bias,
                   mask, dtype)


def _lengths(case):
    """What each row holds before the step and what the step adds, on the host: they follow from the
    case alone, so that the work is the same for every seed."""
    g = torch.Generator().manual_seed(631 + case["rows"])
    n = case["rows"]
    u = torch.rand(n, generator=g, dtype=torch.float64)
    kind = case["ctx"] if case["op"] == "rotate" else case["history"]
    if kind == "none":
        return torch.zeros(n, dtype=torch.long), torch.zeros(n, dtype=torch.long)
    if kind == "prompt":
        held = (1500 + u * 4501).long()
    else:
        base = int(kind.split(":")[1])
        held = (base + u * (base // 20 + 1)).long()
    if case["op"] != "rotate":
        most = 400 if kind == "prompt" else 1 + base // 2
        return held, torch.randint(0, most + 1, (n,), generator=g)  # prompt, written
    step, _, arg = case["step"].partition(":")
    add = torch.ones(n, dtype=torch.long)
    if step == "spec":
        add = torch.randint(1, int(arg) + 1, (n,), generator=g)
    elif step == "chunk":
        add[0] = int(arg)
    elif step == "prefill":
        return torch.zeros(n, dtype=torch.long), held
    elif step == "given":
        add[:] = int(arg)
    return held, add


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _frequencies(case):
    """Radians a position for each pair of values, in 64 bits."""
    R = case["rotary"]
    f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if case["scaling"]:
        turns = 8192 * f / (2 * math.pi)  # over the context that was trained
        share = ((turns - 1) / (32 - 1)).clamp(0, 1)
        f = (1 - share) * f / case["scaling"] + share * f
    return f


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(int(seed) * 6007 + 29)
    held, add = _lengths(case)
    n, dt = case["rows"], DTYPES[case["dtype"]]
    s = dict(op=case["op"])

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    def rand(*shape):
        return torch.rand(shape, generator=g, device=dev, dtype=torch.float32)

    if case["op"] == "rotate":
        T, H, K = int(add.sum()), case["heads"], case["kv_heads"]
        qkv = randn(T, H + 2 * K, case["dim"]).to(dt)  # the projections' output, q, k and v of a token side by side
        s.update(q=qkv[:, :H], k=qkv[:, H:H + K], frequencies=_frequencies(case), interleaved=case["interleaved"],
                 scale=0.1 * math.log(case["scaling"]) + 1 if case["scaling"] else 1.0)
        if case["step"].startswith("given"):
            s["positions"] = torch.randint(0, 1 << 20, (T,), generator=g, device=dev, dtype=torch.int32)
        else:
            zero = torch.zeros(1, dtype=torch.long)
            s.update(row_start=torch.cat([zero, torch.cumsum(add, 0)]).int().to(dev), kv_len=(held + add).int().to(dev))
        s["turned"] = s["frequencies"].to(dev)
        return s
    V = case["vocab"]
    # logits as a model gives them: most of them small, a few dozen far above the others
    x = randn(n, V) * 2.2 - 3
    some = torch.randint(0, V, (n, 40), generator=g, device=dev)
    x.scatter_add_(1, some, 14 * rand(n, 40))
    s.update(logits=x.to(dt), vocab=V)
    rules = {}
    if case["history"] != "none":
        width = int((held + add).max()) + 7
        # a text's tokens: few of them often, and most of the likely next ones among them
        h = (V * rand(n, width) ** 4).long().clamp(max=V - 1)
        h = torch.where(rand(n, width) < 0.1, some[:, :1].expand(-1, width), h)
        h = torch.where(rand(n, width) < 0.05, torch.gather(some, 1, torch.randint(0, 40, (n, width), generator=g, device=dev)), h)
        rules.update(history=h.int(), prompt_len=held.int().to(dev), length=(held + add).int().to(dev),
                     repetition=1 + 0.3 * rand(n), presence=0.6 * rand(n), frequency=0.2 * rand(n))
    if case["bias"]:
        b = case["bias"]
        at = torch.randint(0, V, (n, b), generator=g, device=dev)
        at[:, :1 + b // 4] = some[:, :1].expand(-1, 1 + b // 4)  # the same token more than once, too
        rules.update(bias_start=b * torch.arange(n + 1, device=dev, dtype=torch.int32), bias_token=at.int().view(-1),
                     bias_value=3 * randn(n * b))
    if case["mask"]:
        # states of a grammar: each allows its own part of the vocabulary; rows are in any of them, some in none
        states, words = max(1, n // 2), (V + 31) // 32
        allow = rand(states, words * 32) < case["mask"]
        allow[:, ::97] = True
        bit = torch.tensor(1, dtype=torch.int64, device=dev) << torch.arange(32, device=dev)
        bits = (allow.view(states, words, 32).long() * bit).sum(-1)
        state = torch.randint(0, states, (n,), generator=g, device=dev)
        state[1::8] = -1
        rules.update(mask=torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int(), mask_row=state.int())
    s["rules"] = rules
    if case["op"] == "sample":
        pick = case["pick"]
        kind = torch.arange(n, device=dev) % 5 if pick == "mixed" else torch.full(
            (n,), {"greedy": 0, "plain": 1, "top-p": 2, "top-k": 3}[pick], device=dev)
        T = 0.5 + rand(n)
        s.update(noise=torch.empty((n, V), dtype=torch.float32, device=dev).exponential_(generator=g),
                 temperature=torch.where(kind == 0, 0, T),
                 top_p=torch.where((kind == 2) | (kind == 4), 0.7 + 0.28 * rand(n), 1.0),
                 top_k=torch.where(kind >= 3, torch.randint(2, 200, (n,), generator=g, device=dev), 0).int(),
                 min_p=torch.where(kind == 4, 0.02 * rand(n), 0.0))
    return s


def _plain_rotate(s):
    T = s["q"].shape[0]
    if "positions" in s:
        pos = s["positions"].long()
    else:
        row_start, kv_len = s["row_start"].long(), s["kv_len"].long()
        t = torch.arange(T, device=row_start.device)
        row = torch.searchsorted(row_start[1:], t, right=True)
        pos = kv_len[row] - row_start[row + 1] + t
    angle = pos.double()[:, None] * s["turned"]  # 32 bits lose far positions
    cos, sin = (torch.cos(angle) * s["scale"]).float()[:, None], (torch.sin(angle) * s["scale"]).float()[:, None]
    R = 2 * s["turned"].shape[0]

    def turn(x):
        y = x.float()
        if s["interleaved"]:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            z = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            z = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([z, y[..., R:]], -1).to(x.dtype)

    return dict(q=turn(s["q"]), k=turn(s["k"]))


def _plain_adjust(s):
    """Adjusted logits in 32 bits."""
    x, r, V = s["logits"].float(), s["rules"], s["vocab"]
    n, dev = x.shape[0], x.device
    if "history" in r:
        h = r["history"].long()
        at = torch.arange(h.shape[1], device=dev)[None]
        there = (at < r["length"][:, None]) & (h >= 0) & (h < V)
        h = h.clamp(0, V - 1)
        count = torch.zeros((n, V), dtype=torch.int32, device=dev)
        count.scatter_add_(1, h, (there & (at >= r["prompt_len"][:, None])).int())
        seen = torch.zeros((n, V), dtype=torch.int32, device=dev).scatter_add_(1, h, there.int()) > 0
        rep = r["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = x - (r["frequency"][:, None] * count + r["presence"][:, None] * (count > 0))
    if "bias_start" in r:
        row = torch.repeat_interleave(torch.arange(n, device=dev), torch.diff(r["bias_start"].long()),
                                      output_size=r["bias_token"].shape[0])
        entry = torch.arange(row.shape[0], device=dev)
        last = torch.full((n * V,), -1, dtype=torch.long, device=dev)
        last.scatter_reduce_(0, row * V + r["bias_token"].long(), entry, "amax")  # the last of several counts
        last = last.view(n, V)
        x = torch.where(last >= 0, x + r["bias_value"][last.clamp(min=0)], x)
    if "mask" in r:
        t = torch.arange(V, device=dev)
        state = r["mask_row"].long()
        word = r["mask"][state.clamp(min=0)][:, t // 32]
        x = torch.where(((word >> (t % 32)) & 1 == 1) | (state < 0)[:, None], x, -math.inf)
    return x


def _plain_sample(s):
    x = _plain_adjust(s)
    n, V = x.shape
    greedy = ~(s["temperature"] > 0)
    T = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    x, index = torch.sort(x, dim=1, descending=True, stable=True)
    top = x[:, :1]
    z = torch.where(x > -math.inf, (x.double() - top) / T, -math.inf)  # 64 bits: sums up to a border
    w = torch.exp(z)
    rank = torch.arange(V, device=x.device)[None]
    k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    keep = (x > -math.inf) & (rank < k)
    mass = torch.cumsum(torch.where(keep, w, 0), 1)
    p = s["top_p"].double()[:, None]
    keep = keep & ((p >= 1) | (mass - w < p * mass[:, -1:]) | (rank == 0))
    keep = keep & ((w >= s["min_p"].double()[:, None]) | (rank == 0))
    score = torch.where(keep, z - torch.log(torch.gather(s["noise"], 1, index).double()), -math.inf)
    best = torch.where(keep & (score == score.amax(1, keepdim=True)), index, V).amin(1)  # the lowest of equals
    token = torch.where(greedy, index[:, 0], best)
    mine = torch.where(index == token[:, None], z, -math.inf).amax(1)
    logprob = mine - torch.log(w.sum(1))
    none = top[:, 0] == -math.inf
    return dict(token=torch.where(none, -1, token).int(), logprob=torch.where(none, -math.inf, logprob).float())


def _own(s):
    from paper_2505_05286_gb300 import kvcache, logits
    if s["op"] == "rotate":
        if "rope" not in s:  # the program's table of frequencies
            s["rope"] = kvcache.Rope(s["frequencies"], interleaved=s["interleaved"], scale=s["scale"])
        if "positions" in s:
            q, k = s["rope"].rotate(s["q"], s["k"], positions=s["positions"])
        else:
            q, k = s["rope"].rotate(s["q"], s["k"], s["row_start"], s["kv_len"])
        return dict(q=q, k=k)
    if "handle" not in s:  # the program's tables of what holds for its requests
        r = s["rules"]
        bias = (r["bias_start"], r["bias_token"], r["bias_value"]) if "bias_start" in r else None
        s["handle"] = logits.Rules(bias=bias, **{name: r[name] for name in r if not name.startswith("bias")})
    if s["op"] == "adjust":
        return dict(logits=logits.adjust(s["logits"], s["handle"]))
    token, logprob = logits.sample(s["logits"], s["noise"], temperature=s["temperature"], top_k=s["top_k"],
                                   top_p=s["top_p"], min_p=s["min_p"], rules=s["handle"])
    return dict(token=token, logprob=logprob)


def run(state):
    if own:
        return _own(state)
    if state["op"] == "rotate":
        return _plain_rotate(state)
    if state["op"] == "adjust":
        return dict(logits=_plain_adjust(state).to(state["logits"].dtype))
    return _plain_sample(state)


def work(case):
    held, add = _lengths(case)
    n, size = case["rows"], SIZE[case["dtype"]]
    if case["op"] == "rotate":
        T = int(add.sum())
        h = case["heads"] + case["kv_heads"]
        tables = 4 * T if case["step"].startswith("given") else 8 * n
        return {"bytes": 2 * T * h * case["dim"] * size + tables + 4 * case["rotary"], "flops": 3 * T * h * case["rotary"]}
    V = case["vocab"]
    b = n * V * size
    if case["history"] != "none":
        b += 4 * int((held + add).sum()) + 20 * n
    b += 8 * n * case["bias"]
    if case["mask"]:
        b += 4 * min(n, max(1, n // 2)) * ((V + 31) // 32) + 4 * n
    if case["op"] == "adjust":
        return {"bytes": b + n * V * size, "flops": 4 * n * V}
    # random numbers: of every token where none is left out, of a few where only the likeliest are
    free = n if case["pick"] == "plain" else (n + 3) // 5 if case["pick"] == "mixed" else 0
    share = case["mask"] or 1.0
    return {"bytes": b + int(4 * free * V * min(1.0, 8 * share)) + 24 * n, "flops": 6 * n * V}


def _exact_rotate(s):
    T = s["q"].shape[0]
    if "positions" in s:
        pos = s["positions"].double().cpu()
    else:
        pos = torch.cat([torch.arange(int(b) - int(n), int(b)) for b, n in
                         zip(s["kv_len"].tolist(), torch.diff(s["row_start"]).tolist())]).double()
    f = s["frequencies"]
    m = f.shape[0]
    turn = torch.polar(torch.full((T, m), float(s["scale"]), dtype=torch.float64), pos[:, None] * f[None]).to(s["q"].device)
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for h in range(x.shape[1]):
            if s["interleaved"]:
                z = turn * torch.view_as_complex(x[:, h, :2 * m].reshape(T, m, 2).contiguous())
                y[:, h, :2 * m] = torch.view_as_real(z).reshape(T, 2 * m)
            else:
                z = turn * torch.complex(x[:, h, :m], x[:, h, m:2 * m])
                y[:, h, :m], y[:, h, m:2 * m] = z.real, z.imag
        out[name] = y
    return out


def _exact_row(s, i):
    """One row's adjusted logits."""
    x, r, V = s["logits"][i].double(), s["rules"], s["vocab"]
    if "history" in r:
        n, m = int(r["length"][i]), int(r["prompt_len"][i])
        h = r["history"][i, :n].long()
        h, written = h[(h >= 0) & (h < V)], h[m:][(h[m:] >= 0) & (h[m:] < V)]
        token, times = torch.unique(written, return_counts=True)
        seen = torch.unique(h)
        rep = float(r["repetition"][i])
        x[seen] = torch.where(x[seen] > 0, x[seen] / rep, x[seen] * rep)
        x[token] -= float(r["frequency"][i]) * times.double() + float(r["presence"][i])
    if "bias_start" in r:
        a, b = int(r["bias_start"][i]), int(r["bias_start"][i + 1])
        for t, v in dict(zip(r["bias_token"][a:b].tolist(), r["bias_value"][a:b].tolist())).items():
            x[t] += v
    if "mask" in r and int(r["mask_row"][i]) >= 0:
        word = r["mask"][int(r["mask_row"][i])].long() & 0xffffffff
        allowed = torch.stack([(word >> j) & 1 for j in range(32)], 1).reshape(-1)[:V]
        x[allowed == 0] = -math.inf
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return _exact_rotate(s)
    rows = range(case["rows"])
    if case["op"] == "adjust":
        return dict(logits=torch.stack([_exact_row(s, i) for i in rows]))
    tokens, logprobs = [], []
    for i in rows:
        x = _exact_row(s, i)
        T, k, p, m = (float(s[name][i]) for name in ("temperature", "top_k", "top_p", "min_p"))
        z = x / T if T > 0 else x
        total = torch.logsumexp(z, 0)
        if not bool(total > -math.inf):
            tokens.append(-1)
            logprobs.append(-math.inf)
            continue
        order = torch.argsort(x, descending=True, stable=True)
        order = order[x[order] > -math.inf]
        if T > 0:
            order = order[:int(k)] if k > 0 else order
            q = torch.softmax(z[order], 0)
            if p < 1:
                order = order[:1 + int((torch.cumsum(q, 0) < p).sum())]
                q = q[:len(order)]
            order = order[:max(1, int((q >= m * q[0]).sum()))]
            at = torch.exp(z[order] - z[order[0]]) / s["noise"][i][order].double()
            t = int(order[at == at.max()].min())
        else:
            t = int(order[0])
        tokens.append(t)
        logprobs.append(float(z[t] - total))
    return dict(token=torch.tensor(tokens, dtype=torch.int32), logprob=torch.tensor(logprobs, dtype=torch.float64))
