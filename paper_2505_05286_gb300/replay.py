"""Replay of an instance's running batch: the calls that a logged simulation put
on one instance, run as serving steps of the cache operators on this GPU.

The simulator describes an instance by prompt tokens per second, microseconds
per output token and slots, which do not depend on what the batch holds.  What
does depend on it is the cache: a step maps its tokens to blocks, writes their
keys and values and attends to all that its requests hold.  A replay takes
the calls of one instance in the order in which they started, keeps the instance's
slots filled with them (a prompt comes in chunks, then one token a step),
and times every step on the GPU, so that the constant rates can be held against a
measured cost and its growth with the context.  Before each step a buffer larger than L2
is written: a step finds the cache in device memory, as it does after the other layers'
work, and its launches are waiting when it begins.

    rep = replay(trace, records, cluster, instance=0)
    rep["us_per_step"], rep["us_per_1000_tokens"]     # of steps in which every request decodes
    rep["prompt_us_per_token"]

With Shape.theta queries and keys are turned by their positions first, and with Shape.vocab each row's next token is drawn from
logits at the end, with penalties for the tokens that its request holds; the random numbers for that are written between the steps, outside
of their time.

Queries, keys, values and logits are random; a real model's products are not part of it.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import List, Optional

import numpy as np
import torch

from . import hxsim as H
from . import kvcache as KV
from . import logits as L


@dataclass
class Shape:
    """The attention of one layer; theta: the base of its rotary positions (0: none); vocab: the step ends with a
    token for each row from so many logits (0: it does not)."""
    heads: int = 32
    kv_heads: int = 8
    head_dim: int = 128
    block_tokens: int = 64
    dtype: torch.dtype = torch.bfloat16
    theta: float = 0.0
    vocab: int = 0


@dataclass
class Call:
    """One call: the prompt to read, then the tokens to write (at least one step)."""
    prompt: int
    out: int
    read: int = 0
    written: int = 0


def calls_of(trace, records: dict, instance: int) -> List[Call]:
    """The calls that a recorded simulation started on `instance`, by start time (ties: request id)."""
    here = np.flatnonzero((records["inst"] == instance) & (records["end"] > 0))
    order = here[np.argsort(records["start"][here], kind="stable")]
    return [Call(int(trace.prompt[i]), max(1, int(trace.out[i]))) for i in order]


class Batch:
    """An instance's running batch over its own cache: `slots` rows, each a request or free."""

    def __init__(self, slots: int, longest: int, shape: Shape, seed: int = 0):
        B = shape.block_tokens
        self.shape, self.slots = shape, slots
        width = -(-longest // B) + 1
        n_blocks = slots * width
        self.cache = KV.Cache.empty(n_blocks, shape.kv_heads, B, shape.head_dim)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((slots, width), -1, **i32)
        self.ring = torch.arange(n_blocks, **i32)
        self.state = torch.tensor([0, n_blocks], dtype=torch.int64, device="cuda")
        self.held = np.zeros(slots, np.int32)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.flush = torch.empty(1 << 30, dtype=torch.uint8, device="cuda")
        self.qkv = None
        self.out = None
        self.step = None
        self.q = self.k = None
        self.token = self.logprob = None
        if shape.theta:
            self.rope = KV.Rope(KV.Rope.frequencies(shape.head_dim, shape.theta))
        if shape.vocab:
            V = shape.vocab
            self.prompt = np.zeros(slots, np.int32)
            self.logits = (3 * torch.randn((slots, V), generator=self.gen, device="cuda")).to(shape.dtype)
            self.noise = torch.empty((slots, V), device="cuda").exponential_(generator=self.gen)
            self.history = torch.randint(0, V, (slots, longest + 1), generator=self.gen, **i32)
            self.lengths = torch.zeros((2, slots), **i32)  # held and the prompt's
            full = lambda x: torch.full((slots,), x, device="cuda")
            self.rules = L.Rules(history=self.history, length=self.lengths[0], prompt_len=self.lengths[1], repetition=full(1.1),
                                 presence=full(0.1), frequency=full(0.05))

    def run(self, add: np.ndarray, read: Optional[np.ndarray] = None):
        """One step: row r gets add[r] tokens (0: none, -1: it has ended), of which the first read[r] are of its prompt, the others were
        written.  Without read: more than one token, and a request's first ones, are its prompt's.  Returns the start
        and end events."""
        s = self.shape
        tok = np.maximum(add, 0)
        n = int(tok.sum())
        if self.qkv is None or self.qkv.shape[0] < n:  # the projections' output, q, k and v side by side
            self.qkv = torch.randn((n, s.heads + 2 * s.kv_heads, s.head_dim), generator=self.gen, device="cuda").to(s.dtype)
        both = torch.from_numpy(np.stack([self.held, add]).astype(np.int32)).cuda()
        x = self.qkv[:n]
        if s.vocab:
            if read is None:
                read = np.where((tok > 1) | (self.held == 0), tok, 0)
            self.prompt = np.where((add < 0) | (self.held == 0), 0, self.prompt) + np.minimum(read, tok)
            self.lengths.copy_(torch.from_numpy(np.stack([self.held + tok, self.prompt]).astype(np.int32)))
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        self.flush.zero_()
        begin.record()
        self.step = KV.map_step(both[0], both[1], self.table, self.ring, self.state, n, s.block_tokens)
        if n:
            self.q, self.k = x[:, :s.heads], x[:, s.heads:s.heads + s.kv_heads]
            if s.theta:
                self.q, self.k = self.rope.rotate(self.q, self.k, self.step.row_start, self.step.kv_len)
            self.cache.append(self.k, x[:, s.heads + s.kv_heads:], self.step.runs)
            self.out = self.cache.attend(self.q, self.table, self.step.row_start, self.step.kv_len,
                                         max_q=int(tok.max()))
            if s.vocab:
                self.token, self.logprob = L.sample(self.logits, self.noise, temperature=0.8, top_p=0.95, rules=self.rules)
        end.record()
        if n and s.vocab:  # what each row will have said when its next token is drawn, and other random numbers for that
            self.history.scatter_(1, self.lengths[:1].t().long().clamp(max=self.history.shape[1] - 1), self.token[:, None].clamp(min=0))
            self.noise.exponential_(generator=self.gen)
        self.state = self.step.ring_state
        self.held = np.where(add < 0, 0, self.held + tok).astype(np.int32)
        return begin, end


@dataclass
class _Step:
    tokens: int
    context: int
    decode: bool
    events: tuple = field(repr=False)


def replay(trace, records: dict, cluster, instance: int, shape: Optional[Shape] = None, chunk: int = 512,
           max_steps: int = 1000, warmup: int = 3) -> dict:
    """Run `instance`'s calls (see calls_of) through up to max_steps steps and fit their time.

    records  the columns of Sim.records for one simulation of `trace`
    chunk    prompt tokens of a request in one step at most

    The result: steps, tokens and calls taken, and least-squares fits in microseconds for one
    layer: us_per_step + us_per_1000_tokens * context / 1000 over the steps in which every request
    decodes, prompt_us_per_token over the others; beside them the cluster's constant rates.
    """
    shape = shape or Shape()
    if chunk < 1 or max_steps < 1:
        raise H.HxError(H.HX_ERR_INVALID, "replay: chunk and max_steps must be at least 1")
    if not 0 <= instance < len(cluster.inst_type):
        raise H.HxError(H.HX_ERR_INVALID, "replay: no such instance")
    kind = int(cluster.inst_type[instance])
    slots = int(cluster.slots[kind])
    waiting = calls_of(trace, records, instance)
    if not waiting:
        raise H.HxError(H.HX_ERR_INVALID, "replay: the simulation started nothing on this instance")
    n_calls = len(waiting)
    batch = Batch(slots, max(c.prompt + c.out for c in waiting), shape)
    rows: List[Optional[Call]] = [None] * slots
    steps: List[_Step] = []
    waiting.reverse()
    while len(steps) < max_steps + warmup:
        add, read = np.zeros(slots, np.int32), np.zeros(slots, np.int32)
        for r in range(slots):
            if rows[r] is None and waiting:
                rows[r] = waiting.pop()
            c = rows[r]
            if c is None:
                continue
            if c.read < c.prompt:
                add[r] = read[r] = min(chunk, c.prompt - c.read)
                c.read += int(add[r])
            elif c.written < c.out:
                add[r] = 1
                c.written += 1
            else:
                add[r] = -1
                rows[r] = None
        if not add.any():
            break
        context = int(np.maximum(batch.held, 0).sum() + np.maximum(add, 0).sum())
        # which tokens are prompts' is of matter to those that are drawn
        events = batch.run(add, read) if shape.vocab else batch.run(add)
        steps.append(_Step(int(np.maximum(add, 0).sum()), context, bool((add <= 1).all()) and bool((add == 1).any()), events))
    torch.cuda.synchronize()
    steps = steps[warmup if len(steps) > 2 * warmup else 0:][-max_steps:]
    us = np.array([1000 * s.events[0].elapsed_time(s.events[1]) for s in steps])
    out = {"instance": instance, "slots": slots, "calls": n_calls, "steps": len(steps), "tokens": sum(s.tokens for s in steps),
           "prefill_tok_s": int(cluster.prefill_tok_s[kind]), "decode_us_tok": int(cluster.decode_us_tok[kind])}
    dec = np.array([s.decode for s in steps], bool)
    if dec.sum() >= 2:
        x = np.array([s.context for s in steps], float)[dec] / 1000
        slope, base = np.polyfit(x, us[dec], 1) if np.ptp(x) > 0 else (0.0, float(us[dec].mean()))
        out.update(decode_steps=int(dec.sum()), us_per_step=round(float(base), 3), us_per_1000_tokens=round(float(slope), 4),
                   mean_decode_us=round(float(us[dec].mean()), 3), mean_context=round(float(1000 * x.mean()), 1))
    other = ~dec & np.array([s.tokens > 0 for s in steps], bool)
    if other.any():
        tokens = sum(s.tokens for s, o in zip(steps, other) if o)
        out.update(prompt_steps=int(other.sum()), prompt_us_per_token=round(float(us[other].sum()) / tokens, 4))
    return out
