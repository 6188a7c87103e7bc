"""Which of a request's tokens a replay says are its prompt: penalties are for those that were written."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import replay as R

PROMPTS, OUTS = [513, 0, 1, 512, 1025, 7, 0], [3, 4, 2, 1, 5, 1, 1]


def _calls():
    n = len(PROMPTS)
    trace = SimpleNamespace(prompt=np.array(PROMPTS), out=np.array(OUTS))
    records = {"inst": np.zeros(n, int), "start": np.arange(n), "end": np.arange(1, n + 1)}
    cluster = SimpleNamespace(inst_type=np.array([0]), slots=np.array([3]), prefill_tok_s=np.array([1000]), decode_us_tok=np.array([9]))
    return trace, records, cluster


@pytest.mark.parametrize("chunk", [1, 512, 600])
def test_a_step_s_tokens_are_told_apart(monkeypatch, chunk):
    """A prompt's last chunk of one token, chunks of one token, and calls without a prompt."""
    seen = []

    class Fake:
        def __init__(self, slots, longest, shape):
            self.held = np.zeros(slots, np.int32)

        def run(self, add, read=None):
            seen.append((add.copy(), read.copy()))
            self.held = np.where(add < 0, 0, self.held + np.maximum(add, 0))
            event = SimpleNamespace(elapsed_time=lambda other: 1.0)
            return event, event

    monkeypatch.setattr(R, "Batch", Fake)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    R.replay(*_calls(), instance=0, shape=R.Shape(vocab=300), chunk=chunk, max_steps=10000, warmup=0)
    totals, now = [], [[0, 0] for _ in range(3)]
    for add, read in seen:
        for r in range(3):
            assert 0 <= read[r] <= max(add[r], 0)
            if add[r] < 0:
                totals.append(tuple(now[r]))
                now[r] = [0, 0]
            elif add[r] > 0:
                assert not read[r] or not now[r][1]  # a prompt comes first
                now[r][0] += int(read[r])
                now[r][1] += int(add[r] - read[r])
    totals += [tuple(x) for x in now if sum(x)]
    assert sorted(totals) == sorted(zip(PROMPTS, OUTS))


@pytest.mark.gpu
def test_lengths_of_prompts_over_a_replay(monkeypatch):
    """What the rules of the sampled rows have at the end of each call, against the calls themselves."""
    B_.build()
    run, seen = R.Batch.run, []
    now = [[0, 0] for _ in range(3)]

    def watched(self, add, *read):
        events = run(self, add, *read)
        for r in range(3):
            if add[r] < 0:
                now[r] = [0, 0]
            elif add[r] > 0:
                now[r][0] += int(add[r])
        seen.append((self.lengths.cpu().numpy().copy(), [x[0] for x in now], add.copy()))
        return events

    monkeypatch.setattr(R.Batch, "run", watched)
    shape = R.Shape(2, 1, 64, 16, torch.float16, 0.0, 300)
    R.replay(*_calls(), instance=0, shape=shape, chunk=512, max_steps=10000, warmup=0)
    ends = []
    last = [None] * 3
    for lengths, held, add in seen:
        for r in range(3):
            if add[r] > 0:
                assert lengths[0][r] == held[r]
                last[r] = (int(lengths[1][r]), held[r] - int(lengths[1][r]))
            elif add[r] < 0:
                ends.append(last[r])
                last[r] = None
    ends += [x for x in last if x is not None]
    assert sorted(ends) == sorted(zip(PROMPTS, OUTS))
