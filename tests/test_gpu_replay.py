"""The replay of an instance's calls: the cache operators together, as a serving
loop uses them."""
import json

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import __main__ as M
from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import replay as R
from paper_2505_05286_gb300 import workloads as W
from tests import kv_cases as P


def _records(inst, start):
    n = len(inst)
    return dict(inst=np.array(inst, np.int32), start=np.array(start, np.int64), end=np.array(start, np.int64) + 1)


class _Trace:
    def __init__(self, prompt, out):
        self.prompt, self.out = np.array(prompt, np.int32), np.array(out, np.int32)


def test_calls_in_the_order_of_their_start():
    calls = R.calls_of(_Trace([5, 6, 7, 8], [1, 0, 3, 4]), _records([2, 2, 1, 2], [30, 10, 5, 10]), 2)
    assert [(c.prompt, c.out) for c in calls] == [(6, 1), (8, 4), (5, 1)]


def test_replay_refusals():
    cl = W.make_workload(0, n_queries=20).cluster
    tr, rec = _Trace([5], [1]), _records([0], [0])
    for kw in (dict(instance=99), dict(instance=-1), dict(instance=1), dict(instance=0, chunk=0), dict(instance=0, max_steps=0)):
        with pytest.raises(H.HxError) as e:
            R.replay(tr, rec, cl, **kw)
        assert e.value.code == H.HX_ERR_INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [R.Shape(8, 2, 64, 16, torch.float16), R.Shape(6, 1, 128, 32, torch.bfloat16)])
def test_every_step_attends_to_what_its_requests_hold(shape):
    """Requests of all kinds side by side: each step's output against the 64-bit attention
    over the cache as it then is, and every block in one hand."""
    B_.build()
    rng = np.random.default_rng(3)
    b = R.Batch(5, 300, shape)
    left = rng.integers(1, 250, 5)
    for step in range(14):
        add = np.where(left > 0, np.minimum(left, rng.choice([0, 1, 1, 1, 40, 130], 5)), -(b.held > 0).astype(int)).astype(np.int32)
        left = left - np.maximum(add, 0)
        done = add < 0
        b.run(add)
        left[done] = rng.integers(1, 250, int(done.sum()))
        assert b.step.counts.tolist()[2] == 0
        n = int(np.maximum(add, 0).sum())
        if n:
            q = b.qkv[:n, :shape.heads]
            c = b.cache
            want, _, tol, _ = P.attend_plain(q, c.k, c.v, c.k_scale, c.v_scale, b.table, b.step.row_start.tolist(),
                                             b.step.kv_len.tolist(), shape.head_dim ** -0.5, True, 0)
            assert bool(((b.out.double() - want).abs() <= tol).all())
        head, free = b.state.tolist()
        used = sum(-(-int(h) // shape.block_tokens) for h in b.held)
        assert used + free == c.k.shape[0]
        assert (np.maximum(b.step.kv_len.cpu().numpy(), 0) == b.held).all()


@pytest.mark.gpu
def test_replay_of_a_simulated_schedule(capsys):
    B_.build()
    assert M.main(["--recipe", "1", "--traces", "1", "--queries", "30", "--replay", "6", "--steps", "120"]) == 0
    out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert out["instance"] == 6 and out["slots"] == 16 and out["steps"] > 50 and out["decode_steps"] >= 2
    assert out["tokens"] > 0 and out["us_per_step"] + out["us_per_1000_tokens"] * out["mean_context"] / 1000 > 0
    assert out["prompt_us_per_token"] > 0


@pytest.mark.parametrize("objective,slo", [(None, 0), ("p95", 0), ("p95_slo95", 1)])
def test_replay_takes_the_objective_that_it_is_given(monkeypatch, capsys, objective, slo):
    """The schedule replayed is the best point's by --objective, as without --replay."""
    asked = []

    class Sim:
        def __init__(self, *a, **kw):
            pass

        def __enter__(self):
            return self

        def __exit__(self, *exc):
            pass

        def run(self):
            pass

        def best(self, objective):
            asked.append(objective)
            return 0, 0, 0, np.zeros(1, np.int32)

        def records(self, i):
            return {}

    monkeypatch.setattr(H, "Sim", Sim)
    monkeypatch.setattr(R, "replay", lambda *a, **kw: {})
    wl = W.make_workload(0, n_traces=1, n_queries=20)
    want = wl.objective if objective is None else (W.OBJ_P95_SLO95 if slo else W.OBJ_P95)
    M.main(["--recipe", "0", "--queries", "20", "--replay", "0"] + (["--objective", objective] if objective else []))
    assert asked == [want]


def test_replay_keeps_no_more_steps_than_asked_for(monkeypatch):
    """Steps to warm up with are on top of max_steps and are not counted, however few those are."""
    class Event:
        def elapsed_time(self, other):
            return 0.001

    class Batch:
        def __init__(self, slots, longest, shape):
            self.held = np.zeros(slots, np.int32)

        def run(self, add):
            self.held = np.where(add < 0, 0, self.held + np.maximum(add, 0)).astype(np.int32)
            return Event(), Event()

    monkeypatch.setattr(R, "Batch", Batch)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    cl = W.make_workload(0, n_queries=20).cluster
    for steps in (1, 2, 3, 4, 50):
        out = R.replay(_Trace([5], [100]), _records([0], [0]), cl, 0, max_steps=steps)
        assert out["steps"] == steps
    assert R.replay(_Trace([5], [1]), _records([0], [0]), cl, 0, max_steps=50)["steps"] == 3
