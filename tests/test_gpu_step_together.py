"""The operators of a whole step together, as a serving loop uses them: tables, rotary positions, the cache,
attention, and each row's next token."""
import json

import numpy as np
import pytest
import torch

from paper_2505_05286_gb300 import __main__ as M
from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import kvcache as KV
from paper_2505_05286_gb300 import replay as R
from tests import kv_cases as P
from tests import step_cases as S


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [R.Shape(8, 2, 64, 16, torch.float16, 10000.0, 5003), R.Shape(6, 1, 128, 32, torch.bfloat16, 500000.0, 9000)])
def test_every_step_against_64_bits(shape):
    """Requests of all kinds side by side.  q and k are turned by the positions that the step's tables say, the cache holds the
    turned keys, each output is the attention over it, and each token and its share follow from the request's own
    history."""
    B_.build()
    rng = np.random.default_rng(5)
    b = R.Batch(5, 300, shape)
    freq = KV.Rope.frequencies(shape.head_dim, shape.theta)
    left = rng.integers(1, 250, 5)
    for step in range(12):
        add = np.where(left > 0, np.minimum(left, rng.choice([0, 1, 1, 1, 40, 130], 5)), -(b.held > 0).astype(int)).astype(np.int32)
        left = left - np.maximum(add, 0)
        held, noise = b.held.copy(), b.noise.clone()
        history = b.history.clone()
        b.run(add)
        left[add < 0] = rng.integers(1, 250, int((add < 0).sum()))
        tok = np.maximum(add, 0)
        n = int(tok.sum())
        if not n:
            continue
        pos = torch.from_numpy(np.concatenate([h + np.arange(t) for h, t in zip(held, tok)])).long()
        x = b.qkv[:n]
        for got, src in ((b.q, x[:, :shape.heads]), (b.k, x[:, shape.heads:shape.heads + shape.kv_heads])):
            want, tol = S.rotate_plain(src, pos, freq, False, 1.0)
            assert bool(((got.double().cpu() - want).abs() <= tol).all())
        c = b.cache
        want, _, tol, _ = P.attend_plain(b.q, c.k, c.v, c.k_scale, c.v_scale, b.table, b.step.row_start.tolist(),
                                         b.step.kv_len.tolist(), shape.head_dim ** -0.5, True, 0)
        assert bool(((b.out.double() - want).abs() <= tol).all())
        # a key of the cache is the turned key of its token, to a rounding of 8 bits and of a block's scale
        slots = b.step.slots.cpu()
        for t in (0, n - 1):
            blk, place = int(slots[t]) // shape.block_tokens, int(slots[t]) % shape.block_tokens
            kept = c.k[blk, :, place].float() * c.k_scale[blk][:, None]
            # e4m3 of x / scale: half a step, 2^-4 of the value, or half of the smallest, 2^-10 of the scale
            assert bool(((kept - b.k[t].float()).abs() <= b.k[t].float().abs() * 2.0 ** -4 + c.k_scale[blk][:, None] * 2.0 ** -10).all())
        full = np.full(5, 1, np.float32)
        rules = dict(history=history.cpu().numpy(), length=b.lengths[0].cpu().numpy(), prompt_len=b.lengths[1].cpu().numpy(),
                     repetition=full * np.float32(1.1), presence=full * np.float32(0.1), frequency=full * np.float32(0.05))
        assert (rules["length"] == np.where(add < 0, held, held + tok)).all()
        z, _ = S.adjust_plain(b.logits.float().cpu().numpy(), rules, np.float32)
        for r in range(5):
            token, lp, tol = S.sample_plain(z[r], noise[r].cpu().numpy(), float(np.float32(0.8)), 0, float(np.float32(0.95)), 0.0)
            assert int(b.token[r]) == token and abs(float(b.logprob[r]) - lp) <= tol
            assert int(b.history[r, min(int(rules["length"][r]), 300)]) == token


@pytest.mark.gpu
def test_replay_with_everything(capsys):
    B_.build()
    assert M.main(["--recipe", "1", "--traces", "1", "--queries", "30", "--replay", "6", "--steps", "60", "--rope", "10000",
                   "--vocab", "32000"]) == 0
    out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert out["steps"] > 30 and out["rope"] == 10000 and out["vocab"] == 32000
    # (the fit's constant part alone may have either sign over so few contexts)
    assert out["mean_decode_us"] > 0 and out["prompt_us_per_token"] > 0


def test_the_command_hands_its_options_on(monkeypatch, capsys):
    seen = []

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
            return 0, 0, 0, np.zeros(1, np.int32)

        def records(self, i):
            return {}

    monkeypatch.setattr(M.H, "Sim", Sim)
    monkeypatch.setattr(R, "replay", lambda *a, **kw: seen.append(kw) or {})
    M.main(["--recipe", "0", "--queries", "20", "--replay", "0"])
    M.main(["--recipe", "0", "--queries", "20", "--replay", "0", "--rope", "10000", "--vocab", "1000"])
    assert "shape" not in seen[0] and (seen[1]["shape"].theta, seen[1]["shape"].vocab) == (10000.0, 1000)
