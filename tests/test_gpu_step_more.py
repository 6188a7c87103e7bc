"""Rotary positions and adjusted logits on the GPU: what is refused, and calls beside the usual ones."""
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import kvcache as KV
from paper_2505_05286_gb300 import logits as L
from tests import step_cases as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    B_.build()


def test_a_mask_without_words_is_refused():
    """It allows no token of any vocabulary; it is not the same as no mask.  Without masks at all every row's is out of range."""
    i32 = dict(dtype=torch.int32, device="cuda")
    for kw in ({}, dict(mask_row=torch.zeros(2, **i32))):
        with pytest.raises(H.HxError) as err:
            L.Rules(mask=torch.zeros((2, 0), **i32), **kw)
        assert err.value.code == H.HX_ERR_INVALID and "mask" in str(err.value)
    x = torch.randn((2, 50), device="cuda")
    rules = L.Rules(mask=torch.zeros((0, 2), **i32), mask_row=torch.zeros(2, **i32))
    assert torch.equal(L.adjust(x, rules), x)


def _near(got, want, tol):
    got = got.double().cpu()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())


@pytest.mark.parametrize("scale", [1.25, -0.5, 1.0])
@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient_at_every_scale(scale, interleaved):
    """Against the formula and against differences of sum(w * rotate(x)); twice around is scale * scale times what was turned."""
    g = torch.Generator(device="cuda").manual_seed(3)
    f = KV.Rope.frequencies(8)
    rope = KV.Rope(f, interleaved=interleaved, scale=scale)
    pos = torch.tensor([3, 77, 100000], dtype=torch.int32, device="cuda")
    x, w = (torch.randn((3, 2, 10), generator=g, device="cuda") for _ in range(2))
    x = (x * 1024).round() / 1024  # and half more or less are numbers of 32 bits
    grad = rope.rotate(w, positions=pos, inverse=True)
    _near(grad, *P.rotate_plain(w, pos, f, interleaved, scale, True))
    grad, w64, base = grad.double().cpu(), w.double().cpu(), x.double().cpu()
    value = lambda z: float((P.rotate_plain(z.float(), pos, f, interleaved, scale)[0] * w64).sum())
    for at in [(t, h, d) for t in range(3) for h in range(2) for d in range(10)]:
        a, b = base.clone(), base.clone()
        a[at] += 0.5
        b[at] -= 0.5
        # linear, so exact but for 64 bits; the gradient itself is within 6 roundings of two terms, and its own
        assert abs(value(a) - value(b) - float(grad[at])) <= 16 * P.U * max(1.0, abs(scale)) * float(w.abs().max())
    around = rope.rotate(rope.rotate(x, positions=pos), positions=pos, inverse=True)
    want = base.clone()
    want[..., :8] *= scale * scale
    # of the largest |x|: the first pass 6 roundings of two terms and its own, 13.5 in all, which the second one turns (times 1.5 at
    # most); its own 6 roundings are of two terms with a sum of 2 at most, and its result's is of 1.5
    _near(around, want, torch.full_like(want, 40 * P.U * max(1.0, scale * scale) * float(x.abs().max())))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_the_widest_heads(dtype, interleaved):
    """1024 values, all turned: as many loads to a head as there can be."""
    g = torch.Generator(device="cuda").manual_seed(4)
    f = KV.Rope.frequencies(1024)
    q, k = (torch.randn((21, h, 1024), generator=g, device="cuda").to(dtype) for h in (5, 2))
    pos = torch.randint(0, 1 << 20, (21,), generator=g, device="cuda", dtype=torch.int32)
    for x, y in zip((q, k), KV.Rope(f, interleaved=interleaved, scale=0.75).rotate(q, k, positions=pos)):
        _near(y, *P.rotate_plain(x, pos, f, interleaved, 0.75))
