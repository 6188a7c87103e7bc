"""Rotary positions and adjusted logits on the GPU: what is refused, and calls beside the usual ones."""
import pytest
import torch

from paper_2505_05286_gb300 import build as B_
from paper_2505_05286_gb300 import hxsim as H
from paper_2505_05286_gb300 import logits as L

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
