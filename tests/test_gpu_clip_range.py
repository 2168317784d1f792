"""Clipping at the ends of fp32's range."""
import math

import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("types", [(F32, F32), (BF, BF), (BF, F32)], ids=str)
def test_finite_gradients_whose_norm_is_past_fp32(Bd, types):
    """The norm comes back as infinity, and nothing is scaled: what a caller who looks at the norm expects."""
    g = torch.full((1000,), 3e38, device="cuda").to(types[0])
    assert torch.isfinite(g).all()
    out = torch.zeros(1000, dtype=types[1], device="cuda")
    plan = Bd.GradClip([g], [out])
    assert float(plan.norm()) == math.inf and float(plan.clip(1.0)) == math.inf
    assert torch.equal(out, g.to(types[1]))
    one = torch.full((1,), 3e38, device="cuda")  # fp32 holds this one: scaled as any other
    n = float(one)
    assert float(Bd.GradClip([one]).clip(1e30)) == n and abs(float(one) - 1e30) <= 4 * R.U * 1e30
