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


@pytest.mark.parametrize("types", [(F32, F32), (BF, BF), (BF, F32)], ids=str)
def test_scales_below_the_smallest_normal_number(Bd, types):
    """Large gradients clipped to a small norm: max / n is 1e-38 to 1e-70, the results are ordinary numbers.
    Two roundings of a product of normal numbers (the scale's and the product's) and the store's."""
    g = (1e38 * torch.randn(500, generator=torch.Generator().manual_seed(1)).clamp(-3, 3) / 8).to(types[0])
    n = math.sqrt(float((g.double() ** 2).sum()))
    assert n < 3.4e38
    for max_norm in (4.0, 1.0, 1e-3, 1e-8, 1e-20, 1e-32):
        out = torch.zeros(500, dtype=types[1], device="cuda")
        got = float(Bd.GradClip([g.cuda()], [out]).clip(max_norm))
        assert abs(got - n) <= 2 * R.U * n
        m = float(torch.tensor(max_norm, dtype=F32))
        ref = g.double() * (m / n)
        assert R.worst(out, ref, R.HALF[types[1]] * ref.abs() + 2.5 * R.U * ref.abs() + R.TINY[types[1]]) <= 1, max_norm
