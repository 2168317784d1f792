"""Ratios past fp32: they count as its largest number, clipped or not."""
import math

import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
MOST = (2 - 2.0 ** -23) * 2.0 ** 127


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("low,high", [(0.0, math.inf), (0.8, math.inf), (0.8, 1.25)])
@pytest.mark.parametrize("V", [50, 3000, 40000])
def test_ratio_past_fp32(Bd, V, low, high):
    """old_logp 200 below logp: ratio e^200, which fp32 does not hold.  Advantages are powers of two, so
    the largest number times each is exact, and weights of 2^-100 keep loss and gradient in range."""
    g = torch.Generator().manual_seed(V)
    adv = torch.tensor([-0.5, 0.0, 0.5, -1.0, 1.0, -2.0 ** -20, -0.0])
    x = torch.randn(len(adv), V, generator=g)
    tok = torch.arange(len(adv), dtype=torch.int32)
    old = Bd.token_logprobs(x.cuda(), tok.cuda()).logp - 200
    w = torch.full((len(adv),), 2.0 ** -100)
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), old, None, w.cuda(), clip_low=1 - low, clip_high=high - 1)
    assert bool((r.ratio == math.inf).all())
    A = adv.double()
    hi = min(float(torch.tensor(1.0 + (high - 1))), MOST)
    cut = hi * A < MOST * A
    u = torch.where(cut, 0.0, -MOST * A * 2.0 ** -100)
    loss = torch.where(cut, -hi * A, -MOST * A) * 2.0 ** -100
    assert cut.any() == (high < math.inf)
    assert torch.equal(r.row_loss.cpu().double(), loss)
    assert R.worst(r.d_logits, *R.logprobs_grad(x, tok, u, None)) <= 1
