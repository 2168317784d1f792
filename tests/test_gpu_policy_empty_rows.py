"""The policy loss of rows of nothing but minus infinity."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF = torch.float32, torch.bfloat16
INF = math.inf


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("t", [F32, BF], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("V", [33, 1500, 40000, 140001])
def test_empty_rows(Bd, V, t):
    """Gradient 0 where the loss is finite.  Where it is not (a token past the vocabulary, an advantage that
    is NaN, a reference that gives the token a probability) the gradient is not finite either."""
    x = torch.randn(6, V).to(t)
    x[:5] = -INF
    tok = torch.tensor([3, V, 3, 3, -1, 3], dtype=torch.int32)
    adv = torch.tensor([1.0, 1.0, math.nan, 1.0, 1.0, 1.0])
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), entropy_coef=0.1)
    bad = [False, True, True, False, False, False]
    assert torch.isnan(r.row_loss).tolist() == bad
    assert torch.isnan(r.d_logits).all(-1).tolist() == bad == torch.isnan(r.d_logits).any(-1).tolist()
    assert r.d_logits[[0, 3, 4]].eq(0).all() and r.d_logits[5].any() and float(r.row_loss[3]) == -1
    ref = torch.full((6,), -2.0)
    ref[3] = -INF
    k = Bd.policy_loss(x.cuda(), tok.cuda(), torch.ones(6).cuda(), None, ref.cuda(), kl_coef=0.1)
    assert float(k.kl[0]) == INF == float(k.row_loss[0]) and not torch.isfinite(k.d_logits[0]).any()
    assert k.d_logits[4].eq(0).all() and torch.isfinite(k.d_logits[5]).all()
