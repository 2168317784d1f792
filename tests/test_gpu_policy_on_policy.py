"""The policy loss without old log probabilities: the ratio is 1, but what makes a row's log
probability NaN makes its loss and gradient NaN all the same."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("grad", [True, False], ids=["gradient", "loss"])
@pytest.mark.parametrize("t", [F32, BF, HF], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("V", [33, 90, 3000, 40000, 140001])
def test_what_is_not_a_number_stays_so(Bd, V, t, grad):
    """A token past the vocabulary, NaN or plus infinity among the logits; an advantage of 0 hides none of
    them, and the other rows are as they are without them."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn(8, V, generator=g).to(t)
    tok = torch.arange(8, dtype=torch.int32)
    adv = torch.tensor([1.0, -1.0, 0.0, 1.0, 0.5, -0.5, 0.0, 2.0])
    plain = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), grad=grad)
    tok[0], tok[1], tok[2] = V, 2 ** 31 - 1, V + 7
    x[3, 20], x[4, 25] = NAN, INF
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), grad=grad)
    bad = torch.arange(8) < 5
    assert torch.equal(torch.isnan(r.row_loss).cpu(), bad) and torch.isnan(r.loss)
    assert torch.equal(r.row_loss[5:], plain.row_loss[5:]) and bool((r.ratio[5:] == 1).all())
    if grad:
        assert torch.isnan(r.d_logits[:5]).all() and torch.equal(r.d_logits[5:], plain.d_logits[5:])
    one = Bd.policy_loss(x[:1].cuda(), tok[:1].cuda(), adv[:1].cuda(), grad=grad)
    assert torch.isnan(one.loss)


def test_a_token_of_no_probability(Bd):
    """Its log probability is minus infinity and its ratio 1, as everywhere on policy: loss and gradient are
    finite."""
    x = torch.randn(2, 200)
    x[0, 4] = -INF
    tok, adv = torch.tensor([4, 5], dtype=torch.int32), torch.tensor([0.5, 0.5])
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda())
    assert float(r.logp[0]) == -INF and float(r.ratio[0]) == 1 and float(r.row_loss[0]) == -0.5
    assert torch.isfinite(r.d_logits).all()
