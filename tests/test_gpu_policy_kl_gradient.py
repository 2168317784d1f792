"""The KL term's gradient, e^g - 1 with g = ref_logp - logp, at every distance of the reference: far
below the policy it is -1, as it is at minus infinity."""
import math

import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
BETA = 0.125  # a power of two: the product with it is exact
GAPS = (-3.4e38, -1e30, -1e9, -3e7, -2.0 ** 24 - 64, -2.0 ** 23, -1e5, -1000.0, -60.0, -9.0, -3.0, -0.6, -0.4, -1e-2, -1e-5, 1e-5, 1e-2, 0.4, 0.6, 3.0, 9.0, -math.inf)


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _u(ref, logp):
    """u = -BETA (e^g - 1) of advantage 0, and how far a kernel may be from it, with U of tests/train_ref.py.
    g is rounded once.  For |g| < 1/2 the series for e^g - g - 1 (at most 0.3 |g|) is off by 32 U of itself
    and its sum with g by U: (32 * 0.3 + 1) / 0.78 + 1 < 16 U, as |e^g - 1| >= 0.78 |g|.  Beyond, g's
    rounding, the product with log2 e and that constant put 3 U |g| on the exponent, and exp2 is off by 2 U:
    e^g (3 |g| + 2) U, which below -1/2 is at most (3 / e + 2 * 0.61) / 0.39 < 6 U of |e^g - 1| (>= 0.39),
    above 1/2 2.6 (3 |g| + 2) U of it; then the difference's rounding and the last product's."""
    g = ref.double() - logp.double()
    e = torch.expm1(g)
    rel = 20 + torch.where(g > 0, 8 * g.clamp(0, 100), 0.0)
    return -BETA * e, BETA * e.abs() * rel * R.U


def _check(Bd, x, tok, ref, **kw):
    adv = torch.zeros(len(tok), device="cuda")
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv, None, ref, kl_coef=BETA, **kw)
    u, u_b = _u(ref.cpu(), r.logp.cpu())
    want, b = R.logprobs_grad(x, tok, u, None)
    p = R.logprobs(x, tok)["p"]
    one = torch.zeros_like(p).scatter_(1, tok.long()[:, None], 1.0)
    return R.worst(r.d_logits, want, b + u_b[:, None] * (one - p).abs())


@pytest.mark.parametrize("V", [12, 300, 3000, 40000])
@pytest.mark.parametrize("t", [F32, BF, HF], ids=lambda v: str(v).replace("torch.", ""))
def test_gradient_at_every_distance(Bd, t, V):
    rows = len(GAPS)
    g = torch.Generator().manual_seed(V)
    x = torch.randn(rows, V, generator=g).to(t)
    tok = torch.randint(0, V, (rows,), generator=g, dtype=torch.int32)
    ref = Bd.token_logprobs(x.cuda(), tok.cuda()).logp + torch.tensor(GAPS, device="cuda")
    got = _check(Bd, x, tok, ref)
    print(V, t, round(got, 3), flush=True)
    assert got <= 1


@pytest.mark.parametrize("t", [F32, BF], ids=lambda v: str(v).replace("torch.", ""))
def test_reference_masked_by_a_finite_value(Bd, t):
    """A reference that rules the sampled token out by -1e9 or the type's lowest value pulls the policy away
    from it with all of kl_coef."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(4, 500, generator=g).to(t)
    tok = torch.tensor([3, 4, 5, 6], dtype=torch.int32)
    masked = x.clone()
    masked[0, 3], masked[1, 4], masked[2, 5] = -1e9, torch.finfo(t).min, -3e7
    ref = Bd.token_logprobs(masked.cuda(), tok.cuda()).logp
    assert _check(Bd, x, tok, ref) <= 1
