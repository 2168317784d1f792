"""A row's gradient by its log probability is one number: with the policy a few steps of fp32 away from
its reference, a last bit more or less of the row's sums would be a tenth of it."""
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


@pytest.mark.parametrize("V", [100, 1500, 3000, 20000, 40000, 70001])
def test_near_the_reference(Bd, V):
    """g = ref_logp - logp is exact (both are within a factor of two); e^g - 1 by its series, at most 16 U off
    relative, and its product with kl_coef (tests/test_gpu_policy_kl_gradient.py)."""
    rows = 48
    gen = torch.Generator().manual_seed(V)
    x = torch.randn(rows, V, generator=gen)
    tok = torch.randint(0, V, (rows,), generator=gen, dtype=torch.int32)
    adv = torch.zeros(rows, device="cuda")
    logp = Bd.policy_loss(x.cuda(), tok.cuda(), adv).logp
    ref = logp + 1e-5 * torch.linspace(-1, 1, rows, device="cuda")
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv, None, ref, kl_coef=0.5)
    assert torch.equal(r.logp, logp)
    u = -0.5 * torch.expm1(ref.cpu().double() - logp.cpu().double())
    want, b = R.logprobs_grad(x, tok, u, None)
    p = R.logprobs(x, tok)["p"]
    one = torch.zeros_like(p).scatter_(1, tok.long()[:, None], 1.0)
    worst = R.worst(r.d_logits, want, b + 20 * R.U * (u.abs()[:, None] * (one - p).abs()))
    print(V, round(worst, 3), flush=True)
    assert worst <= 1
