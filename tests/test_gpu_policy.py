"""GPU parity of the policy loss and its gradient against 64-bit references (bounds:
tests/step_ref.py)."""
import math

import pytest

from tests import step_ref as S
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF, HF]
IDS = lambda v: str(v).replace("torch.", "")
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _inputs(rows, V, t, seed=0, scale=2.5, low=0.8, high=1.3):
    """Ratios 1e-3 or more off the clipping borders, where the gradient jumps."""
    g = torch.Generator().manual_seed(seed + 31 * rows + V)
    rnd = lambda *s: torch.randn(*s, generator=g)
    x = (rnd(rows, V) * scale).to(t)
    tok = torch.randint(0, V, (rows,), generator=g, dtype=torch.int32)
    lp = torch.log_softmax(x.double(), -1).gather(1, tok.long()[:, None])[:, 0]
    step = 0.3 * rnd(rows).double()
    for b in (math.log(low) if low else -99, math.log(high)):
        step = torch.where((step - b).abs() < 1e-3, step + 3e-3, step)
    tok[torch.rand(rows, generator=g) < 0.15] = -1
    w = 0.5 + torch.rand(rows, generator=g)
    w[torch.rand(rows, generator=g) < 0.1] = 0
    return x, tok, rnd(rows), (lp - step).float(), (lp + 0.4 * rnd(rows)).float(), w


def _check(Bd, x, tok, adv, old, ref, w, low=0.8, high=1.3, beta=0.05, c=0.02, where="", **kw):
    dev = lambda t: t if t is None or t.is_cuda else t.cuda()
    X = dev(x)
    keep = X.cpu().clone()
    args = dict(clip_low=1 - low, clip_high=high - 1, kl_coef=beta if ref is not None else 0.0, entropy_coef=c)
    r = Bd.policy_loss(X, dev(tok), dev(adv), dev(old), dev(ref), dev(w), **args, **kw)
    torch.cuda.synchronize()
    # the bounds as the call had them, in fp32
    lo, hi = float(torch.tensor(1.0 - args["clip_low"])), float(torch.tensor(1.0 + args["clip_high"]))
    want = S.policy(keep, tok, adv, old, ref, w, lo, hi, float(torch.tensor(args["kl_coef"])), float(torch.tensor(c)))
    names = ["loss", "row_loss", "logp", "ratio", "entropy"] + (["kl"] if ref is not None else []) + (["d_logits"] if r.d_logits is not None else [])
    got = {n: R.worst(getattr(r, n), want[n], want[n + "_b"]) for n in names}
    print(where, tuple(keep.shape), {k: round(v, 3) for k, v in got.items()}, flush=True)
    assert all(v <= 1.0 for v in got.values()), (where, got)
    off = ~want["on"]
    for n in names[1:]:
        assert not getattr(r, n).cpu()[off].any(), n  # exactly 0
    return r, want


SIZES = [(1, 1), (2, 2), (3, 5), (9, 63), (5, 64), (4, 65), (130, 100), (37, 130), (6, 511), (7, 1024), (3, 1025), (5, 2048), (4, 2051), (3, 4096), (3, 4100),
         (2, 8192), (2, 16385), (5, 30522), (3, 50257), (2, 65536), (2, 65543), (1, 131072), (2, 140001)]


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,V", SIZES)
def test_parity(Bd, rows, V, t):
    x, tok, adv, old, ref, w = _inputs(rows, V, t)
    _check(Bd, x, tok, adv, old, ref, w, where="all")
    _check(Bd, x, tok, adv, old, None, None, c=0.0, where="plain")
    _check(Bd, x, tok, adv, None, ref, w, beta=0.3, where="on policy")
    _check(Bd, x, tok, adv, old, ref, w, grad=False, where="loss alone")


def test_many_rows(Bd):
    """More rows than one pass of a grid; the sum of their losses."""
    x, tok, adv, old, ref, w = _inputs(70_001, 17, F32)
    _check(Bd, x, tok, adv, old, ref, w / 70_001)


def test_clipping_by_sign(Bd):
    """The lesser of the two by the advantage's sign: a clipped row has no gradient from its ratio."""
    rows = 8
    x, _, _, _, _, _ = _inputs(rows, 50, F32)
    tok = torch.arange(rows, dtype=torch.int32)
    lp = torch.log_softmax(x.double(), -1).gather(1, tok.long()[:, None])[:, 0]
    ratio = torch.tensor([0.5, 0.5, 1.0, 1.0, 2.0, 2.0, 1.1, 0.9], dtype=torch.float64)
    adv = torch.tensor([1.0, -1.0] * 4)
    old = (lp - ratio.log()).float()
    r, _ = _check(Bd, x, tok, adv, old, None, None, c=0.0)
    zero = ~r.d_logits.cpu().any(-1)
    assert zero.tolist() == [False, True, False, False, True, False, False, False]
    # not clipped at all
    r, _ = _check(Bd, x, tok, adv, old, None, None, low=0.0, high=INF, c=0.0)
    assert r.d_logits.cpu().any(-1).all()
    # nor is a row of advantage 0, whose loss and gradient are 0
    r, _ = _check(Bd, x, tok, torch.zeros(rows), old, None, None, c=0.0)
    assert not r.d_logits.any() and not r.row_loss.any()


@pytest.mark.parametrize("t", TYPES, ids=IDS)
def test_rows_that_do_not_count(Bd, t):
    """Rows without a token, or of weight 0, are 0 whatever their logits, advantage or log
    probabilities hold; a batch of nothing else has loss 0."""
    x, tok, adv, old, ref, w = _inputs(12, 3001, t)
    tok[:6], w[:6] = 5, 1.0
    tok[6:9], w[9:] = -1, 0
    tok[9:] = 7
    x[6], x[7], x[9], x[10] = NAN, INF, NAN, -INF
    adv[6:], old[8:11], ref[7:] = NAN, INF, -INF
    _check(Bd, x, tok, adv, old, ref, w)
    r = Bd.policy_loss(x[6:].contiguous().cuda(), tok[6:].cuda(), adv[6:].cuda(), old[6:].cuda(), ref[6:].cuda(), w[6:].cuda(), kl_coef=0.1, entropy_coef=0.1)
    assert float(r.loss) == 0 and not r.d_logits.any() and not r.logp.any() and not r.ratio.any()


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("V", [33, 1500, 40000])
def test_masked_logits(Bd, t, V):
    """Minus infinity, and the type's lowest value, have probability 0 and gradient 0; a token of
    them has ratio 0 (and no gradient without a reference)."""
    x, tok, adv, old, ref, _ = _inputs(6, V, t)
    tok = torch.tensor([1, 1, 2, 2, 2, 2], dtype=torch.int32)
    x[:, 3::2] = -INF
    x[1:, 0] = torch.finfo(t).min
    lp = torch.log_softmax(x.double(), -1).gather(1, tok.long()[:, None])[:, 0]
    old, ref = (lp - 0.1).float(), (lp + 0.2).float()
    r, _ = _check(Bd, x, tok, adv, old, ref, None)
    assert not r.d_logits[:, 3::2].any()
    x[4, 2], x[5, 2] = -INF, torch.finfo(t).min
    old[4:], adv[4], adv[5] = -3.0, 1.0, -1.0
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), old.cuda(), entropy_coef=0.01)
    assert float(r.ratio[4]) == 0 == float(r.ratio[5]) and float(r.logp[4]) == -INF
    assert torch.isfinite(r.d_logits).all() and torch.isfinite(r.row_loss).all()
    ref[4:] = -3.0
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), old.cuda(), ref.cuda(), kl_coef=0.0)
    assert float(r.kl[4]) == INF and torch.isfinite(r.d_logits).all()


def test_near_the_reference(Bd):
    """The KL estimate of a policy that has hardly moved: d^2 / 2, without cancellation (a bound of a few
    roundings of it and the log probability's own error times d)."""
    x, tok, adv, old, _, _ = _inputs(64, 300, F32, scale=0.5)
    tok = tok.clamp(min=0)
    r0 = Bd.token_logprobs(x.cuda(), tok.cuda())
    for gap in (1e-6, 1e-4, 1e-2, 0.4, 0.6, 3.0, -0.3, -9.0):
        ref = (r0.logp + gap)
        r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), old.cuda(), ref, kl_coef=0.1)
        d = (ref - r.logp).double()
        want = torch.expm1(d) - d if abs(gap) > 1e-3 else d * d / 2 * (1 + d / 3)
        rel = float(((r.kl.double() - want).abs() / want).max())
        assert rel <= 32 * R.U * (1 if abs(gap) < 0.5 else 4 + 4 * abs(gap)), (gap, rel)


def test_a_token_outside_the_vocabulary(Bd):
    x, tok, adv, old, ref, w = _inputs(5, 200, BF)
    tok[:], w[:] = 3, 1.0
    tok[2] = 200
    r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), old.cuda(), ref.cuda(), w.cuda(), kl_coef=0.1)
    assert torch.isnan(r.d_logits[2]).all() and torch.isnan(r.row_loss[2]) and torch.isnan(r.loss)
    on = torch.arange(5) != 2
    assert torch.isfinite(r.d_logits.cpu()[on]).all() and torch.isfinite(r.row_loss.cpu()[on]).all()


@pytest.mark.parametrize("off,ld", [(0, 24), (1, 0), (3, 5), (4, 7)])
@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("V", [100, 5000])
def test_strides_and_in_place(Bd, t, V, off, ld):
    rows = 9
    x, tok, adv, old, ref, w = _inputs(rows, V, t)

    def strided(fill):
        buf = torch.full((off + rows * (V + ld),), fill, dtype=t, device="cuda")
        v = buf[off:].view(rows, V + ld)[:, :V]
        v.copy_(x)
        return buf, v
    base, _ = _check(Bd, x, tok, adv, old, ref, w)
    r, _ = _check(Bd, strided(NAN)[1], tok, adv, old, ref, w, where=f"ld {ld} off {off}")
    buf, v = strided(7.0)
    i, _ = _check(Bd, v, tok, adv, old, ref, w, where="in place", out=v)
    assert i.d_logits is v and torch.equal(v, r.d_logits)
    v.fill_(7.0)
    assert (buf == 7).all()


def test_shapes_and_empty(Bd):
    x, tok, adv, old, ref, w = (t.cuda() for t in _inputs(12, 90, F32))
    a = Bd.policy_loss(x, tok, adv, old, ref, w, kl_coef=0.1)
    b = Bd.policy_loss(x.view(3, 4, 90), tok.view(3, 4), adv.view(3, 4), old.view(3, 4), ref.view(3, 4), w.view(3, 4), kl_coef=0.1)
    assert b.logp.shape == (3, 4) and b.loss.shape == () and all(torch.equal(s.reshape(-1), t.reshape(-1)) for s, t in zip(a, b))
    e = Bd.policy_loss(x[:0], tok[:0], adv[:0])
    assert float(e.loss) == 0 and e.d_logits.shape == (0, 90)


def test_equals_the_loss_in_two_calls(Bd):
    """On policy without a KL term the gradient is token_logprobs_backward's for -A w, whose u differs by
    two roundings at most."""
    x, tok, adv, _, _, w = (t.cuda() for t in _inputs(50, 700, F32))
    r = Bd.policy_loss(x, tok, adv, weights=w)
    d, _ = Bd.token_logprobs_backward(x, tok, -adv * w)
    assert bool(((r.d_logits - d).abs() <= 4 * R.U * d.abs() + 1e-37).all())


def test_repeats_are_equal(Bd):
    x, tok, adv, old, ref, w = (t.cuda() for t in _inputs(3000, 2000, BF))
    run = lambda: Bd.policy_loss(x, tok, adv, old, ref, w, kl_coef=0.1, entropy_coef=0.01)
    a = run()
    for _ in range(3):
        assert all(torch.equal(s, t) for s, t in zip(a, run()))


def test_not_a_number_stays_in_its_row(Bd):
    """NaN or plus infinity among a row's logits, or NaN in what the loss is formed from, makes that row's
    loss and gradient NaN and no other's."""
    for V in (90, 3000, 40000):
        x, _, adv, old, ref, _ = _inputs(8, V, F32)
        tok = torch.arange(8, dtype=torch.int32)
        x[0, 50], x[1, 20], adv[2], old[3], ref[4] = NAN, INF, NAN, NAN, NAN
        r = Bd.policy_loss(x.cuda(), tok.cuda(), adv.cuda(), old.cuda(), ref.cuda(), kl_coef=0.1, entropy_coef=0.01)
        bad = torch.arange(8) < 5
        assert torch.equal(torch.isnan(r.row_loss).cpu(), bad) and torch.isnan(r.loss)
        assert torch.equal(torch.isnan(r.d_logits).all(-1).cpu(), bad) and torch.isfinite(r.d_logits.cpu()[~bad]).all()
        assert torch.isfinite(r.logp.cpu()[2:]).all() and torch.isfinite(r.entropy.cpu()[2:]).all()


def test_past_32_bits(Bd):
    """Offsets past 2^31 elements: the last rows of 2.2e9 logits."""
    rows, V = 270_000, 8192
    assert rows * V > 2 ** 31
    x = torch.empty(rows, V, dtype=BF, device="cuda")
    x.normal_()
    tok = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
    adv, w = torch.ones(rows, device="cuda"), torch.full((rows,), 1.0 / rows, device="cuda")
    r = Bd.policy_loss(x, tok, adv, weights=w, entropy_coef=0.1)
    c = float(torch.tensor(0.1))
    want = S.policy(x[-3:].cpu(), tok[-3:].cpu(), adv[-3:].cpu(), None, None, w[-3:].cpu(), 0.8, 1.2, 0.0, c)
    for n in ("logp", "entropy", "row_loss", "d_logits"):
        assert R.worst(getattr(r, n)[-3:], want[n], want[n + "_b"]) <= 1, n
    assert abs(float(r.loss) - float(r.row_loss.double().sum())) <= R.U * abs(float(r.loss)) + 1e-12
