"""GPU parity of token log probabilities, entropies, alternatives and the gradient of the logits
against 64-bit references (bounds: tests/train_ref.py)."""
import math

import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF, HF]
IDS = lambda v: str(v).replace("torch.", "")


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _inputs(rows, V, t, seed=0, scale=2.5):
    g = torch.Generator().manual_seed(seed + 31 * rows + V)
    x = torch.randn(rows, V, generator=g) * scale
    tok = torch.randint(0, V, (rows,), generator=g, dtype=torch.int32)
    u, c = torch.randn(rows, generator=g), 0.3 * torch.randn(rows, generator=g)
    return x.to(t), tok, u, c


def _score(Bd, x, tok, top, where=""):
    X = x if x.is_cuda else x.cuda()
    r = Bd.token_logprobs(X, tok.cuda(), top, lse=True)
    torch.cuda.synchronize()
    x = X.cpu()
    ref = R.logprobs(x, tok, top)
    got = {n: R.worst(getattr(r, n), ref[n], ref[n + "_b"]) for n in ("logp", "entropy", "lse")}
    if top:
        assert torch.equal(r.top_ids.cpu(), ref["top_ids"]), where
        got["top"] = R.worst(r.top_logp, ref["top_logp"], ref["top_b"])
    print(where, tuple(x.shape), {k: round(v, 3) for k, v in got.items()}, flush=True)
    assert all(v <= 1.0 for v in got.values()), (where, got)
    return r


def _grad(Bd, x, tok, u, c, where="", **kw):
    X = x if x.is_cuda else x.cuda()
    dev = lambda t: None if t is None else t.cuda()
    keep = X.cpu().clone()
    d, r = Bd.token_logprobs_backward(X, tok.cuda(), dev(u), dev(c), entropy=True, lse=True, **kw)
    torch.cuda.synchronize()
    ref, b = R.logprobs_grad(keep, tok, u, c)
    fw = R.logprobs(keep, tok)
    got = dict(d=R.worst(d, ref, b), logp=R.worst(r.logp, fw["logp"], fw["logp_b"]),
               entropy=R.worst(r.entropy, fw["entropy"], fw["entropy_b"]), lse=R.worst(r.lse, fw["lse"], fw["lse_b"]))
    print(where, tuple(keep.shape), {k: round(v, 3) for k, v in got.items()}, flush=True)
    assert all(v <= 1.0 for v in got.values()), (where, got)
    return d


SIZES = [(1, 1), (2, 2), (3, 5), (9, 63), (5, 64), (4, 65), (130, 100), (6, 511), (7, 1024), (3, 1025), (5, 2048), (4, 2051),
         (3, 4096), (3, 4100), (2, 8192), (2, 16385), (3, 30522), (2, 50257), (1, 65536), (1, 65543), (1, 131072), (1, 140001)]


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,V", SIZES)
def test_score(Bd, rows, V, t):
    x, tok, _, _ = _inputs(rows, V, t)
    for top in sorted({0, 1, min(5, V), min(20, V), min(64, V)}):
        _score(Bd, x, tok, top, f"top {top}")


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,V", SIZES)
def test_gradient(Bd, rows, V, t):
    x, tok, u, c = _inputs(rows, V, t)
    _grad(Bd, x, tok, u, None, "u")
    _grad(Bd, x, tok, u, c, "u, c")


def test_row_counts(Bd):
    for rows in (0, 1, 3, 4, 255, 256, 257, 1025, 9000):
        x, tok, u, c = _inputs(rows, 101, BF)
        if rows:
            _score(Bd, x, tok, 3)
            _grad(Bd, x, tok, u, c)
        else:
            r = Bd.token_logprobs(x.cuda(), tok.cuda(), 3)
            assert r.logp.shape == (0,) and r.top_ids.shape == (0, 3)
            assert Bd.token_logprobs_backward(x.cuda(), tok.cuda())[0].shape == (0, 101)


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("V", [70, 3000, 30522])
def test_masked_vocabulary(Bd, V, t):
    """Minus infinity and the type's lowest value as masks: rows with all, all but one and all but
    two logits masked, the given token among the masked ones, alternatives past the last unmasked."""
    x, tok, u, c = _inputs(12, V, t)
    low = torch.finfo(t).min
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, V // 2] = 1.5
    tok[1] = V // 2
    x[2] = -math.inf
    x[2, [3, V - 1]] = torch.tensor([0.5, 2.0]).to(t)
    tok[2] = 5  # masked
    x[3] = low
    x[4] = low
    x[4, 7] = 0.0
    x[5, : V - 9] = -math.inf
    tok[5] = V - 4
    x[6, ::2] = low
    x[7, 1::2] = -math.inf
    tok[7] = 4
    x[8] = -math.inf
    tok[8] = -1
    for top in (0, 4, 20, 64):
        _score(Bd, x, tok, top, f"masked top {top}")
    # a gradient of entropy where one logit of the type's lowest value meets another is 0 * huge
    rows = [i for i in range(12) if i not in (4, 6)] if t == F32 else list(range(12))
    _grad(Bd, x[rows].contiguous(), tok[rows], u[rows], None, "masked u")
    _grad(Bd, x[rows].contiguous(), tok[rows], u[rows], c[rows], "masked u, c")


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("V", [64, 900, 50257])
def test_ties_go_to_the_lowest_id(Bd, V, t):
    """Equal logits everywhere, few distinct values, a block of equal maxima, both zeros."""
    g = torch.Generator().manual_seed(V)
    x = torch.zeros(8, V)
    x[1] = torch.randint(0, 3, (V,), generator=g).float()
    x[2] = -1.0
    x[2, V // 3: V // 3 + 40] = 4.0
    x[3] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)
    x[4] = torch.arange(V).float() / V
    x[5] = -torch.arange(V).float() / V
    x[6] = torch.randn(V, generator=g).round()
    x[7, :] = 3.0
    x[7, V - 1] = 5.0
    for top in (1, 7, 32, 64):
        _score(Bd, x.to(t), torch.zeros(8, dtype=torch.int32), top, f"ties top {top}")


def test_few_unmasked_ids(Bd):
    """Fewer finite logits than alternatives, at the start, the end and within, one lane's or all lanes';
    the rest are the lowest masked ids."""
    for t in TYPES:
        for V in (65, 300, 5000, 50257):
            x = torch.full((8, V), -math.inf)
            x[0, 0] = 1.0
            x[1, V - 1] = 1.0
            x[2, [1, 3, V // 2]] = torch.tensor([0.5, 0.5, 2.0])
            x[3, ::max(1, V // 5)] = -1.0
            x[4, 2:40] = torch.arange(38).float()
            x[5, torch.arange(0, V, 64)[:60]] = 3.0
            x[7, : min(V, 64)] = 0.25
            tok = torch.zeros(8, dtype=torch.int32)
            for top in (1, 5, 20, 64):
                _score(Bd, x.to(t), tok, top, f"few V {V} top {top}")


def test_sorted_clusters(Bd):
    """The largest logits next to each other, and a stride apart: they fall to few lanes, or one."""
    for V in (5000, 50257):
        for t in (F32, BF):
            for step in (1, 64, 256, 512, 1024, 2048):
                x, tok, _, _ = _inputs(2, V, t)
                at = torch.arange(0, min(V, 64 * step), step)
                x[0, at] = (20 + torch.arange(len(at)).float() / 8).to(t)
                x[1, at] = (20 - torch.arange(len(at)).float() / 8).to(t)
                _score(Bd, x, tok, 64, f"step {step}")


def test_tokens_outside_the_vocabulary(Bd):
    """Negative: no token, logp 0, no gradient from u.  vocab and above: NaN.  No tokens at all."""
    x, tok, u, c = _inputs(6, 300, BF)
    tok[0], tok[1], tok[2], tok[3] = -1, -(2 ** 31), 300, 2 ** 31 - 1
    r = _score(Bd, x, tok, 2)
    assert r.logp[0] == 0 and r.logp[1] == 0 and torch.isnan(r.logp[2:4]).all()
    d = _grad(Bd, x, tok, u, None)
    assert not d[:2].any() and torch.isnan(d[2:4]).all()
    _grad(Bd, x, tok, u, c)
    r = Bd.token_logprobs(x.cuda(), None, 1)
    assert not r.logp.any() and torch.equal(r.top_ids[:, 0].cpu().long(), x.float().argmax(-1))


def test_values_that_are_not_finite(Bd):
    x, tok, u, c = _inputs(6, 1000, F32)
    x[1, 500], x[2, 0], x[4, 999] = float("nan"), math.inf, -float("nan")
    r = Bd.token_logprobs(x.cuda(), tok.cuda(), 3, lse=True)
    d, _ = Bd.token_logprobs_backward(x.cuda(), tok.cuda(), u.cuda(), c.cuda())
    for i in (1, 2, 4):
        assert torch.isnan(r.logp[i]) and torch.isnan(r.entropy[i]) and torch.isnan(r.lse[i])
        assert torch.isnan(r.top_logp[i]).all() and torch.isnan(d[i]).all()
    assert r.top_ids[1, 0] == 500 and r.top_ids[2, 0] == 0 and r.top_ids[4, 0] == 999
    good = [0, 3, 5]
    _score(Bd, x[good].contiguous(), tok[good], 3)
    ref, b = R.logprobs_grad(x[good], tok[good], u[good], c[good])
    assert R.worst(d[good], ref, b) <= 1


def test_extreme_logits(Bd):
    """Large offsets and spreads: the maximum is taken out first."""
    for t, off in ((F32, 1e4), (F32, -3e37), (HF, 6e4), (BF, 1e30), (BF, -1e30)):
        x, tok, u, _ = _inputs(4, 777, F32)
        x = (x + off).to(t) if abs(off) < 1e5 else (torch.full_like(x, off) * (1 + x / 64)).to(t)
        _score(Bd, x, tok, 4, f"{t} {off}")
        _grad(Bd, x, tok, u, None, f"{t} {off}")


@pytest.mark.parametrize("t", TYPES, ids=IDS)
@pytest.mark.parametrize("V,ld,off,ldd", [(1000, 1008, 0, 1008), (1000, 1003, 0, 1000), (4099, 4099, 1, 4100), (30522, 30523, 5, 30528),
                                          (100, 101, 3, 107), (50257, 50260, 2, 50257)])
def test_strides_and_alignment(Bd, V, ld, off, ldd, t):
    """Rows ld apart from an odd start; NaN between them is not read, and out's gaps stay as they were."""
    rows = 5
    x, tok, u, c = _inputs(rows, V, t)
    buf = torch.full((rows * ld + off,), float("nan"), dtype=t, device="cuda")
    X = buf[off:].view(rows, ld)[:, :V]
    X.copy_(x)
    _score(Bd, X, tok, 6)
    out = torch.full((rows * ldd + 3,), 7.0, dtype=t, device="cuda")
    o = out[3:].view(rows, ldd)[:, :V]
    _grad(Bd, X, tok, u, c, out=o)
    assert (out[:3] == 7).all() and (out[3:].view(rows, ldd)[:, V:] == 7).all()
    assert torch.isnan(buf[off:].view(rows, ld)[:, V:]).all()
    Y = X.clone(memory_format=torch.contiguous_format)
    a, _ = Bd.token_logprobs_backward(Y.clone(), tok.cuda(), u.cuda(), c.cuda())
    _grad(Bd, Y, tok, u, c, out=Y)  # in place
    assert torch.equal(a, Y)


def test_more_dimensions_and_null_gradients(Bd):
    x, tok, u, c = (t.cuda() for t in _inputs(24, 500, BF))
    r = Bd.token_logprobs(x.view(2, 3, 4, 500), tok.view(2, 3, 4), 3)
    q = Bd.token_logprobs(x, tok, 3)
    assert r.logp.shape == (2, 3, 4) and r.top_ids.shape == (2, 3, 4, 3)
    assert torch.equal(r.logp.view(-1), q.logp) and torch.equal(r.top_ids.view(24, 3), q.top_ids)
    d, _ = Bd.token_logprobs_backward(x, tok)
    assert not d.any()
    a, _ = Bd.token_logprobs_backward(x, None, u, c)
    b, _ = Bd.token_logprobs_backward(x, None, None, c)
    assert torch.equal(a, b)


def test_offsets_past_32_bits(Bd):
    """Logits of 4.6 GB: rows past 2^31 elements."""
    rows, V = 46_000, 50_000
    x = torch.empty(rows, V, dtype=BF, device="cuda").normal_()
    tok = torch.randint(0, V, (rows,), dtype=torch.int32, device="cuda")
    u = torch.rand(rows, device="cuda")
    r = Bd.token_logprobs(x, tok, 2)
    pick = [0, 1, 42_949, 42_950, rows - 1]
    xs, toks, us = x[pick].cpu(), tok[pick].cpu(), u[pick].cpu()
    ref = R.logprobs(xs, toks, 2)
    assert R.worst(r.logp[pick], ref["logp"], ref["logp_b"]) <= 1 and torch.equal(r.top_ids[pick].cpu(), ref["top_ids"])
    d, _ = Bd.token_logprobs_backward(x, tok, u, out=x)
    rd, b = R.logprobs_grad(xs, toks, us, None)
    assert R.worst(d[pick], rd, b) <= 1


def test_same_result_on_every_run(Bd):
    x, tok, u, c = (t.cuda() for t in _inputs(700, 5003, BF))
    a = Bd.token_logprobs(x, tok, 9, lse=True)
    d, _ = Bd.token_logprobs_backward(x, tok, u, c)
    for _ in range(3):
        b = Bd.token_logprobs(x, tok, 9, lse=True)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        assert torch.equal(d, Bd.token_logprobs_backward(x, tok, u, c)[0])


def test_difference_quotient(Bd):
    """The gradient against differences of the framework's own forward pass in fp32 (error e^2 of the
    third derivative, of terms of size 8; rounding U |logp| / e)."""
    x, tok, u, c = (t.cuda() for t in _inputs(30, 400, F32))
    d, r = Bd.token_logprobs_backward(x, tok, u, c, entropy=True)
    v = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    e = 2.0 ** -7

    def f(s):
        q = Bd.token_logprobs(x + s * e * v, tok)
        return float((q.logp.double() * u + q.entropy.double() * c).sum())
    got, want = (f(1) - f(-1)) / (2 * e), float((d.double() * v).sum())
    size = float((u.abs() * 8 + c.abs() * 8).sum())
    noise = float((u.abs() * r.logp.abs() + c.abs() * r.entropy).sum()) * 100 * R.U / e
    assert abs(got - want) <= 8 * size * e * e + noise
