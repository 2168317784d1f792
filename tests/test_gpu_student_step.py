"""The student's step with every operator together: a pre-norm block of the rotary backbone with norms
of queries and keys under the SingleForward mask, dropout after its products, the tied head and the
clipped policy loss, with every gradient, against the same step in 64 bits by autograd under the
same masks; captured into a HIP graph with its seed in device memory and replayed; on other streams."""
import math

import pytest

import oracle as O
from tests import step_ref as S

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32
B, H, N, K, DH, V = 2, 2, 24, 3, 32, 307
D, ROWS = H * DH, N + N * K
P, SEED = 0.2, 1234567
POS = torch.cat([torch.arange(N), (torch.arange(N)[:, None] + 1 + torch.arange(K)).reshape(-1)]).int()


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _params(seed):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    mat = lambda o, i: (rnd(o, i) / math.sqrt(i)).to(BF)
    return dict(g1=1 + 0.1 * rnd(D), wqkv=mat(3 * D, D), gq=1 + 0.1 * rnd(DH), gk=1 + 0.1 * rnd(DH), wo=mat(D, D), g2=1 + 0.1 * rnd(D),
                w1=mat(2 * D, D), w2=mat(D, 2 * D), g3=1 + 0.1 * rnd(D), head=mat(V, D))


def _batch(seed, p):
    """Residual rows, and tokens with log probabilities of a policy near the model's own (random logits
    of unit variance: log p about -log V - 1/2)."""
    g = torch.Generator().manual_seed(100 + seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    tok = torch.randint(0, V, (B, ROWS), generator=g, dtype=torch.int32)
    tok[:, :N] = -1  # the loss is over the noise rows
    tok[1, N + 5] = -1
    near = torch.full((B, ROWS), -math.log(V) - 0.5)
    w = torch.full((B, ROWS), 1.0 / (B * N * K))
    return rnd(B, ROWS, D), tok, rnd(B, ROWS) + 0.3, near, near + 0.2 * rnd(B, ROWS), w


def _step(Bd, p, table, pos, x, tok, adv, old, ref, w, seed):
    """No clipping: at a border of it the 64-bit step and this one may differ by a whole row's gradient."""
    mm = lambda a, b: torch.mm(a.reshape(-1, a.shape[-1]), b).view(*a.shape[:-1], -1)
    wg = lambda d, a: torch.mm(d.reshape(-1, d.shape[-1]).float().t(), a.reshape(-1, a.shape[-1]).float())
    y1, s1 = Bd.layer_norm(x, p["g1"], rms=True, out_dtype=BF)
    qkv = mm(y1, p["wqkv"].t())
    q, k, v = Bd.qkv_heads(qkv, H, None, table, pos, p["gq"], p["gk"])
    o, lse = Bd.training_attention_lse(Bd.KF_MASK_SINGLE, q, k, v, N, K)
    r = o.transpose(1, 2).reshape(B, ROWS, D)
    x2, y2, s2 = Bd.dropout_norm(mm(r, p["wo"].t()), x, p["g2"], None, P, seed, 0, rms=True)
    u = mm(y2, p["w1"].t())
    a = u.float().clamp(min=0).to(BF)
    x3 = Bd.dropout(mm(a, p["w2"].t()), P, seed, 1, residual=x2)
    y3, s3 = Bd.layer_norm(x3, p["g3"], rms=True, out_dtype=BF)
    logits = mm(y3, p["head"].t())
    l = Bd.policy_loss(logits, tok, adv, old, ref, w, clip_low=1.0, clip_high=math.inf, kl_coef=0.1, entropy_coef=0.01)
    dhead = wg(l.d_logits, y3)
    dx3, dg3, _ = Bd.layer_norm_backward(mm(l.d_logits, p["head"]), x3, p["g3"], s3, rms=True)
    dz = Bd.dropout_backward(dx3, P, seed, 1, BF)
    dw2 = wg(dz, a)
    du = mm(dz, p["w2"]) * (u > 0)
    dw1 = wg(du, y2)
    dx2, dro, dg2, _ = Bd.dropout_norm_backward(mm(du, p["w1"]), x2, p["g2"], s2, P, seed, 0, rms=True, dres=dx3)
    dwo = wg(dro, r)
    do = mm(dro, p["wo"]).view(B, ROWS, H, DH).transpose(1, 2).contiguous()
    dq, dk, dv = Bd.training_attention_backward(Bd.KF_MASK_SINGLE, q, k, v, o, lse, do, N, K)
    dqkv, dgq, dgk = Bd.qkv_heads_backward(dq, dk, dv, qkv, table, pos, p["gq"], p["gk"])
    dwqkv = wg(dqkv, y1)
    dx, dg1, _ = Bd.layer_norm_backward(mm(dqkv, p["wqkv"]), x, p["g1"], s1, rms=True, dres=dx2)
    grads = dict(x=dx, g1=dg1, wqkv=dwqkv, gq=dgq, gk=dgk, wo=dwo, g2=dg2, w1=dw1, w2=dw2, g3=dg3, head=dhead)
    return l, grads


def _reference(p, table, x, tok, adv, old, ref, w, seed):
    q = {n: t.double().requires_grad_(True) for n, t in p.items()}
    x = x.double().requires_grad_(True)
    rms = lambda t, g: t / torch.sqrt((t ** 2).mean(-1, keepdim=True) + 1e-5) * g
    drop = lambda t, site: t * (S.kept(B * ROWS, D, P, seed, site).view(B, ROWS, D) * 65536 / (65536 - S.threshold(P)))
    M = torch.from_numpy(O.training_mask("single", N, K)).bool()
    c, s = S._angles(table, POS, B, ROWS, DH)
    qh, kh, vh = S._split(rms(x, q["g1"]) @ q["wqkv"].t(), H, H, DH)
    qh, kh = (S.turn(rms(t, g), c, s)[0] for t, g in ((qh, q["gq"]), (kh, q["gk"])))
    a = (qh @ kh.transpose(-1, -2) / math.sqrt(DH)).masked_fill(~M, -math.inf)
    o = (torch.softmax(a, -1) @ vh).transpose(1, 2).reshape(B, ROWS, D)
    x2 = x + drop(o @ q["wo"].t(), 0)
    x3 = x2 + drop(torch.relu(rms(x2, q["g2"]) @ q["w1"].t()) @ q["w2"].t(), 1)
    lp = torch.log_softmax(rms(x3, q["g3"]) @ q["head"].t(), -1)
    on = tok >= 0
    at = lp.gather(-1, tok.long().clamp(min=0)[..., None])[..., 0]
    ratio, d = torch.exp(at - old.double()), ref.double() - at
    row = -ratio * adv.double() + 0.1 * (torch.expm1(d) - d) + 0.01 * (lp.exp() * lp).sum(-1)
    loss = (row * on * w.double()).sum()
    return loss.detach(), dict(zip(["x"] + list(q), torch.autograd.grad(loss, [x] + list(q.values()))))


def _table(Bd):
    return Bd.rope_table(N + K, DH)


def test_step_against_64_bits(Bd):
    """Some 22 stored bf16 tensors lie between a gradient and the loss; each is off by half a step, 2^-8 of
    itself at most and 2^-8 / sqrt(3) of its norm, and attention's P and dS by twice more.  A row's
    ratio, exp of a difference of log probabilities of size 6 that ten of them enter, is off as
    they are.  Gradients agree to 40 such errors, were they all alike; the ReLU's sign flips where a
    product is within its own error of 0, for a share 2^-8 of the elements, whose gradients are whole:
    sqrt(2^-8) of the norm of what comes through it."""
    p, b = _params(1), _batch(1, None)
    table = _table(Bd)
    l, grads = _step(Bd, {n: t.cuda() for n, t in p.items()}, table, POS.cuda(), *(t.cuda() for t in b), SEED)
    torch.cuda.synchronize()
    loss, want = _reference(p, table.cpu(), *b, SEED)
    tol = 40 * 2.0 ** -8 / math.sqrt(3) + 2.0 ** -4
    print("loss", float(l.loss), float(loss))
    assert abs(float(l.loss - loss)) <= 40 * 2.0 ** -8 / math.sqrt(3) * max(1.0, abs(float(loss)))
    for n, g in want.items():
        rel = float((grads[n].double().cpu() - g).norm() / g.norm())
        print(n, rel, flush=True)
        assert rel <= tol, n


def test_gradient_against_a_difference(Bd):
    """The step's loss along its own gradient of the norms' gains, which fp32 holds: a central difference
    of step h is off by the loss' rounding over h and by h^2; the loss' error is the same on both
    sides to a few parts in a hundred of the change."""
    p = {n: t.cuda() for n, t in _params(4).items()}
    b = [t.cuda() for t in _batch(4, None)]
    args = (_table(Bd), POS.cuda(), *b, SEED)
    _, g = _step(Bd, p, *args)
    names = ["g1", "g2", "g3", "gq", "gk"]
    size = math.sqrt(sum(float((g[n].double() ** 2).sum()) for n in names))
    h = 0.1

    def at(t):
        q = dict(p)
        for n in names:
            q[n] = p[n] + t * g[n] / size
        return float(_step(Bd, q, *args)[0].row_loss.double().sum())
    diff = (at(h) - at(-h)) / (2 * h)
    print(diff, size)
    assert abs(diff - size) <= 0.1 * size


def test_captured_step_replays(Bd):
    """Captured with the seed in device memory: each replay, on new data and with eager work between,
    has its own mask and equals the eager step of that seed bit for bit."""
    p = {n: t.cuda() for n, t in _params(2).items()}
    b = [t.cuda() for t in _batch(2, None)]
    table, pos, seed = _table(Bd), POS.cuda(), torch.tensor([SEED], device="cuda")
    eager0 = _step(Bd, p, table, pos, *b, SEED)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _step(Bd, p, table, pos, *b, seed)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l, grads = _step(Bd, p, table, pos, *b, seed)
    for n, v in ((3, 5), (4, SEED + 1), (2, SEED)):
        for t, new in zip(b, _batch(n, None)):
            t.copy_(new)
        seed.fill_(v)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in l if t is not None] + [t.clone() for t in grads.values()]
        e = _step(Bd, p, table, pos, *(t.cuda() for t in _batch(n, None)), v)
        assert all(torch.equal(x, y) for x, y in zip(got, [t for t in e[0] if t is not None] + list(e[1].values()))), n
    assert all(torch.equal(x, y) for x, y in zip(got, [t for t in eager0[0] if t is not None] + list(eager0[1].values())))


def test_another_stream(Bd):
    """Calls given a stream of their own equal those on the current one; inputs may be dropped while they
    still run."""
    x, res = torch.randn(3000, 768, device="cuda").to(BF), torch.randn(3000, 768, device="cuda")
    gain, g64 = torch.rand(768, device="cuda"), torch.rand(64, device="cuda")
    logits, tok = torch.randn(600, 9001, device="cuda"), torch.zeros(600, dtype=torch.int32, device="cuda")
    adv = torch.randn(600, device="cuda")
    seed = torch.tensor([9], device="cuda")

    def run(stream=None):
        kw = dict(stream=stream)
        t = Bd.rope_table(1000, 64, **kw)
        q, k, v = Bd.qkv_heads(x.view(3, 1000, 768), 4, 4, t, None, g64, g64, **kw)
        r = [t, q, k, v, *Bd.qkv_heads_backward(q, k, v, x.view(3, 1000, 768), t, None, g64, g64, **kw)]
        r += [Bd.dropout(x, 0.2, seed, 1, residual=res, **kw), Bd.dropout_backward(res, 0.2, seed, 1, BF, **kw)]
        h, y, st = Bd.dropout_norm(x, res, gain, None, 0.2, seed, 2, **kw)
        r += [h, y, st, *Bd.dropout_norm_backward(y, h, gain, st, 0.2, seed, 2, **kw)]
        return r + list(Bd.policy_loss(logits, tok, adv, adv, adv, adv, kl_coef=0.1, **kw))
    want = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(s)
    s.synchronize()
    torch.cuda.synchronize()
    assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(want, got))


def test_two_calls_at_once(Bd):
    """Steps on two streams share nothing: each has its own workspaces."""
    p = {n: t.cuda() for n, t in _params(6).items()}
    table, pos = _table(Bd), POS.cuda()
    batches = [[t.cuda() for t in _batch(n, None)] for n in (7, 8)]
    want = [_step(Bd, p, table, pos, *b, 3 + i) for i, b in enumerate(batches)]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(4):
        for i, (s, b) in enumerate(zip(streams, batches)):
            with torch.cuda.stream(s):
                got[i] = _step(Bd, p, table, pos, *b, 3 + i)
    torch.cuda.synchronize()
    for (l0, g0), (l1, g1) in zip(want, got):
        assert torch.equal(l0.loss, l1.loss) and all(torch.equal(g0[n], g1[n]) for n in g0)
