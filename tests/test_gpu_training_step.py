"""The training step's operators together, as a student's step uses them: one pre-norm attention
block over the SingleForward rows, the tied head, the loss over Stage-1 style targets, every
gradient, and clipping, against the same step in 64 bits by autograd; then captured into a HIP
graph and replayed."""
import math

import pytest

import oracle as O
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32
B, H, N, K, DH, V = 2, 2, 24, 3, 32, 307
D, ROWS = H * DH, N + N * K


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _params(seed):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    return dict(g1=1 + 0.1 * rnd(D), b1=0.1 * rnd(D), wqkv=(rnd(3 * D, D) / math.sqrt(D)).to(BF), wo=(rnd(D, D) / math.sqrt(D)).to(BF),
                g2=1 + 0.1 * rnd(D), b2=0.1 * rnd(D), head=(rnd(V, D) / math.sqrt(D)).to(BF))


def _batch(seed):
    g = torch.Generator().manual_seed(100 + seed)
    x = torch.randn(B, ROWS, D, generator=g)
    tok = torch.randint(0, V, (B, ROWS), generator=g, dtype=torch.int32)
    tok[:, :N] = -1  # the loss is over the noise rows
    tok[1, N + 5] = -1
    w = torch.full((B, ROWS), -1.0 / (B * N * K))
    return x, tok, w


def _heads(t):  # [B][rows][D] -> [B][H][rows][DH]
    return t.view(B, ROWS, H, DH).transpose(1, 2).contiguous()


def _rows(t):
    return t.transpose(1, 2).reshape(B, ROWS, D)


def _step(Bd, p, x, tok, w, out=None, plan=None, max_norm=0.05):
    """Losses and gradients; `out` and `plan`: the buffers of an earlier call (a captured step's)."""
    mm = lambda a, b: torch.mm(a.reshape(-1, a.shape[-1]), b).view(*a.shape[:-1], -1)
    y1, s1 = Bd.layer_norm(x, p["g1"], p["b1"], out_dtype=BF)
    q, k, v = (_heads(t) for t in mm(y1, p["wqkv"].t()).split(D, -1))
    o, lse = Bd.training_attention_lse(Bd.KF_MASK_SINGLE, q, k, v, N, K)
    r = _rows(o)
    x2 = x + mm(r, p["wo"].t()).float()
    y2, s2 = Bd.layer_norm(x2, p["g2"], p["b2"], out_dtype=BF)
    logits = mm(y2, p["head"].t())
    dl, lp = Bd.token_logprobs_backward(logits, tok, w)
    loss = (lp.logp * w).sum()
    wg = lambda d, a: torch.mm(d.reshape(-1, d.shape[-1]).float().t(), a.reshape(-1, a.shape[-1]).float())
    dhead = wg(dl, y2)
    dx2, dg2, db2 = Bd.layer_norm_backward(mm(dl, p["head"]), x2, p["g2"], s2)
    do_ = dx2.to(BF)
    dwo = wg(do_, r)
    dq, dk, dv = Bd.training_attention_backward(Bd.KF_MASK_SINGLE, q, k, v, o, lse, _heads(mm(do_, p["wo"])), N, K)
    dqkv = torch.cat([_rows(t) for t in (dq, dk, dv)], -1)
    dwqkv = wg(dqkv, y1)
    dx, dg1, db1 = Bd.layer_norm_backward(mm(dqkv, p["wqkv"]), x, p["g1"], s1, dres=dx2)
    grads = [dg1, db1, dwqkv, dwo, dg2, db2, dhead]
    if out is None:
        out = [torch.empty_like(g) for g in grads]
    for a, b in zip(out, grads):
        a.copy_(b)
    plan = plan or Bd.GradClip(out)
    norm = plan.clip(max_norm)
    return loss, norm, dx, out, plan


def _reference(p, x, tok, w):
    """The step in 64 bits by autograd on the same values."""
    q = {n: t.double().requires_grad_(True) for n, t in p.items()}
    x = x.double().requires_grad_(True)
    norm = lambda t, g, b: (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + 1e-5) * g + b
    M = torch.from_numpy(O.training_mask("single", N, K)).bool()
    qkv = norm(x, q["g1"], q["b1"]) @ q["wqkv"].t()
    a, k, v = (t.view(B, ROWS, H, DH).transpose(1, 2) for t in qkv.split(D, -1))
    s = (a @ k.transpose(-1, -2) / math.sqrt(DH)).masked_fill(~M, -math.inf)
    o = (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(B, ROWS, D)
    x2 = x + o @ q["wo"].t()
    lp = torch.log_softmax(norm(x2, q["g2"], q["b2"]) @ q["head"].t(), -1)
    at = tok.long().clamp(min=0)
    loss = (lp.gather(-1, at[..., None])[..., 0] * (tok >= 0) * w.double()).sum()
    names = ["g1", "b1", "wqkv", "wo", "g2", "b2", "head"]
    grads = torch.autograd.grad(loss, [x] + [q[n] for n in names])
    return loss.detach(), grads[0], grads[1:]


def test_step_against_64_bits(Bd):
    """Each of the step's 16 stored bf16 tensors between a gradient and the loss is off by half a
    step, 2^-8 of itself at most and 2^-8 / sqrt(3) of its norm; attention's P and dS twice more.
    Norms of gradients therefore agree to 20 such errors, were they all alike."""
    p, (x, tok, w) = _params(1), _batch(1)
    loss, norm, dx, out, _ = _step(Bd, {n: t.cuda() for n, t in p.items()}, x.cuda(), tok.cuda(), w.cuda())
    torch.cuda.synchronize()
    rl, rdx, rg = _reference(p, x, tok, w)
    tol = 20 * 2.0 ** -8 / math.sqrt(3)
    total = math.sqrt(sum(float((g ** 2).sum()) for g in rg))
    assert total > 0.05
    print("loss", float(loss), float(rl), "norm", float(norm), total)
    assert abs(float(loss - rl)) <= tol * float(rl.abs())
    assert abs(float(norm) - total) <= tol * total
    for n, a, b in [("x", dx, rdx)] + list(zip(("g1", "b1", "wqkv", "wo", "g2", "b2", "head"), out, [g * (0.05 / total) for g in rg])):
        rel = float((a.double().cpu() - b).norm() / b.norm())
        print(n, rel)
        assert rel <= 2 * tol, n  # the gradient's own error and the norm's
    clipped = math.sqrt(sum(float((o.double() ** 2).sum()) for o in out))
    assert abs(clipped - 0.05) <= 1e-6


def test_captured_step_replays(Bd):
    """The step captured into a HIP graph, replayed on new batches with eager work between, against
    the eager step bit for bit; an eager step's results live through the capture."""
    p = {n: t.cuda() for n, t in _params(2).items()}
    x, tok, w = (t.cuda() for t in _batch(2))
    eager0 = _step(Bd, p, x, tok, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _, _, _, out, plan = _step(Bd, p, x, tok, w)  # warm-up, and the buffers of the plan
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm, dx, _, _ = _step(Bd, p, x, tok, w, out, plan)
    for seed in (3, 4, 2):
        nx, ntok, nw = (t.cuda() for t in _batch(seed))
        x.copy_(nx)
        tok.copy_(ntok)
        graph.replay()
        torch.cuda.synchronize()
        got = [loss.clone(), norm.clone(), dx.clone()] + [o.clone() for o in out]
        e = _step(Bd, p, nx, ntok, nw)
        want = [e[0], e[1], e[2]] + e[3]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
    assert all(torch.equal(a, b) for a, b in zip(got, [eager0[0], eager0[1], eager0[2]] + eager0[3]))


def test_another_stream(Bd):
    """Work given a stream of its own, its results allocated there, equals the current stream's."""
    x, gain = torch.randn(3000, 768, device="cuda"), torch.rand(768, device="cuda")
    logits, tok = torch.randn(600, 9001, device="cuda"), torch.zeros(600, dtype=torch.int32, device="cuda")
    u = torch.rand(600, device="cuda")
    q, k, v, do = (torch.randn(2, 3, 75, 64, device="cuda").to(BF) for _ in range(4))
    g = [torch.randn(100_000, device="cuda"), torch.randn(7, device="cuda")]

    def run(stream=None):
        y, st = Bd.layer_norm(x, gain, rms=True, out_dtype=BF, stream=stream)
        r = [y, st, *Bd.layer_norm_backward(y, x, gain, st, rms=True, stream=stream)[:2]]
        r += Bd.token_logprobs(logits, tok, 4, lse=True, stream=stream)
        r += [Bd.token_logprobs_backward(logits, tok, u, stream=stream)[0]]
        o, l = Bd.training_attention_lse(0, q, k, v, 25, 2, stream=stream)
        r += [o, l, *Bd.training_attention_backward(0, q, k, v, o, l, do, 25, 2, stream=stream)]
        out = [torch.empty_like(t) for t in g]
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        plan = Bd.GradClip(g, out, stream=stream)
        r += [plan.clip(1.0, stream=stream), plan.norm(stream=stream)] + out
        return r
    want = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(s)
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
