"""The operators of the training step in 64 bits, on the CPU, and bounds on how far a kernel
may be from them.

U is the unit roundoff of the fp32 sums; HALF[type] half a step of a stored value, relative to
it (2^-8 bf16, 2^-11 fp16, 2^-24 fp32).  A sum of n fp32 terms is off by at most n U times the sum
of their magnitudes whatever its order; the kernels add at most n / 64 terms one after another
(64 or more lanes share a row) and join the lanes in a tree of fewer than 16 levels.
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half a step of the smallest values, which a relative step does not cover (bf16 and fp32: the
# smallest normal number, below which results may be flushed to zero)
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def worst(got, ref, bound):
    """The largest error in units of its bound; an infinity or NaN must be met exactly."""
    got, ref = got.double().cpu(), ref.double()
    odd = ~torch.isfinite(ref)
    assert torch.equal(torch.isnan(got[odd]), torch.isnan(ref[odd]))
    plain = odd & ~torch.isnan(ref)
    assert torch.equal(got[plain], ref[plain])
    assert torch.isfinite(got[~odd]).all()
    if not (~odd).any():
        return 0.0
    return float(((got - ref).abs() / bound.expand_as(ref))[~odd].max())


# ------------------------------------------------------------------- norms
def norm(x, gain, shift, eps, rms):
    x = x.double()
    mu = torch.zeros_like(x[..., :1]) if rms else x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt(((x - mu) ** 2).mean(-1, keepdim=True) + eps)
    y = (x - mu) * r * gain.double()
    return (y if shift is None else y + shift.double()), mu, r


def norm_bound(x, gain, shift, eps, rms, out_type):
    """The mean is off by K U mean|x| (K terms one after another and a few roundings), the root by
    K U of itself; then a handful of roundings of each element."""
    y, mu, r = norm(x, gain, shift, eps, rms)
    x = x.double()
    K = x.shape[-1] / 64 + 32
    mag = ((x - mu).abs() + x.abs().mean(-1, keepdim=True)) * r * gain.double().abs()
    if shift is not None:
        mag = mag + shift.double().abs()
    return HALF[out_type] * y.abs() + K * U * mag + TINY[out_type]


def norm_grad(dy, x, gain, eps, rms, dres=None):
    """(dx, dgain, dshift) and their bounds."""
    _, mu, r = norm(x, gain, None, eps, rms)
    t = x.dtype
    x, dy, g = x.double(), dy.double(), gain.double()
    xh, w = (x - mu) * r, dy * g
    mean = lambda a: a.mean(-1, keepdim=True)
    dx = r * (w - xh * mean(w * xh) - (0 if rms else mean(w)))
    size = xh.abs() + mean(x.abs()) * r  # what an error of x hat is relative to
    mag = r * (w.abs() + mean(w.abs()) + size * mean(w.abs() * size))
    if dres is not None:
        dx, mag = dx + dres.double(), mag + dres.double().abs()
    K, rows = x.shape[-1] / 64 + 32, x.reshape(-1, x.shape[-1]).shape[0]
    bound = HALF[t] * dx.abs() + K * U * mag + TINY[t]
    lead = tuple(range(x.dim() - 1))
    dg, db = (dy * xh).sum(lead), dy.sum(lead)
    C = rows + K
    return (dx, dg, db), (bound, C * U * (dy.abs() * size).sum(lead) + 1e-30, C * U * dy.abs().sum(lead) + 1e-30)


# ------------------------------------------------------- log probabilities
def logprobs(logits, tokens, n_top=0):
    """dict of the results and of their bounds (keys with _b)."""
    x = logits.double()
    V = x.shape[-1]
    empty = (x == -math.inf).all(-1)
    m = x.max(-1, keepdim=True).values
    m = torch.where(empty[..., None], torch.zeros_like(m), m)
    e = torch.exp(x - m)
    s = e.sum(-1)
    ls = torch.log(s)
    lse = m[..., 0] + ls
    p = e / s.masked_fill(empty, 1.0)[..., None]
    lp = torch.where(empty[..., None], torch.full_like(x, -math.inf), (x - m) - ls[..., None])  # m + log s can lose log s
    plp = torch.where(p == 0, torch.zeros_like(p), p * lp)
    entropy = -plp.sum(-1)
    entropy = torch.where(empty, torch.zeros_like(entropy), entropy)
    tok = tokens.long()
    logp = lp.gather(-1, tok.clamp(0, V - 1)[..., None])[..., 0]
    logp = torch.where(tok < 0, torch.zeros_like(logp), logp)
    logp = torch.where(tok >= V, torch.full_like(logp, math.nan), logp)
    spread = torch.where(p == 0, torch.zeros_like(p), p * (m - x)).sum(-1)  # sum p (max - l)
    K = V / 64 + 100  # terms in a row, the exponentials' own errors (2 U |l - max| each), the log
    out = dict(spread=spread, logp=logp, lse=lse, entropy=entropy, p=p, lp=lp, empty=empty,
               lse_b=U * (K + 8 * spread + 4 * lse.abs()),
               logp_b=U * (K + 8 * spread + 4 * (logp.abs() + lse.abs())),
               entropy_b=U * (K + 8 * spread) * (2 + 2 * spread + torch.log(s.clamp(min=1))))
    if n_top:
        key = torch.where(torch.isnan(x), torch.full_like(x, math.inf), x)
        big = torch.isnan(x).long()
        ids = torch.arange(V).expand(x.shape)
        # larger first, NaN before all, equal ones by the lower id
        order = torch.argsort(key, dim=-1, descending=True, stable=True)
        order = order.gather(-1, torch.argsort(big.gather(-1, order), dim=-1, descending=True, stable=True))
        out["top_ids"] = ids.gather(-1, order)[..., :n_top].int()
        out["top_logp"] = lp.gather(-1, order)[..., :n_top]
        out["top_b"] = U * (K + 8 * spread[..., None] + 4 * (out["top_logp"].abs() + lse.abs()[..., None]))
    return out


def logprobs_grad(logits, tokens, u, c):
    """d_logits and its bound."""
    r = logprobs(logits, tokens)
    x, V, t = logits.double(), logits.shape[-1], logits.dtype
    tok = tokens.long()
    u = torch.zeros(tok.shape, dtype=torch.float64) if u is None else u.double()
    u = torch.where(tok < 0, torch.zeros_like(u), u)
    u = torch.where(tok >= V, torch.full_like(u, math.nan), u)[..., None]
    c = torch.zeros(tok.shape, dtype=torch.float64)[..., None] if c is None else c.double()[..., None]
    one = torch.zeros_like(x).scatter_(-1, tok.clamp(0, V - 1)[..., None], 1.0)
    one = torch.where((tok < 0)[..., None], torch.zeros_like(one), one)
    h, p = r["entropy"][..., None], r["p"]
    lp = torch.where(p == 0, torch.zeros_like(p), r["lp"])
    d = u * (one - p) - c * p * (lp + h)
    d = torch.where(r["empty"][..., None], torch.zeros_like(d), d)
    K = V / 64 + 100
    rel = U * (K + 8 * (lp.abs() + r["spread"][..., None]))  # of one probability, e / s
    mag = u.abs().nan_to_num() * (p * rel + one * U * 4) + c.abs() * p * ((rel + 4 * U) * (lp.abs() + h + 1) + r["entropy_b"][..., None])
    return d, HALF[t] * d.abs().nan_to_num() + mag + TINY[t] * (1 + u.abs().nan_to_num() + c.abs() * 128)


# -------------------------------------------------------------- attention
def attention(q, k, v, mask, scale):
    """(o, lse, p) of one or more heads in fp64; mask [rows][keys] bool."""
    a = torch.matmul(q.double(), k.double().transpose(-1, -2)) * scale
    a = a.masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(a, -1)
    p = torch.exp(a - lse[..., None])
    return torch.matmul(p, v.double()), lse, p


def attention_grad(q, k, v, do, mask, scale):
    """((dq, dk, dv), their bounds).  With h half a bf16 step: the forward call's row sums are of
    probabilities rounded to bf16, so lse and with it P is off by h; P is rounded again for dV
    (2 h in all), dS once (3 h); O is off by 2 h sum P|v| (rounded probabilities) and h |O|, and D =
    dO.O with it; scores by (d_head + 8) U sum|q k|.  The results are rounded once (h)."""
    h = HALF[torch.bfloat16]
    o, _, p = attention(q, k, v, mask, scale)
    q, k, v, do = (t.double() for t in (q, k, v, do))
    T = lambda t: t.transpose(-1, -2)
    dp = do @ T(v)
    D = (do * o).sum(-1, keepdim=True)
    ds = p * (dp - D)
    dq, dk, dv = ds @ k * scale, T(ds) @ q * scale, T(p) @ do
    n = q.shape[-1] + 8
    score = n * U * abs(scale) * (q.abs() @ T(k.abs()))
    rows, keys = p.shape[-2:]
    pe = p * (2 * h + score + (rows + 8) * U)
    de = (do.abs() * (2 * h * (p @ v.abs()) + h * o.abs())).sum(-1, keepdim=True) + n * U * (do.abs() @ T(v.abs()))
    se = ds.abs() * (3 * h + score + (rows + keys) * U) + p * de
    ab = abs(scale)
    bounds = (ab * (se @ k.abs()) + h * dq.abs(), ab * (T(se) @ q.abs()) + h * dk.abs(),
              T(pe) @ do.abs() + h * dv.abs())
    return (dq, dk, dv), tuple(1.05 * b + 1e-6 for b in bounds)  # 1.05: products of two errors
