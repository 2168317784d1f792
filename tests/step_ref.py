"""Heads of a QKV product, dropout and the policy loss in 64 bits, on the CPU, and bounds on how far
a kernel may be from them (U, HALF and TINY as in tests/train_ref.py)."""
import math

import numpy as np
import torch

from tests.train_ref import HALF, TINY, U, logprobs, logprobs_grad

# Roundings of a head's root: at most 8 squares one after another in a lane, 6 levels over lanes, the
# mean, eps, the root and the quotient, each U of the sum or less; then x r and its gain.
C_NORM = 24


# ------------------------------------------------------------------- heads
def _split(t, Hq, Hkv, dh):
    """[B][L][W] as q, k, v [B][H][L][dh]."""
    B, L, _ = t.shape
    return t.view(B, L, Hq + 2 * Hkv, dh).transpose(1, 2).split([Hq, Hkv, Hkv], 1)


def _angles(table, pos, B, L, dh):
    """cos and sin [B][1][L][dh / 2] of every pair, 1 and 0 past the table's columns."""
    c, s = torch.ones(B, L, (dh + 1) // 2, dtype=torch.float64), torch.zeros(B, L, (dh + 1) // 2, dtype=torch.float64)
    if table is not None:
        at = (torch.arange(L).expand(B, L) if pos is None else pos.expand(B, L)).long()
        out = (at < 0) | (at >= table.shape[0])
        rows = table.double()[at.clamp(0, table.shape[0] - 1)]
        n = rows.shape[2]
        c[..., :n] = torch.where(out[..., None], math.nan, rows[..., 0])
        s[..., :n] = torch.where(out[..., None], math.nan, rows[..., 1])
    return c[:, None], s[:, None]


def turn(t, c, s, way=1):
    """(the turned t, the sums of the magnitudes that entered each element)."""
    dh = t.shape[-1]
    if dh % 2:
        t = torch.nn.functional.pad(t, (0, 1))
    a, b = t[..., 0::2], t[..., 1::2]
    s = way * s
    # (an angle of 0 takes nothing from the other of a pair, whatever that is)
    y = torch.stack([a * c - torch.where(s == 0, 0.0, b * s), torch.where(s == 0, 0.0, a * s) + b * c], -1).flatten(-2)
    m = torch.stack([(a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()], -1).flatten(-2)
    return y[..., :dh], m[..., :dh]


def heads(x, Hq, Hkv, dh, table, pos, gq, gk, eps, out_type):
    """[(value, bound)] of q, k and v."""
    B, L, _ = x.shape
    c, s = _angles(table, pos, B, L, dh)
    out = []
    for t, g, turned in zip(_split(x.double(), Hq, Hkv, dh), (gq, gk, None), (True, True, False)):
        C = 4.0
        if g is not None:
            t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * g.double()
            C += C_NORM
        y, m = turn(t, c, s) if turned else (t, t.abs())
        out.append((y, HALF[out_type] * y.abs() + C * U * m + TINY[out_type]))
    return out


def heads_grad(dq, dk, dv, x, Hq, Hkv, dh, table, pos, gq, gk, eps, x_type):
    """((dx, bound), (dgq, bound), (dgk, bound)); x may be None without gains."""
    B, _, L, _ = (dq if Hq else dk).shape
    c, s = _angles(table, pos, B, L, dh)
    xs = _split(x.double(), Hq, Hkv, dh) if x is not None else (None,) * 3
    parts, bounds, gains = [], [], []
    for d, t, g, turned in zip((dq, dk, dv), xs, (gq, gk, None), (True, True, False)):
        d = d.double()
        w, m = turn(d, c, s, -1) if turned else (d, d.abs())
        C = 4.0
        if g is not None:
            r = 1 / torch.sqrt((t * t).mean(-1, keepdim=True) + eps)
            xh, wg, mg = t * r, w * g.double(), m * g.double().abs()
            gains.append(((w * xh).sum((0, 1, 2)), (B * L * d.shape[1] + 2 * C_NORM + 16) * U * (m * xh.abs()).sum((0, 1, 2)) + 1e-30))
            w = r * (wg - xh * (wg * xh).mean(-1, keepdim=True))
            m = r * (mg + xh.abs() * (mg * xh.abs()).mean(-1, keepdim=True))
            C += 4 * C_NORM  # r thrice and the mean of dh products
        elif turned:
            gains.append(None)
        parts.append(w)
        bounds.append(HALF[x_type] * w.abs() + C * U * m + TINY[x_type])
    join = lambda p: torch.cat(p, 1).transpose(1, 2).reshape(B, L, -1)
    return (join(parts), join(bounds)), gains[0], gains[1]


# ----------------------------------------------------------------- dropout
def philox(c, key):
    """Philox4x32-10 of counters c, four arrays, under key, two numbers (Salmon et al., SC'11)."""
    c = [np.asarray(v, dtype=np.uint64) for v in c]
    low, k = np.uint64(0xFFFFFFFF), list(key)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return [v.astype(np.uint32) for v in c]


def threshold(p):
    return int(np.rint(np.float32(p) * np.float32(65536)))


def kept(rows, d, p, seed, site, row0=0):
    """Which elements of rows row0 .. row0 + rows - 1 stay, bool [rows][d]."""
    seed &= 2 ** 64 - 1
    g = (d + 7) // 8
    row = np.repeat(np.arange(row0, row0 + rows, dtype=np.uint64), g)
    w = philox([np.tile(np.arange(g, dtype=np.uint64), rows), row % 2 ** 32, row // 2 ** 32, np.full(rows * g, 2 ** 31 + site)],
               (seed % 2 ** 32, seed // 2 ** 32))
    n = np.stack([v for x in w for v in (x & 0xFFFF, x >> 16)], -1).reshape(rows, -1)[:, :d]
    return torch.from_numpy(n.astype(np.int64) >= threshold(p))


def dropout(x, p, seed, site, res, out_type, row0=0):
    """(value, bound) for x [rows][d]: the scale is off by U, the product or sum by U."""
    T = threshold(p)
    s = 0.0 if T == 65536 else 65536 / (65536 - T)
    keep = kept(*x.shape, p, seed, site, row0)
    y = torch.where(keep, x.double() * s, 0.0)
    m = y.abs()
    if res is not None:
        y, m = y + res.double(), m + res.double().abs()
    return y, HALF[out_type] * y.abs() + torch.where(keep, 3 * U * m + TINY[out_type], 0.0)


# ------------------------------------------------------------- policy loss
def policy(logits, tokens, adv, old, ref, w, low, high, beta, c):
    """dict of the results (rows [R]) and their bounds (keys with _b)."""
    rows, V = logits.shape
    w = torch.ones(rows, dtype=torch.float64) if w is None else w.double()
    on = (tokens >= 0) & (w != 0)
    tok = torch.where(on, tokens, torch.full_like(tokens, -1))
    x = torch.where(on[:, None], logits.double(), 0.0)  # a row that does not count may hold anything
    r = logprobs(x, tok)
    lp, H, lp_b, H_b = r["logp"], r["entropy"], r["logp_b"], r["entropy_b"]
    A = adv.double()
    gap = torch.zeros_like(lp) if old is None else lp - old.double()
    ratio = torch.exp(gap)
    gap_b = torch.zeros_like(lp) if old is None else lp_b + U * (6 * gap.abs().nan_to_num(posinf=0) + 8)
    ratio_b = torch.where(ratio == 0, 0.0, ratio * gap_b) + TINY[torch.float32]
    plain, clipped = ratio * A, ratio.clamp(low, high) * A
    cut = plain > clipped
    loss = -torch.where(cut, clipped, plain)
    u = torch.where(cut, 0.0, -plain)
    loss_b = A.abs() * (ratio_b + 4 * U * torch.where(cut, clipped.abs(), plain.abs()))
    u_b = torch.where(cut, 0.0, A.abs() * ratio_b + 4 * U * plain.abs())
    kl = kl_b = torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        e = torch.expm1(d)
        kl = torch.where(d == math.inf, math.inf, e - d)
        d_b = lp_b + U * d.abs()
        # the series' 8 terms, relative; past 1/2 the exponential (its argument off by 3 U |d|) and two sums
        own = torch.where(d.abs() < 0.5, 32 * U * kl, U * ((e + 1) * (4 * d.abs() + 6) + 4 * d.abs() + 4))
        kl_b = e.abs() * d_b + (e + 1) * d_b ** 2 + own
        if beta:
            loss, loss_b = loss + beta * kl, loss_b + abs(beta) * (kl_b + 4 * U * kl)
            u, u_b = u - beta * e, u_b + abs(beta) * (kl_b + d_b + 4 * U * (kl + d.abs()))
    if c:
        loss, loss_b = loss - c * H, loss_b + abs(c) * (H_b + 4 * U * H)
    loss, loss_b, u, u_b = loss * w, (loss_b + 8 * U * loss.abs()) * w.abs(), u * w, (u_b + 4 * U * u.abs()) * w.abs()
    none = lambda t: torch.where(on, t, torch.zeros_like(t))
    out = dict(on=on, logp=none(lp), ratio=none(ratio), kl=none(kl), entropy=none(H), row_loss=none(loss), u=none(u), c=none(-w * c),
               cut=cut, logp_b=lp_b, ratio_b=ratio_b, kl_b=kl_b, entropy_b=H_b, row_loss_b=none(loss_b) + 1e-38, u_b=none(u_b))
    for n in ("logp", "ratio", "kl", "entropy"):
        out[n + "_b"] = none(out[n + "_b"]) + 1e-38
    out["loss"] = out["row_loss"].sum()
    out["loss_b"] = out["row_loss_b"].sum() + U * out["loss"].abs() + 1e-38
    # the gradient from u and c exactly, and what u's error adds
    t = logits.dtype
    d, d_b = logprobs_grad(x.to(t) if t != torch.float64 else x, tok, out["u"], out["c"])
    one = torch.zeros_like(d).scatter_(1, tok.long().clamp(0, V - 1)[:, None], 1.0) * (tok >= 0)[:, None]
    out["d_logits"], out["d_logits_b"] = d, d_b + torch.where(r["p"] + one == 0, 0.0, out["u_b"][:, None] * (one - r["p"]).abs())
    return out
