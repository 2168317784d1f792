"""More operators of a K-Forcing student's training step, as cases that can be timed and compared.

Four operators, each in its plain form (elementary torch operations in 32 bits) and through the
Python binding of the C ABI:

  heads         rows of a QKV product into attention's layout, with an RMS norm of each query and key
                head and rotary positions ("forward"), and with the gradients ("step")
  dropout       dropout from a counter-based generator, added to a residual, and its gradient
  dropout_norm  the same sum with the norm of its rows in one pass, and the gradients
  policy        the clipped policy loss with a KL term and an entropy bonus over rows of logits, alone
                ("forward") or with the gradient of the logits ("step")

Sizes are those of the model shapes that the benchmark and the tests run (the toy model, the
LM1B- and OpenWebText-shaped backbones, the 24-layer backbone) and of batches of their training.

The generator is Philox4x32-10 with the seed as its key: the four words of counter (c / 8, row,
row / 2^32, 2^31 + site) are eight 16-bit numbers, low half first, for columns c .. c + 7 of a row.
An element is dropped where its number is below round(p 65536); the others are scaled by
65536 / (65536 - round(p 65536)).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
PAIRS = [("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp16"), ("bf16", "bf16"), ("fp16", "fp16")]
EPS = 1e-5
BASE = 10000.0
M32 = 0xFFFFFFFF


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # The eight rows of one decode block of one sequence in the paper's rotary backbone: latency.
        dict(name="heads_block", op="heads", mode="forward", B=1, L=8, Hq=12, Hkv=12, dh=64, rot=64, norm=False, x="bf16", y="bf16", start=500, k=0),
        # A training step of the LM1B shape under the SingleForward layout (128 context rows, four noise
        # rows after each), with norms of queries and keys.
        dict(name="heads_step_lm1b", op="heads", mode="step", B=64, L=640, Hq=12, Hkv=12, dh=64, rot=64, norm=True, x="bf16", y="bf16", start=0, k=4),
        # The 24-layer backbone with the paper's rotary positions alone, OpenWebText-length sequences.
        dict(name="heads_step_large", op="heads", mode="step", B=16, L=5120, Hq=16, Hkv=16, dh=64, rot=64, norm=False, x="bf16", y="bf16", start=0, k=4),
        # Shared key and value heads of an unusual width, part of it rotated, a single-precision product,
        # far positions, an odd length.
        dict(name="heads_shared", op="heads", mode="step", B=3, L=1021, Hq=16, Hkv=4, dh=96, rot=48, norm=True, x="fp32", y="bf16", start=30000, k=0),
        # The embedding dropout of one short toy sequence in single precision: latency.
        dict(name="dropout_toy", op="dropout", rows=80, d=128, x="fp32", y="fp32", p=0.1),
        # The residual dropout after a block's last product, LM1B shape: bf16 into the fp32 stream and back.
        dict(name="dropout_step_lm1b", op="dropout", rows=64 * 640, d=768, x="bf16", y="fp32", p=0.1),
        # A ragged handful of rows of an odd width.
        dict(name="dropout_norm_odd", op="dropout_norm", rms=False, rows=37, d=771, x="fp32", y="fp32", p=0.2),
        # The joint of a pre-norm block at the LM1B shape: fp32 residual stream, bf16 products.
        dict(name="dropout_norm_lm1b", op="dropout_norm", rms=False, rows=64 * 640, d=768, x="fp32", y="bf16", p=0.1),
        # The same at the 24-layer backbone's width with RMSNorm and a bf16 stream.
        dict(name="dropout_norm_large", op="dropout_norm", rms=True, rows=16 * 5120, d=1024, x="bf16", y="bf16", p=0.05),
        # Two short answers of the toy model: latency.
        dict(name="policy_toy", op="policy", mode="step", rows=32, V=1024, dtype="fp32", ref=True, entropy=0.01, ignored=0.1),
        # Answers sampled by the OpenWebText-shaped model, a quarter of the batch padding: the largest logits.
        dict(name="policy_owt", op="policy", mode="step", rows=8192, V=50257, dtype="bf16", ref=True, entropy=0.0, ignored=0.25),
        # The loss alone over a held-out LM1B batch, single-precision logits, an odd number of rows.
        dict(name="policy_lm1b", op="policy", mode="forward", rows=4099, V=30522, dtype="fp32", ref=True, entropy=0.01, ignored=0.05),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["heads", "heads", "dropout", "dropout_norm", "policy"])
    x, y = rng.choice(PAIRS)
    if op == "heads":
        dh = rng.choice([32, 64, 64, 128, 8 * rng.randint(1, 32), rng.randint(5, 200)])
        rot = rng.choice([0, min(64, dh // 2 * 2), dh // 2 * 2, dh // 4 * 2])
        Hkv = rng.choice([1, 2, 4, 12, 16])
        Hq = Hkv * rng.choice([1, 1, 2, 3])
        rows = _log(rng, 1, max(1, 60_000_000 // ((Hq + 2 * Hkv) * dh)))
        B = _log(rng, 1, min(rows, 64))
        k = rng.choice([0, 0, 1, 2, 4])
        L = max(1, rows // B // (1 + k)) * (1 + k)
        return dict(op=op, mode=rng.choice(["forward", "step", "step"]), B=B, L=L, Hq=Hq, Hkv=Hkv, dh=dh, rot=rot,
                    norm=rng.random() < 0.6, x=x, y=y, start=0 if k else rng.choice([0, 1000, 60000]), k=k)
    if op in ("dropout", "dropout_norm"):
        d = rng.choice([_log(rng, 33, 8192), 64 * rng.randint(1, 32)])
        rows = _log(rng, 1, max(1, 40_000_000 // d))
        p = rng.choice([0.0, 0.05, 0.1, 0.3, 0.5])
        if op == "dropout":
            x, y = rng.choice([("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp32"), ("bf16", "bf16"), ("fp16", "fp16")])
            return dict(op=op, rows=rows, d=d, x=x, y=y, p=p)
        return dict(op=op, rms=rng.random() < 0.4, rows=rows, d=d, x=x, y=y, p=p)
    V = rng.choice([30522, 50257, _log(rng, 100, 130000)])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    rows = _log(rng, 1, max(1, 400_000_000 // V // BYTES[dtype]))
    return dict(op=op, mode=rng.choice(["forward", "step", "step"]), rows=rows, V=V, dtype=dtype, ref=rng.random() < 0.7,
                entropy=rng.choice([0.0, 0.0, 0.01]), ignored=rng.choice([0.0, 0.1, 0.6]))


# ------------------------------------------------------------------ inputs
def _positions(case):
    """Positions of the rows: the SingleForward layout for k > 0 (context t at t, noise j of group t at
    t + 1 + j), the same for every sequence; otherwise each sequence goes on from where it is."""
    B, L, k = case["B"], case["L"], case["k"]
    if k:
        N = L // (1 + k)
        t = torch.arange(N)
        return torch.cat([t, (t[:, None] + 1 + torch.arange(k)).reshape(-1)]).int()
    return (case["start"] + 7 * torch.arange(B)[:, None] + torch.arange(L)).int()


def _table(n, rot):
    """cos and sin of position times base^(-2i / rot), kept by a program as the weights are."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * BASE ** (-2 * i / rot)
    return torch.stack([torch.cos(a), torch.sin(a)], -1).float().contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = dict(case=case)
    if case["op"] == "heads":
        B, L, Hq, Hkv, dh = (case[n] for n in ("B", "L", "Hq", "Hkv", "dh"))
        # a product's rows: columns of unlike strength, a few strong ones
        W = (Hq + 2 * Hkv) * dh
        col = (0.5 + rand(W)) * (1 + 6 * (rand(W) < 0.02).float())
        s["qkv"] = (randn(B, L, W) * col).to(TYPES[case["x"]])
        pos = _positions(case)
        s["pos"] = pos.cuda()
        s["table"] = _table(int(pos.max()) + 1, case["rot"]) if case["rot"] else None
        s["gq"] = 1 + 0.2 * randn(dh) if case["norm"] else None
        s["gk"] = 1 + 0.2 * randn(dh) if case["norm"] else None
        if case["mode"] == "step":
            yt = TYPES[case["y"]]
            s["dq"], s["dk"], s["dv"] = ((0.1 * randn(B, H, L, dh)).to(yt) for H in (Hq, Hkv, Hkv))
    elif case["op"] in ("dropout", "dropout_norm"):
        rows, d = case["rows"], case["d"]
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=g, device="cuda"))
        s["site"] = seed % 48
        if case["op"] == "dropout":
            s["x"] = randn(rows, d).to(TYPES[case["x"]])
            s["res"] = (randn(rows, d) * 3).to(TYPES[case["y"]])
            s["dy"] = (0.1 * randn(rows, d)).to(TYPES[case["y"]])
        else:  # x is the residual stream's type here, y the products'
            xt, yt = TYPES[case["x"]], TYPES[case["y"]]
            s["x"] = randn(rows, d).to(yt)
            s["res"] = (randn(rows, d) * (1 + 8 * (rand(d) < 0.01).float()) + 0.5 * randn(rows, 1)).to(xt)
            s["gain"] = 1 + 0.2 * randn(d)
            s["shift"] = None if case["rms"] else 0.1 * randn(d)
            s["dy"] = (0.1 * randn(rows, d)).to(yt)
            s["dres"] = (0.1 * randn(rows, d)).to(xt)
    else:
        rows, V = case["rows"], case["V"]
        x = randn(rows, V) * 2.5
        tok = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
        # a trained model's rows: the sampled token often among the likely ones
        x.scatter_add_(1, tok.long()[:, None], 8 * rand(rows, 1))
        s["logits"] = x.to(TYPES[case["dtype"]])
        x = s["logits"].float()
        lp = x.gather(1, tok.long()[:, None])[:, 0] - torch.logsumexp(x, 1)
        # The policy that sampled is some updates older than this one.  Ratios stay 1e-3 off the clipping
        # borders: on either side of one the gradient jumps, so there the last bits of the logarithm decide.
        step = 0.2 * randn(rows)
        for border in (math.log(0.8), math.log(1.28)):
            step = torch.where((step - border).abs() < 1e-3, step + 3e-3, step)
        s["old"] = lp - step
        s["ref"] = lp + 0.3 * randn(rows) if case["ref"] else None
        s["adv"] = randn(rows) + 0.5  # rewards over a baseline that lags behind
        s["w"] = (0.5 + rand(rows)) / rows
        if case["dtype"] == "fp16":  # a scaled loss, as half-precision training has it
            s["w"] *= 64.0 * rows
        tok[rand(rows) < case["ignored"]] = -1
        s["tok"] = tok
    return s


# ------------------------------------------------------------------ the framework's calls
def _run_own(s):
    from paper_2606_10820_amd import binding as kfb
    case = s["case"]
    if case["op"] == "heads":
        args = dict(table=s["table"], positions=s["pos"], q_gain=s["gq"], k_gain=s["gk"], eps=EPS)
        q, k, v = kfb.qkv_heads(s["qkv"], case["Hq"], case["Hkv"], out_dtype=TYPES[case["y"]], **args)
        if case["mode"] == "forward":
            return [q, k, v]
        d, dgq, dgk = kfb.qkv_heads_backward(s["dq"], s["dk"], s["dv"], s["qkv"], **args)
        return [q, k, v, d] + ([dgq, dgk] if case["norm"] else [])
    if case["op"] == "dropout":
        y = kfb.dropout(s["x"], case["p"], s["seed"], s["site"], residual=s["res"])
        return [y, kfb.dropout_backward(s["dy"], case["p"], s["seed"], s["site"], out_dtype=TYPES[case["x"]])]
    if case["op"] == "dropout_norm":
        h, y, stats = kfb.dropout_norm(s["x"], s["res"], s["gain"], s["shift"], case["p"], s["seed"], s["site"], eps=EPS, rms=case["rms"])
        dh, dx, dgain, dshift = kfb.dropout_norm_backward(s["dy"], h, s["gain"], stats, case["p"], s["seed"], s["site"], rms=case["rms"], dres=s["dres"])
        return [h, y, dh, dx, dgain] + ([] if case["rms"] else [dshift])
    r = kfb.policy_loss(s["logits"], s["tok"], s["adv"], s["old"], s["ref"], s["w"], clip_low=0.2, clip_high=0.28,
                        kl_coef=0.05 if case["ref"] else 0.0, entropy_coef=case["entropy"], grad=case["mode"] == "step")
    return [r.loss, r.row_loss, r.logp, r.ratio, r.entropy] + ([r.kl] if case["ref"] else []) + ([r.d_logits] if case["mode"] == "step" else [])


# ------------------------------------------------------------------ the plain forms
def _turn(x, cs, rot, back=False):
    """Pairs (2i, 2i + 1) of the first `rot` columns turned by the rows' angles, or back."""
    if not rot:
        return x
    c, sn = cs[..., 0], -cs[..., 1] if back else cs[..., 1]
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2), x[..., rot:]], -1)


def _heads_plain(s):
    case = s["case"]
    B, L, Hq, Hkv, dh, rot = (case[n] for n in ("B", "L", "Hq", "Hkv", "dh", "rot"))
    yt = TYPES[case["y"]]
    x = s["qkv"].float().view(B, L, Hq + 2 * Hkv, dh)
    cs = s["table"][s["pos"].long()].unsqueeze(-3) if rot else None  # [B or none][L][1][rot / 2][2]
    gains = torch.cat([s["gq"].expand(Hq, dh), s["gk"].expand(Hkv, dh)]) if case["norm"] else None
    qk = x[:, :, :Hq + Hkv]
    if case["norm"]:
        r = 1 / torch.sqrt((qk * qk).mean(-1, keepdim=True) + EPS)
        xh = qk * r
        qk = xh * gains
    qk = _turn(qk, cs, rot)
    y = torch.cat([qk, x[:, :, Hq + Hkv:]], 2).transpose(1, 2).to(yt)
    out = [t.contiguous() for t in y.split([Hq, Hkv, Hkv], 1)]
    if case["mode"] == "forward":
        return out
    dy = torch.cat([s["dq"], s["dk"], s["dv"]], 1).transpose(1, 2).float()
    w = _turn(dy[:, :, :Hq + Hkv], cs, rot, back=True)
    dg = []
    if case["norm"]:
        t = (w * xh).sum((0, 1))
        dg = [t[:Hq].sum(0), t[Hq:].sum(0)]
        w = w * gains
        w = r * (w - xh * (w * xh).mean(-1, keepdim=True))
    d = torch.cat([w, dy[:, :, Hq + Hkv:]], 2).reshape(B, L, -1)
    return out + [d.to(TYPES[case["x"]])] + dg


def _threshold(p):
    return int(torch.round(torch.tensor(p, dtype=torch.float32) * 65536))


def _keep(rows, d, p, seed, site):
    """The elements that dropout keeps, [rows][d]."""
    row = torch.arange(rows, device="cuda")[:, None]
    c0 = torch.arange((d + 7) // 8, device="cuda").expand(rows, -1)
    c = [c0, (row & M32).expand_as(c0), (row >> 32).expand_as(c0), torch.full_like(c0, 2 ** 31 + site)]
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & M32) ^ c[1] ^ k0, b & M32, (a >> 32 & M32) ^ c[3] ^ k1, a & M32]
        k0, k1 = k0 + 0x9E3779B9 & M32, k1 + 0xBB67AE85 & M32
    w = torch.stack(c, -1)
    h = torch.stack([w & 0xFFFF, w >> 16], -1).view(rows, -1)[:, :d]
    return h >= _threshold(p)


def _dropped(x, s):
    case = s["case"]
    T = _threshold(case["p"])
    return torch.where(_keep(case["rows"], case["d"], case["p"], s["seed"], s["site"]), x.float() * (65536.0 / (65536 - T)), 0.0)


def _dropout_plain(s):
    case = s["case"]
    y = (s["res"].float() + _dropped(s["x"], s)).to(TYPES[case["y"]])
    return [y, _dropped(s["dy"], s).to(TYPES[case["x"]])]


def _dropout_norm_plain(s):
    case = s["case"]
    xt, yt = TYPES[case["x"]], TYPES[case["y"]]
    h = (s["res"].float() + _dropped(s["x"], s)).to(xt)
    f = h.float()
    fc = f if case["rms"] else f - f.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((fc * fc).mean(-1, keepdim=True) + EPS)
    xh = fc * r
    y = xh * s["gain"] if case["rms"] else xh * s["gain"] + s["shift"]
    dy = s["dy"].float()
    w = dy * s["gain"]
    dh = w - xh * (w * xh).mean(-1, keepdim=True)
    if not case["rms"]:
        dh = dh - w.mean(-1, keepdim=True)
    dh = (dh * r + s["dres"].float()).to(xt)
    out = [h, y.to(yt), dh, _dropped(dh, s).to(yt), (dy * xh).sum(0)]
    return out if case["rms"] else out + [dy.sum(0)]


def _policy_plain(s):
    case = s["case"]
    x = s["logits"].float()
    m = x.max(-1, keepdim=True).values
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    lse = m + torch.log(z)
    given = s["tok"] >= 0
    at = s["tok"].long().clamp(min=0)[:, None]
    zero = torch.zeros_like(lse[:, 0])
    lp = x.gather(1, at)[:, 0] - lse[:, 0]
    p = e / z
    H = -torch.where(p > 0, p * (x - lse), torch.zeros_like(p)).sum(-1)
    ratio = torch.exp(lp - s["old"])
    plain, clipped = ratio * s["adv"], ratio.clamp(0.8, 1.28) * s["adv"]
    loss = -torch.minimum(plain, clipped) - case["entropy"] * H
    u = torch.where(plain <= clipped, -plain, zero)
    if case["ref"]:
        d = s["ref"] - lp
        kl = torch.exp(d) - d - 1
        loss = loss + 0.05 * kl
        u = u + 0.05 * (1 - torch.exp(d))
    row_loss = torch.where(given, loss * s["w"], zero)
    out = [row_loss.double().sum().float(), row_loss, torch.where(given, lp, zero), torch.where(given, ratio, zero), torch.where(given, H, zero)]
    out += [torch.where(given, kl, zero)] if case["ref"] else []
    if case["mode"] == "forward":
        return out
    w = torch.where(given, s["w"], zero)
    u = torch.where(given, u * w, zero)[:, None]
    d = -p * u
    if case["entropy"]:
        d = d + torch.where(p > 0, p * (x - lse + H[:, None]), torch.zeros_like(p)) * (case["entropy"] * w)[:, None]
    d.scatter_add_(1, at, u)
    return out + [d.to(s["logits"].dtype)]


def run(state):
    if own:
        return _run_own(state)
    return {"heads": _heads_plain, "dropout": _dropout_plain, "dropout_norm": _dropout_norm_plain, "policy": _policy_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------ the definition in 64 bits
def _heads_exact(s):
    case = s["case"]
    B, L, Hq, Hkv, dh, rot = (case[n] for n in ("B", "L", "Hq", "Hkv", "dh", "rot"))
    step = case["mode"] == "step"
    pos = s["pos"].double().expand(B, L)
    x = s["qkv"].double().requires_grad_(step)
    g = [t.double().requires_grad_(step) if t is not None else None for t in (s["gq"], s["gk"])]
    outs = []
    for t, gain in zip(x.view(B, L, -1, dh).transpose(1, 2).split([Hq, Hkv, Hkv], 1), (*g, None)):
        turned = len(outs) < 2
        if gain is not None:
            t = t * ((t ** 2).sum(-1, keepdim=True) / dh + EPS) ** -0.5 * gain
        if turned and rot:  # as complex numbers
            a = pos[:, None, :, None] * torch.exp(torch.arange(rot // 2, device="cuda", dtype=torch.float64) * (-2 * math.log(BASE) / rot))
            z = torch.view_as_complex(t[..., :rot].reshape(B, -1, L, rot // 2, 2)) * torch.polar(torch.ones_like(a), a)
            t = torch.cat([torch.view_as_real(z).reshape(B, -1, L, rot), t[..., rot:]], -1)
        outs.append(t.contiguous())
    if not step:
        return outs
    wrt = [x] + ([*g] if case["norm"] else [])
    grads = torch.autograd.grad(outs, wrt, [s[n].double() for n in ("dq", "dk", "dv")])
    return [o.detach() for o in outs] + list(grads)


def _factors_exact(s):
    """0 or 1 / (1 - p) for each element, from the generator in numpy's unsigned numbers."""
    case = s["case"]
    rows, d = case["rows"], case["d"]
    groups = -(-d // 8)
    T = round(float(np.float32(case["p"])) * 65536)
    out = np.empty((rows, groups, 8), np.uint16)
    u64 = np.uint64
    size = max(1, 1_000_000 // groups)
    for r0 in range(0, rows, size):
        n = min(size, rows - r0)
        x0 = np.tile(np.arange(groups, dtype=u64), n)
        x1 = np.repeat(np.arange(r0, r0 + n, dtype=u64), groups)
        x2, x3 = np.zeros_like(x0), np.full_like(x0, 0x80000000 + s["site"])
        ka, kb = s["seed"] % 2 ** 32, s["seed"] // 2 ** 32
        for i in range(10):
            pa, pb = x0 * u64(0xD2511F53), x2 * u64(0xCD9E8D57)
            x0, x1, x2, x3 = (pb >> u64(32)) ^ x1 ^ u64(ka), pb & u64(M32), (pa >> u64(32)) ^ x3 ^ u64(kb), pa & u64(M32)
            ka, kb = (ka + 0x9E3779B9) % 2 ** 32, (kb + 0xBB67AE85) % 2 ** 32
        words = np.stack([x0, x1, x2, x3], -1).astype("<u4")
        out[r0:r0 + n] = words.view("<u2").reshape(n, groups, 8)
    kept = torch.from_numpy(out.reshape(rows, -1)[:, :d].astype(np.int32)).cuda() >= T
    return kept.double() * (65536 / (65536 - T))


def _dropout_exact(s):
    f = _factors_exact(s)
    return [s["res"].double() + f * s["x"].double(), f * s["dy"].double()]


def _dropout_norm_exact(s):
    case = s["case"]
    f = _factors_exact(s)
    h = s["res"].double() + f * s["x"].double()
    # a stream of 16 bits is what it holds: the norm is of the stored rows
    stored = (lambda t: t) if case["x"] == "fp32" else (lambda t: t.to(TYPES[case["x"]]).double())
    x = stored(h).requires_grad_(True)
    gain = s["gain"].double().requires_grad_(True)
    shift = (torch.zeros_like(gain) if case["rms"] else s["shift"].double()).requires_grad_(True)
    mu = 0 if case["rms"] else x.sum(1, keepdim=True) / case["d"]
    var = ((x - mu) ** 2).sum(1, keepdim=True) / case["d"]
    y = (x - mu) / (var + EPS) ** 0.5 * gain + shift
    dx, dg, db = torch.autograd.grad(y, [x, gain, shift], s["dy"].double())
    dh = dx + s["dres"].double()
    out = [h, y.detach(), dh, f * stored(dh), dg]
    return out if case["rms"] else out + [db]


def _policy_exact(s):
    case = s["case"]
    rows, V = case["rows"], case["V"]
    size = max(1, 100_000_000 // V)
    parts = []
    for i in range(0, rows, size):
        x = s["logits"][i:i + size].double().requires_grad_(True)
        tok = s["tok"][i:i + size].long()
        on = (tok >= 0).double()
        logs = torch.log_softmax(x, 1)
        lp = logs.gather(1, tok.clamp(min=0)[:, None])[:, 0]
        H = -(logs.exp() * logs).sum(1)
        A = s["adv"][i:i + size].double()
        ratio = (lp - s["old"][i:i + size].double()).exp()
        # the smaller of the two, written by the advantage's sign
        bounded = torch.where(A > 0, ratio.clamp(max=1.28), ratio.clamp(min=0.8)) * A
        loss = -bounded - case["entropy"] * H
        kl = None
        if case["ref"]:
            gap = s["ref"][i:i + size].double() - lp
            kl = torch.expm1(gap) - gap
            loss = loss + 0.05 * kl
        row_loss = loss * on * s["w"][i:i + size].double()
        total = row_loss.sum()
        part = [total.detach()[None], row_loss, lp * on, ratio * on, H * on] + ([kl * on] if case["ref"] else [])
        part = [t.detach() for t in part]
        if case["mode"] == "step":
            part.append(torch.autograd.grad(total, x)[0])
        parts.append(part)
    out = [torch.cat(t) for t in zip(*parts)]
    return [out[0].sum()] + out[1:]


def exact(case, seed):
    s = prepare(case, seed)
    return {"heads": _heads_exact, "dropout": _dropout_exact, "dropout_norm": _dropout_norm_exact, "policy": _policy_exact}[case["op"]](s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "heads":
        Hq, Hkv, dh = case["Hq"], case["Hkv"], case["dh"]
        rows = case["B"] * case["L"]
        n, bx, by = rows * (Hq + 2 * Hkv) * dh, BYTES[case["x"]], BYTES[case["y"]]
        turned = rows * (Hq + Hkv) * dh
        passes = 2 if case["mode"] == "step" else 1
        # positions, and the table's rows once
        more = 4 * (case["L"] if case["k"] else rows) + 4 * case["rot"] * case["L"]
        return dict(bytes=passes * (n * (bx + by)) + more, flops=turned * (3 + 5 * case["norm"]) * (1 if passes == 1 else 3))
    if case["op"] == "dropout":
        n, bx, by = case["rows"] * case["d"], BYTES[case["x"]], BYTES[case["y"]]
        return dict(bytes=n * (2 * bx + 3 * by), flops=3 * n)
    if case["op"] == "dropout_norm":
        n, bx, by = case["rows"] * case["d"], BYTES[case["x"]], BYTES[case["y"]]
        return dict(bytes=n * (4 * bx + 4 * by) + 16 * case["d"], flops=25 * n)
    b, rows = BYTES[case["dtype"]], case["rows"]
    read = int(rows * (1 - case["ignored"])) * case["V"] * b  # a row without a token is not needed
    written = rows * case["V"] * b if case["mode"] == "step" else 0
    return dict(bytes=read + written + rows * 36, flops=8 * read // b)
