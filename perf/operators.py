"""The operators that train a K-Forcing model, as cases that can be timed and compared.

Four operators, each in its plain form (elementary torch operations in 32 bits) and through the
Python binding of the C ABI:

  norm       LayerNorm or RMSNorm of rows, alone ("forward") or with the gradients of its input,
             gain and shift ("step"; the gradient of the residual path is added to the input's)
  logprobs   log probabilities of given tokens with entropies and the most probable alternatives
             ("score"), or with the gradient of the logits ("step")
  clip       the norm of a model's whole gradient, and the gradients scaled to a largest norm
  attention  attention under the SingleForward or DoubleForward mask with the gradients of its
             queries, keys and values

Sizes are those of the model shapes that the benchmark and the tests run (the toy model, the
LM1B- and OpenWebText-shaped backbones, the 24-layer backbone) and of batches of their training.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5
SHAPES = {  # layers, d_model, MLP, vocabulary, positions
    "toy": (2, 128, 512, 1024, 128),
    "lm1b": (12, 768, 3072, 30522, 128),
    "owt": (12, 768, 3072, 50257, 1024),
}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # The rows of one decode block of one sequence, an odd width: a single short launch.
        dict(name="norm_few_rows", op="norm", mode="forward", rms=False, rows=8, d=771, x="fp32", y="bf16"),
        # A training step of the LM1B shape: 64 sequences of 128 context and 512 noise rows, the
        # single-precision residual stream into bf16 GEMM inputs, and back.
        dict(name="norm_step_lm1b", op="norm", mode="step", rms=False, rows=64 * 128 * 5, d=768, x="fp32", y="bf16"),
        # The paper's RMSNorm at the width of the 24-layer backbone, 16 sequences of 1024 + 4096 rows.
        dict(name="norm_step_large", op="norm", mode="step", rms=True, rows=16 * 1024 * 5, d=1024, x="bf16", y="bf16"),
        # Four sequences decode one token each and report what it could have been: latency.
        dict(name="score_decode", op="logprobs", mode="score", rows=4, V=50257, dtype="fp32", top=5, masked=0.0),
        # Scoring a batch of LM1B-length texts, with alternatives, part of the vocabulary masked.
        dict(name="score_lm1b", op="logprobs", mode="score", rows=64 * 128, V=30522, dtype="bf16", top=8, masked=0.1),
        # The next-k-token loss of two OpenWebText-length sequences (k = 4): the largest logits.
        dict(name="loss_owt", op="logprobs", mode="step", rows=2 * 1024 * 4, V=50257, dtype="bf16", entropy=False, ignored=0.02),
        # Loss with an entropy term on single-precision logits, a ragged batch with padded rows.
        dict(name="loss_entropy", op="logprobs", mode="step", rows=1003, V=30522, dtype="fp32", entropy=True, ignored=0.3),
        # The toy model's 30 gradients: small tensors, latency.
        dict(name="clip_toy", op="clip", shape="toy", tensors=0, n=0, src="fp32", dst="fp32", clipped=True),
        # The OpenWebText-shaped model's gradients (130 M), bf16 from the GEMMs, fp32 for the optimiser.
        dict(name="clip_owt", op="clip", shape="owt", tensors=0, n=0, src="bf16", dst="fp32", clipped=True),
        # One short sequence of the toy model.
        dict(name="attn_toy", op="attention", mask="single", B=1, H=4, N=16, k=4, dh=32),
        # A training step of the LM1B shape.
        dict(name="attn_single_lm1b", op="attention", mask="single", B=64, H=12, N=128, k=4, dh=64),
        # Self-forcing over OpenWebText-length sequences: 8192 queries, 9216 keys a head.
        dict(name="attn_double_owt", op="attention", mask="double", B=4, H=12, N=1024, k=4, dh=64),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "logprobs", "clip", "attention"])
    if op == "norm":
        d = rng.choice([_log(rng, 33, 8192), 64 * rng.randint(1, 32)])
        rows = _log(rng, 1, max(1, 80_000_000 // d))
        x, y = rng.choice([("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp16"), ("bf16", "bf16"), ("fp16", "fp16")])
        return dict(op=op, mode=rng.choice(["forward", "step", "step"]), rms=rng.random() < 0.4, rows=rows, d=d, x=x, y=y)
    if op == "logprobs":
        V = rng.choice([30522, 50257, _log(rng, 100, 130000)])
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        rows = _log(rng, 1, max(1, 400_000_000 // V // BYTES[dtype]))
        if rng.random() < 0.5:
            return dict(op=op, mode="score", rows=rows, V=V, dtype=dtype, top=rng.randint(0, 20), masked=rng.choice([0.0, 0.0, 0.3, 0.9]))
        return dict(op=op, mode="step", rows=rows, V=V, dtype=dtype, entropy=rng.random() < 0.4, ignored=rng.choice([0.0, 0.05, 0.5]))
    if op == "clip":
        src, dst = rng.choice([("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
        return dict(op=op, shape="", tensors=_log(rng, 1, 400), n=_log(rng, 1000, 60_000_000), src=src, dst=dst, clipped=rng.random() < 0.7)
    mask, dh = rng.choice(["single", "double"]), rng.choice([32, 64, 64, 128])
    k, N = rng.randint(1, 8), _log(rng, 1, 700)
    rows = N * (1 + k) if mask == "single" else 2 * N * k
    heads = max(1, min(512, 200_000_000_000 // (rows * rows * dh)))
    H = rng.choice([1, 3, 4, 12, 16])
    return dict(op=op, mask=mask, B=_log(rng, 1, max(1, heads // H)), H=H, N=N, k=k, dh=dh)


def _sizes(case):
    """Elements of each gradient of a clip case, in a model's order of tensors."""
    if case["shape"]:
        L, d, f, V, n_ctx = SHAPES[case["shape"]]
        out = [V * d, n_ctx * d, 4 * d * d, 4 * d, 4 * d * d, d]
        for _ in range(L):
            out += [d, d, 3 * d * d, 3 * d, d * d, d, d, d, d * f, f, d * f, d]
        return out + [d, d]
    # most of the elements in a few tensors, many short ones beside them
    n, t = case["n"], case["tensors"]
    parts = [1.0 / (i + 1) if i % 3 == 0 else 0.001 for i in range(t)]
    return [max(1, int(n * p / sum(parts))) for p in parts]


def _rows_keys(case):
    N, k = case["N"], case["k"]
    return (N + N * k, N + N * k) if case["mask"] == "single" else (2 * N * k, N + 2 * N * k)


def _entries(case):
    """Visible (query, key) pairs of one head."""
    N, k = case["N"], case["k"]
    noise = k * N * (N + 1) // 2 + N * k * (k + 1) // 2
    return N * (N + 1) // 2 + noise if case["mask"] == "single" else 2 * noise + N * k * k


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _gen(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = dict(case=case)
    if case["op"] == "norm":
        rows, d, xt, yt = case["rows"], case["d"], TYPES[case["x"]], TYPES[case["y"]]
        # residual rows as deep layers have them: an offset, and a few strong columns
        col = 1 + 8 * (rand(d) < 0.01).float()
        s["x"] = (randn(rows, d) * col + 0.5 * randn(rows, 1)).to(xt)
        s["gain"] = 1 + 0.2 * randn(d)
        s["shift"] = None if case["rms"] else 0.1 * randn(d)
        if case["mode"] == "step":
            s["dy"] = (0.1 * randn(rows, d)).to(yt)
            s["dres"] = (0.1 * randn(rows, d)).to(xt)
    elif case["op"] == "logprobs":
        rows, V = case["rows"], case["V"]
        x = randn(rows, V) * 2.5
        s["tokens"] = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
        # a trained model's rows: the given token often among the likely ones
        x.scatter_add_(1, s["tokens"].long()[:, None], 8 * rand(rows, 1))
        if case["mode"] == "score":
            if case["masked"]:
                off = rand(V) < case["masked"]
                off[s["tokens"].long()] = False
                x.masked_fill_(off, -math.inf)
        else:
            s["tokens"][rand(rows) < case["ignored"]] = -1
            s["d_logp"] = -(0.5 + rand(rows)) / rows
            s["d_entropy"] = -0.01 * rand(rows) / rows if case["entropy"] else None
            if case["dtype"] == "fp16":  # a scaled loss, as half-precision training has it
                s["d_logp"] *= 64.0 * rows
                s["d_entropy"] = s["d_entropy"] * (64.0 * rows) if case["entropy"] else None
        s["logits"] = x.to(TYPES[case["dtype"]])
    elif case["op"] == "clip":
        src, dst = TYPES[case["src"]], TYPES[case["dst"]]
        s["src"] = [(10 ** (-1 - 2 * float(i % 7) / 7) * randn(n)).to(src) for i, n in enumerate(_sizes(case))]
        # one flat buffer for the optimiser, a stretch of it for each tensor
        s["flat"] = torch.empty(sum(_sizes(case)), dtype=dst, device="cuda")
        s["dst"] = list(s["flat"].split(_sizes(case)))
        about = math.sqrt(sum(float(t.numel()) * 100.0 ** (-1 - 2 * float(i % 7) / 7) for i, t in enumerate(s["src"])))
        s["max_norm"] = about * (0.3 if case["clipped"] else 3.0)
        if own:
            from paper_2606_10820_amd import binding as kfb
            s["plan"] = kfb.GradClip(s["src"], s["dst"])
    else:
        B, H, dh = case["B"], case["H"], case["dh"]
        rows, keys = _rows_keys(case)
        for name, n in (("q", rows), ("k", keys), ("v", keys), ("do", rows)):
            s[name] = randn(B, H, n, dh).to(torch.bfloat16)
    return s


# ------------------------------------------------------------------ the framework's calls
def _run_own(s):
    from paper_2606_10820_amd import binding as kfb
    case = s["case"]
    if case["op"] == "norm":
        y, stats = kfb.layer_norm(s["x"], s["gain"], s["shift"], eps=EPS, rms=case["rms"], out_dtype=TYPES[case["y"]])
        if case["mode"] == "forward":
            return y
        dx, dgain, dshift = kfb.layer_norm_backward(s["dy"], s["x"], s["gain"], stats, rms=case["rms"], dres=s["dres"])
        return [y, dx, dgain] if case["rms"] else [y, dx, dgain, dshift]
    if case["op"] == "logprobs":
        if case["mode"] == "score":
            r = kfb.token_logprobs(s["logits"], s["tokens"], n_top=case["top"])
            return [r.logp, r.entropy] + ([r.top_ids, r.top_logp] if case["top"] else [])
        d_logits, r = kfb.token_logprobs_backward(s["logits"], s["tokens"], s["d_logp"], s["d_entropy"])
        return [r.logp, d_logits]
    if case["op"] == "clip":
        return [s["plan"].clip(s["max_norm"]), s["flat"]]
    mask = kfb.KF_MASK_SINGLE if case["mask"] == "single" else kfb.KF_MASK_DOUBLE
    o, lse = kfb.training_attention_lse(mask, s["q"], s["k"], s["v"], case["N"], case["k"])
    dq, dk, dv = kfb.training_attention_backward(mask, s["q"], s["k"], s["v"], o, lse, s["do"], case["N"], case["k"])
    return [o, dq, dk, dv]


# ------------------------------------------------------------------ the plain forms
def _norm_plain(s):
    case = s["case"]
    xt, yt = TYPES[case["x"]], TYPES[case["y"]]
    x = s["x"].float()
    xc = x if case["rms"] else x - x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((xc * xc).mean(-1, keepdim=True) + EPS)
    xhat = xc * rstd
    y = xhat * s["gain"] if case["rms"] else xhat * s["gain"] + s["shift"]
    y = y.to(yt)
    if case["mode"] == "forward":
        return y
    dy = s["dy"].float()
    w = dy * s["gain"]
    dx = w - xhat * (w * xhat).mean(-1, keepdim=True)
    if not case["rms"]:
        dx = dx - w.mean(-1, keepdim=True)
    dx = (dx * rstd + s["dres"].float()).to(xt)
    out = [y, dx, (dy * xhat).sum(0)]
    return out if case["rms"] else out + [dy.sum(0)]


def _logprobs_plain(s):
    case = s["case"]
    x = s["logits"].float()
    m = x.max(-1, keepdim=True).values
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    lse = m + torch.log(z)
    tok = s["tokens"].long()
    given = tok >= 0
    at = tok.clamp(min=0)[:, None]
    logp = torch.where(given, x.gather(1, at)[:, 0] - lse[:, 0], torch.zeros_like(lse[:, 0]))
    if case["mode"] == "score":
        p = e / z
        entropy = -torch.where(p > 0, p * (x - lse), torch.zeros_like(p)).sum(-1)
        if not case["top"]:
            return [logp, entropy]
        # the largest values, equal ones by the lowest id: one whole number orders both
        b = (x + 0.0).view(torch.int32)
        order = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long()
        V = case["V"]
        key = order * (1 << 32) + (V - 1 - torch.arange(V, device=x.device))
        ids = (V - 1 - (key.topk(case["top"], dim=-1).values & 0xFFFFFFFF))
        return [logp, entropy, ids.int(), x.gather(1, ids) - lse]
    p = e / z
    u = torch.where(given, s["d_logp"], torch.zeros_like(s["d_logp"]))[:, None]
    d = -p * u
    if case["entropy"]:
        lp = x - lse
        h = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1, keepdim=True)
        d = d - torch.where(p > 0, p * (lp + h), torch.zeros_like(p)) * s["d_entropy"][:, None]
    d.scatter_add_(1, at, u)
    return [logp, d.to(s["logits"].dtype)]


def _clip_plain(s):
    total = torch.stack([(t.float() * t.float()).sum() for t in s["src"]]).sum()
    norm = torch.sqrt(total)
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    for a, b in zip(s["src"], s["dst"]):
        b.copy_(a.float() * scale)
    return [norm, s["flat"]]


def _visible(case):
    """The mask of one head, rows x keys."""
    N, k = case["N"], case["k"]
    rows, keys = _rows_keys(case)
    r = torch.arange(rows, device="cuda")[:, None]
    c = torch.arange(keys, device="cuda")[None, :]
    nk = N * k
    if case["mask"] == "single":
        noise, rq = r >= N, (r - N).clamp(min=0)
        group = torch.where(noise, rq // k, r)
        kq = (c - N).clamp(min=0)
        inside = noise & (c >= N) & (kq // k == rq // k) & (kq <= rq)
        return ((c < N) & (c <= group)) | inside
    second, rq = r >= nk, r % nk
    kq = (c - N).clamp(min=0) % nk
    f1 = (c >= N) & (c < N + nk) & (kq // k == rq // k) & (second | (kq <= rq))
    f2 = second & (c >= N + nk) & (kq // k == rq // k) & (kq <= rq)
    return ((c < N) & (c <= rq // k)) | f1 | f2


def _attention_plain(s):
    case = s["case"]
    B, H, dh = case["B"], case["H"], case["dh"]
    rows, keys = _rows_keys(case)
    hidden = ~_visible(case)
    scale = dh ** -0.5
    out = [torch.empty_like(s["q"]), torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])]
    flat = [t.view(B * H, -1, dh) for t in (s["q"], s["k"], s["v"], s["do"])]
    to = [t.view(B * H, -1, dh) for t in out]
    step = max(1, 400_000_000 // (rows * keys))  # heads at a time: a few GB of scores
    for i in range(0, B * H, step):
        q, k, v, do = (t[i:i + step].float() for t in flat)
        a = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
        a.masked_fill_(hidden, -math.inf)
        a = torch.exp(a - a.max(-1, keepdim=True).values)
        p = a / a.sum(-1, keepdim=True)
        dp = torch.bmm(do, v.transpose(1, 2).contiguous())
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        to[0][i:i + step] = torch.bmm(p, v)
        to[1][i:i + step] = torch.bmm(ds, k)
        to[2][i:i + step] = torch.bmm(ds.transpose(1, 2).contiguous(), q)
        to[3][i:i + step] = torch.bmm(p.transpose(1, 2).contiguous(), do)
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _norm_plain, "logprobs": _logprobs_plain, "clip": _clip_plain, "attention": _attention_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------ the definition in 64 bits
def _norm_exact(s):
    case = s["case"]
    step = case["mode"] == "step"
    x = s["x"].double().requires_grad_(step)
    gain = s["gain"].double().requires_grad_(step)
    shift = torch.zeros_like(gain) if case["rms"] else s["shift"].double()
    shift.requires_grad_(step)
    if case["rms"]:
        y = x / ((x ** 2).sum(1, keepdim=True) / case["d"] + EPS) ** 0.5 * gain
    else:
        mu = x.sum(1, keepdim=True) / case["d"]
        var = ((x - mu) ** 2).sum(1, keepdim=True) / case["d"]
        y = (x - mu) / (var + EPS) ** 0.5 * gain + shift
    if not step:
        return y
    dx, dg, db = torch.autograd.grad(y, [x, gain, shift] if not case["rms"] else [x, gain, gain], s["dy"].double())
    out = [y.detach(), dx + s["dres"].double(), dg]
    return out if case["rms"] else out + [db]


def _logprobs_exact(s):
    case = s["case"]
    parts = []
    rows, V = case["rows"], case["V"]
    size = max(1, 100_000_000 // V)
    for i in range(0, rows, size):
        x = s["logits"][i:i + size].double()
        tok = s["tokens"][i:i + size].long()
        if case["mode"] == "score":
            lp = x - torch.logsumexp(x, 1, keepdim=True)
            logp = torch.stack([lp[torch.arange(len(tok), device="cuda"), tok.clamp(min=0)], torch.zeros(len(tok), device="cuda", dtype=torch.float64)])[(tok < 0).long(), torch.arange(len(tok), device="cuda")]
            q = lp.exp()
            h = -(q * lp.nan_to_num(neginf=0.0)).sum(1)
            part = [logp, h]
            if case["top"]:
                v, ids = torch.sort(x, dim=1, descending=True, stable=True)
                part += [ids[:, :case["top"]].int(), lp.gather(1, ids[:, :case["top"]])]
        else:
            x.requires_grad_(True)
            lp = torch.log_softmax(x, 1)
            logp = lp.gather(1, tok.clamp(min=0)[:, None])[:, 0] * (tok >= 0)
            total = (logp * s["d_logp"][i:i + size].double()).sum()
            if case["entropy"]:
                total = total - ((lp.exp() * lp).sum(1) * s["d_entropy"][i:i + size].double()).sum()
            part = [logp.detach(), torch.autograd.grad(total, x)[0]]
        parts.append(part)
    return [torch.cat(p) for p in zip(*parts)]


def _clip_exact(s):
    norm = sum(float((t.double() ** 2).sum()) for t in s["src"]) ** 0.5
    scale = min(1.0, s["max_norm"] / norm)
    return [torch.tensor(norm, dtype=torch.float64, device="cuda"), torch.cat([t.double() * scale for t in s["src"]])]


def _attention_exact(s):
    case = s["case"]
    B, H, dh, N, k = case["B"], case["H"], case["dh"], case["N"], case["k"]
    rows, keys = _rows_keys(case)
    # the mask from the last visible context key of each row and its group's rows
    see = torch.zeros(rows, keys, dtype=torch.bool, device="cuda")
    row = torch.arange(rows, device="cuda")
    if case["mask"] == "single":
        last = torch.where(row < N, row, (row - N) // k)
        blocks = [(N, N, True)]
    else:
        last = (row % (N * k)) // k
        blocks = [(0, N, True), (N * k, N, False), (N * k, N + N * k, True)]
    see[:, :N] = torch.arange(N, device="cuda") <= last[:, None]
    group = torch.arange(N, device="cuda").repeat_interleave(k * k) * k
    i = torch.arange(k, device="cuda").repeat_interleave(k).repeat(N)
    j = torch.arange(k, device="cuda").repeat(k).repeat(N)
    for r0, c0, causal in blocks:
        keep = i >= j if causal else i >= 0
        see[(r0 + group + i)[keep], (c0 + group + j)[keep]] = True
    out = [torch.empty(B, H, n, dh, dtype=torch.float64, device="cuda") for n in (rows, rows, keys, keys)]
    for b in range(B):
        for h in range(H):
            q, kk, v = (s[n][b, h].double().requires_grad_(True) for n in "qkv")
            a = torch.where(see, q @ kk.t() / dh ** 0.5, -math.inf)
            o = torch.softmax(a, 1) @ v
            grads = torch.autograd.grad(o, [q, kk, v], s["do"][b, h].double())
            for t, x in zip(out, [o.detach(), *grads]):
                t[b, h] = x
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "logprobs": _logprobs_exact, "clip": _clip_exact, "attention": _attention_exact}[case["op"]](s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        n, bx, by = case["rows"] * case["d"], BYTES[case["x"]], BYTES[case["y"]]
        if case["mode"] == "forward":
            return dict(bytes=n * (bx + by) + 8 * case["d"], flops=8 * n)
        return dict(bytes=n * (3 * bx + 2 * by) + 16 * case["d"], flops=22 * n)
    if case["op"] == "logprobs":
        n, b = case["rows"] * case["V"], BYTES[case["dtype"]]
        if case["mode"] == "score":
            return dict(bytes=n * b + case["rows"] * (12 + 8 * case["top"]), flops=6 * n)
        return dict(bytes=2 * n * b + case["rows"] * (12 + 4 * case["entropy"]), flops=(12 if case["entropy"] else 8) * n)
    if case["op"] == "clip":
        n = sum(_sizes(case))
        return dict(bytes=n * (BYTES[case["src"]] + BYTES[case["dst"]]), flops=3 * n)
    rows, keys = _rows_keys(case)
    heads, dh = case["B"] * case["H"], case["dh"]
    return dict(bytes=heads * dh * 2 * (4 * rows + 4 * keys), flops=heads * 14 * dh * _entries(case))
