"""GPU parity of a QKV product's heads (norms, rotary positions, attention's layout) and their
gradients against 64-bit references (bounds: tests/step_ref.py)."""
import pytest

from tests import step_ref as S
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (F32, BF), (F32, HF), (BF, BF), (HF, HF)]
IDS = lambda v: str(v).replace("torch.", "")
EPS = 1e-5


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _inputs(B, L, Hq, Hkv, dh, rot, xt, yt, seed=0, n_pos=0, norm=(True, True)):
    g = torch.Generator().manual_seed(seed + 1000 * L + dh)
    rnd = lambda *s: torch.randn(*s, generator=g)
    x = (rnd(B, L, (Hq + 2 * Hkv) * dh) * (0.3 + 2 * torch.rand((Hq + 2 * Hkv) * dh, generator=g))).to(xt)
    table = None
    if rot:
        a = torch.arange(n_pos or L, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        table = torch.stack([torch.cos(a), torch.sin(a)], -1).float().contiguous()
    gains = [1 + 0.3 * rnd(dh) if n else None for n in norm]
    grads = [rnd(B, H, L, dh).to(yt) for H in (Hq, Hkv, Hkv)]
    return x, table, gains, grads


def _both(Bd, x, Hq, Hkv, dh, table, pos, gains, grads, yt, where=""):
    dev = lambda t: t if t is None or t.is_cuda else t.cuda()
    X, T, P, (gq, gk), G = dev(x), dev(table), dev(pos), [dev(g) for g in gains], [dev(g) for g in grads]
    out = Bd.qkv_heads(X, Hq, Hkv, T, P, gq, gk, EPS, yt)
    dx, dgq, dgk = Bd.qkv_heads_backward(*G, X, T, P, gq, gk, EPS)
    torch.cuda.synchronize()
    x, pos, grads = X.cpu(), None if P is None else P.cpu(), [g.cpu() for g in G]
    ref = S.heads(x, Hq, Hkv, dh, table, pos, *gains, EPS, yt)
    (rdx, bdx), rgq, rgk = S.heads_grad(*grads, x, Hq, Hkv, dh, table, pos, *gains, EPS, x.dtype)
    got = {n: R.worst(o, *r) for n, o, r in zip("qkv", out, ref)}
    got["dx"] = R.worst(dx, rdx, bdx)
    for n, d, r in (("dgq", dgq, rgq), ("dgk", dgk, rgk)):
        assert (d is None) == (r is None)
        if r is not None:
            got[n] = R.worst(d, *r)
    print(where, tuple(x.shape), Hq, Hkv, {k: round(v, 3) for k, v in got.items()}, flush=True)
    assert all(v <= 1.0 for v in got.values()), got
    return out, dx, dgq, dgk


SHAPES = [  # B, L, Hq, Hkv, dh, rot
    (1, 1, 1, 1, 1, 0), (1, 1, 12, 12, 64, 64), (2, 3, 4, 4, 32, 32), (1, 7, 3, 1, 2, 2), (3, 5, 2, 2, 7, 4), (2, 8, 12, 12, 64, 64),
    (2, 9, 16, 4, 96, 48), (1, 17, 5, 5, 128, 64), (2, 33, 3, 2, 80, 20), (1, 5, 2, 1, 256, 64), (1, 4, 1, 1, 512, 512), (2, 3, 2, 2, 509, 6),
    (1, 65, 50, 50, 8, 8), (1, 3, 400, 8, 16, 10), (5, 129, 2, 2, 72, 70), (1, 9, 0, 3, 40, 8), (1, 9, 3, 0, 40, 8), (2, 6, 1, 1, 24, 0)]


@pytest.mark.parametrize("pair", PAIRS, ids=lambda p: f"{IDS(p[0])}-{IDS(p[1])}")
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_parity(Bd, shape, pair):
    B, L, Hq, Hkv, dh, rot = shape
    for norm in ((True, True), (False, False), (False, True), (True, False)):
        x, table, gains, grads = _inputs(*shape, *pair, seed=PAIRS.index(pair), norm=norm)
        _both(Bd, x, Hq, Hkv, dh, table, None, gains, grads, pair[1], str(norm))


@pytest.mark.parametrize("L", [1, 3, 4, 5, 255, 1023, 4099])
def test_lengths(Bd, L):
    """More tokens than workgroups with sums, ragged ends of theirs."""
    x, table, gains, grads = _inputs(3, L, 2, 1, 32, 32, F32, BF)
    _both(Bd, x, 2, 1, 32, table, None, gains, grads, BF)


def test_positions(Bd):
    """One list for all sequences (the SingleForward layout), one for each, and positions outside the
    table, which give NaN in the turned columns of that row alone."""
    B, L, H, dh, rot = 3, 20, 2, 64, 32
    x, table, gains, grads = _inputs(B, L, H, H, dh, rot, BF, BF, n_pos=100)
    N, k = 4, 4
    t = torch.arange(N)
    single = torch.cat([t, (t[:, None] + 1 + torch.arange(k)).reshape(-1)]).int()
    _both(Bd, x, H, H, dh, table, single, gains, grads, BF, "shared")
    each = (torch.arange(L) + torch.tensor([0, 40, 80])[:, None]).int()
    _both(Bd, x, H, H, dh, table, each, gains, grads, BF, "each")
    bad = each.clone()
    bad[1, 3], bad[2, 19], bad[0, 0] = -1, 100, 2 ** 31 - 1
    off = [None, None]
    (q, _, v), dx, _, _ = _both(Bd, x, H, H, dh, table, bad, off, grads, BF, "outside")
    assert torch.isnan(q[1, :, 3, :rot]).all() and not torch.isnan(q[1, :, 3, rot:]).any() and not torch.isnan(v).any()
    assert int(torch.isnan(q).sum()) == 3 * H * rot


@pytest.mark.parametrize("off,ld", [(0, 8), (1, 0), (3, 5), (4, 4), (8, 16)])
@pytest.mark.parametrize("pair", [PAIRS[1], PAIRS[3]], ids=["fp32-bf16", "bf16-bf16"])
def test_strides_and_alignment(Bd, pair, off, ld):
    """Rows apart and misaligned, results into views of larger tensors, gradients from such views:
    what lies between is not read (NaN there) and not written."""
    B, L, Hq, Hkv, dh = 2, 5, 3, 2, 64
    x, table, gains, grads = _inputs(B, L, Hq, Hkv, dh, 64, *pair)
    W = x.shape[2] + ld

    def strided(t, fill):
        buf = torch.full((off + B * L * W,), fill, dtype=t.dtype, device="cuda")
        v = buf[off:].view(B, L, W)[..., :t.shape[2]]
        v.copy_(t)
        return buf, v

    def view(t, fill):
        H = t.shape[1]
        buf = torch.full((off + B * H * (L + 3) * (dh + ld),), fill, dtype=t.dtype, device="cuda")
        v = buf[off:].view(B, H, L + 3, dh + ld)[:, :, 2:2 + L, :dh]
        v.copy_(t)
        return buf, v
    nan = float("nan")
    _, X = strided(x, nan)
    G = [view(g, nan)[1] for g in grads]
    want, dx, dgq, dgk = _both(Bd, X, Hq, Hkv, dh, table, None, gains, G, pair[1], f"ld {ld} off {off}")
    outs = [view(torch.zeros_like(g, dtype=pair[1]), 7.0) for g in grads]
    gq, gk = (g.cuda() for g in gains)
    got = Bd.qkv_heads(X, Hq, Hkv, table.cuda(), None, gq, gk, EPS, out=[v for _, v in outs])
    dbuf, D = strided(torch.zeros_like(x), 7.0)
    Bd.qkv_heads_backward(*G, X, table.cuda(), None, gq, gk, EPS, out=D)
    torch.cuda.synchronize()
    for (buf, v), w, g in zip(outs, want, got):
        assert g is v and torch.equal(v, w)
        v.fill_(7.0)
        assert (buf == 7).all()
    assert torch.equal(D, dx)
    D.fill_(7.0)
    assert (dbuf == 7).all()


def test_unwanted_expanded_and_in_place(Bd):
    """Results that are not wanted, gradients that are one row or head expanded, dqkv over qkv."""
    B, L, H, dh = 2, 11, 4, 32
    x, table, gains, grads = _inputs(B, L, H, H, dh, 32, BF, BF)
    X, T, (gq, gk) = x.cuda(), table.cuda(), [g.cuda() for g in gains]
    q, k, v = Bd.qkv_heads(X, H, None, T, None, gq, gk)
    only = torch.zeros_like(k)
    r = Bd.qkv_heads(X, H, None, T, None, gq, gk, out=(None, only, None))
    assert r[0] is None and r[2] is None and torch.equal(only, k)
    G = [g.cuda() for g in grads]
    wide = G[0][:, :1, :1].expand(B, H, L, dh)
    a = Bd.qkv_heads_backward(wide, G[1], G[2], X, T, None, gq, gk)
    b = Bd.qkv_heads_backward(wide.contiguous(), G[1], G[2], X, T, None, gq, gk)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    Y = X.clone()
    c = Bd.qkv_heads_backward(*G, Y, T, None, gq, gk, out=Y)
    d = Bd.qkv_heads_backward(*G, X, T, None, gq, gk)
    assert c[0] is Y and all(torch.equal(s, t) for s, t in zip(c, d))
    # without gains the product is not needed
    e = Bd.qkv_heads_backward(*G, X, T)
    f = Bd.qkv_heads_backward(*G, None, T)
    assert torch.equal(e[0], f[0]) and e[1] is e[2] is None
    w = Bd.qkv_heads_backward(*G, None, T, out_dtype=F32)[0]
    assert w.dtype == F32 and torch.equal(w.to(BF), e[0])


def test_empty(Bd):
    g = torch.ones(32, device="cuda")
    for B, L in ((0, 5), (3, 0)):
        x = torch.zeros(B, L, 6 * 32, device="cuda")
        q, k, v = Bd.qkv_heads(x, 2, q_gain=g, k_gain=g)
        assert q.shape == (B, 2, L, 32)
        dx, a, b = Bd.qkv_heads_backward(q, k, v, x, q_gain=g, k_gain=g)
        assert dx.shape == x.shape and not a.any() and not b.any()


def test_zero_rows_and_infinities(Bd):
    """A head of zeros is zero after its norm (eps); a NaN or infinity stays within its head."""
    B, L, H, dh = 1, 6, 3, 64
    x, table, gains, grads = _inputs(B, L, H, H, dh, 64, F32, F32)
    h = x.view(B, L, 3 * H, dh)
    h[0, 0, 0] = 0
    h[0, 1, 1, 5] = float("nan")
    h[0, 2, 4, 7] = float("inf")
    X = x.cuda()
    q, k, v = Bd.qkv_heads(X, H, None, table.cuda(), None, *(g.cuda() for g in gains))
    dx, _, _ = Bd.qkv_heads_backward(*(g.cuda() for g in grads), X, table.cuda(), None, *(g.cuda() for g in gains))
    assert not q[0, 0, 0].any()
    bad = torch.zeros(B, L, 3 * H, dtype=torch.bool)
    bad[0, 1, 1] = bad[0, 2, 4] = True
    assert torch.equal(torch.isnan(dx.cpu().view(B, L, 3 * H, dh)).any(-1), bad)
    assert torch.isnan(q[0, 1, 1]).all() and int(torch.isnan(q).any(-1).sum()) == 1
    assert torch.isnan(k[0, 1, 2]).any() and int(torch.isnan(k).any(-1).sum()) == 1 and torch.isfinite(v).all()


def test_repeats_are_equal(Bd):
    x, table, gains, grads = _inputs(4, 700, 4, 2, 64, 64, BF, BF)
    run = lambda: Bd.qkv_heads_backward(*(g.cuda() for g in grads), x.cuda(), table.cuda(), None, *(g.cuda() for g in gains))
    a = run()
    for _ in range(3):
        assert all(torch.equal(s, t) for s, t in zip(a, run()))


def test_past_32_bits(Bd):
    """Offsets past 2^31 elements: the last rows of a product of 2.2e9 elements."""
    Hq, Hkv, dh, L = 18, 16, 64, 690_000
    W = (Hq + 2 * Hkv) * dh
    assert L * W > 2 ** 31
    x = torch.empty(1, L, W, dtype=BF, device="cuda")
    x.normal_()
    table = Bd.rope_table(L, 64)
    g = torch.ones(dh, device="cuda")
    q, k, v = Bd.qkv_heads(x, Hq, Hkv, table, None, g, g)
    dx, _, _ = Bd.qkv_heads_backward(q, k, v, x, table, None, g, g)
    tail = slice(L - 3, L)
    pos = torch.arange(L - 3, L, dtype=torch.int32)
    ref = S.heads(x[:, tail].cpu(), Hq, Hkv, dh, table.cpu(), pos, g.cpu(), g.cpu(), EPS, BF)
    for o, r in zip((q, k, v), ref):
        assert R.worst(o[:, :, tail], *r) <= 1
    (rdx, b), _, _ = S.heads_grad(q[:, :, tail].cpu(), k[:, :, tail].cpu(), v[:, :, tail].cpu(), x[:, tail].cpu(), Hq, Hkv, dh, table.cpu(), pos,
                                  g.cpu(), g.cpu(), EPS, BF)
    assert R.worst(dx[:, tail], rdx, b) <= 1


@pytest.mark.parametrize("n,rot,base", [(1, 2, 10000.0), (1024, 64, 10000.0), (70001, 32, 10000.0), (300, 512, 500000.0)])
def test_rope_table(Bd, n, rot, base):
    """Angles in fp64 (off by 3 of its roundings of the angle, 1e-11 at position 70000), one rounding to
    fp32."""
    t = Bd.rope_table(n, rot, base).cpu().double()
    a = torch.arange(n, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    assert t.shape == (n, rot // 2, 2)
    for got, want in ((t[..., 0], torch.cos(a)), (t[..., 1], torch.sin(a))):
        assert bool(((got - want).abs() <= R.U * want.abs() + 1e-10).all())


@pytest.mark.parametrize("L", [1, 2, 5, 40])
@pytest.mark.parametrize("Hq,Hkv", [(2, 0), (0, 2), (1, 1), (12, 3)])
def test_few_rows_and_single_gains(Bd, L, Hq, Hkv):
    """One workgroup's sums are written without a second launch, several are joined; a gain that has no
    heads has gradient 0; either gradient alone."""
    for dh in (64, 7):
        for norm in ((True, True), (True, False), (False, True)):
            x, table, gains, grads = _inputs(1, L, Hq, Hkv, dh, 4, BF, BF, norm=norm)
            _, _, dgq, dgk = _both(Bd, x, Hq, Hkv, dh, table, None, gains, grads, BF, str(norm))
            assert dgq is None or Hq or not dgq.any()
            assert dgk is None or Hkv or not dgk.any()


def test_double_mask_layout(Bd):
    """The DoubleForward mask's keys, [context | Future-1 | Future-2], from two products straight into the
    regions of one tensor, and their gradients back out of it."""
    B, N, K, H, dh = 2, 5, 3, 2, 32
    rows = 2 * N * K
    g = torch.Generator().manual_seed(0)
    ctx, fut = (torch.randn(B, n, 3 * H * dh, generator=g).to(BF).cuda() for n in (N, rows))
    t = torch.arange(N)[:, None] + 1 + torch.arange(K)
    pos = torch.cat([t.reshape(-1), (t + K).reshape(-1)]).int().cuda()
    table = Bd.rope_table(N + 2 * K, dh)
    gain = torch.full((dh,), 1.1, device="cuda")
    k, v = (torch.empty(B, H, N + rows, dh, dtype=BF, device="cuda") for _ in range(2))
    q = torch.empty(B, H, rows, dh, dtype=BF, device="cuda")
    args = (table, None, gain, gain)
    Bd.qkv_heads(ctx, H, None, *args, out=(None, k[:, :, :N], v[:, :, :N]))
    Bd.qkv_heads(fut, H, None, table, pos, gain, gain, out=(q, k[:, :, N:], v[:, :, N:]))
    a, b = Bd.qkv_heads(ctx, H, None, *args), Bd.qkv_heads(fut, H, None, table, pos, gain, gain)
    assert torch.equal(q, b[0]) and torch.equal(k, torch.cat([a[1], b[1]], 2)) and torch.equal(v, torch.cat([a[2], b[2]], 2))
    o, lse = Bd.training_attention_lse(Bd.KF_MASK_DOUBLE, q, k, v, N, K)
    dq, dk, dv = Bd.training_attention_backward(Bd.KF_MASK_DOUBLE, q, k, v, o, lse, o, N, K)
    got = Bd.qkv_heads_backward(dq, dk[:, :, N:], dv[:, :, N:], fut, table, pos, gain, gain)
    want = Bd.qkv_heads_backward(dq, dk[:, :, N:].contiguous(), dv[:, :, N:].contiguous(), fut, table, pos, gain, gain)
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    zero = torch.zeros(B, H, 1, 1, dtype=BF, device="cuda").expand(B, H, N, dh)
    with pytest.raises(ValueError):  # a head's columns are consecutive
        Bd.qkv_heads_backward(zero, dk[:, :, :N], dv[:, :, :N], ctx, *args)
    zero = torch.zeros(1, 1, 1, dh, dtype=BF, device="cuda").expand(B, H, N, dh)
    d, _, dgk = Bd.qkv_heads_backward(zero, dk[:, :, :N], dv[:, :, :N], ctx, *args)
    assert not d[..., :H * dh].any() and d[..., H * dh:].any() and dgk.any()
