"""Argument checks of heads, dropout and the policy loss (no GPU: every call here is refused before
a launch, or is an empty problem), the generator against published vectors, and the 64-bit
references against differences."""
import ctypes
import math
import os

import numpy as np
import pytest

from paper_2606_10820_amd import binding as Bd
from tests import step_ref as S
from tests import train_ref as R

torch = pytest.importorskip("torch")
P = ctypes.c_void_p
A = P(0x10000)  # 256-byte aligned, never dereferenced
NAN, INF = float("nan"), float("inf")
GOLDEN = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")


@pytest.fixture(scope="module")
def L():
    return Bd.lib()


def _h(ptr=0x100000, batch=640, head=64, row=8):
    return Bd.KfHeads(ptr, batch, head, row)


HEADS = dict(xt=0, yt=0, B=2, L=8, Hq=10, Hkv=2, dh=8, x=A, ldx=112, gq=A, gk=A, eps=1e-5, tab=A, n_pos=8, rot=8, pos=A, pos_ld=0)
BAD_HEADS = (dict(xt=3), dict(xt=1, yt=0), dict(xt=1, yt=2), dict(B=-1), dict(L=-1), dict(B=1 << 16, L=(1 << 14) + 1), dict(Hq=-1), dict(Hkv=-1),
             dict(Hq=0, Hkv=0), dict(Hq=65537), dict(Hkv=40000), dict(dh=0), dict(dh=513), dict(rot=7), dict(rot=10), dict(rot=-2), dict(eps=-1.0), dict(eps=NAN),
             dict(eps=INF), dict(ldx=111), dict(gq=P(0x10001)), dict(gk=P(0x10002)), dict(tab=None), dict(tab=P(0x10004)), dict(n_pos=0), dict(n_pos=-4),
             dict(pos=P(0x10002)), dict(pos_ld=-1), dict(pos_ld=7), dict(pos_ld=1 << 60))


def test_heads_refusals(L):
    def call(q=None, k=None, v=None, **kw):
        a = dict(HEADS, **kw)
        q, k, v = q or _h(), k or _h(0x200000, 128), v or _h(0x300000, 128)
        return L.kf_qkv_heads(None, a["xt"], a["yt"], a["B"], a["L"], a["Hq"], a["Hkv"], a["dh"], a["x"], a["ldx"], a["gq"], a["gk"], a["eps"],
                              a["tab"], a["n_pos"], a["rot"], a["pos"], a["pos_ld"], q, k, v)

    for bad in BAD_HEADS + (dict(x=None), dict(x=P(0x10002))):
        assert call(**bad) == Bd.KF_EINVAL, bad
    for q in (_h(0x100002), _h(batch=-1), _h(head=-64), _h(row=-8), _h(row=7), _h(head=63), _h(batch=639), _h(0x100000, 0, 64, 8), _h(0x100000, 640, 64, 0),
              _h(0x100000, 1 << 59), _h(0x100000, 640, 8, 8), _h(0x10000), _h(0x200000), _h(0x300000)):
        assert call(q=q) == Bd.KF_EINVAL, (q.ptr, q.batch, q.head, q.row)
    assert call(k=_h(0x300000, 128)) == Bd.KF_EINVAL
    for empty in (dict(B=0), dict(L=0)):
        assert call(x=None, tab=None, **empty) == Bd.KF_OK


def test_heads_backward_refusals(L):
    def call(dq=None, dk=None, dv=None, **kw):
        a = dict(HEADS, dx=P(0x40000), lddx=112, dgq=A, dgk=P(0x11000), ws=A, n=1 << 30)
        a.update(kw)
        dq, dk, dv = dq or _h(), dk or _h(0x200000, 128), dv or _h(0x300000, 128)
        return L.kf_qkv_heads_backward(None, a["xt"], a["yt"], a["B"], a["L"], a["Hq"], a["Hkv"], a["dh"], dq, dk, dv, a["x"], a["ldx"], a["gq"], a["gk"],
                                       a["eps"], a["tab"], a["n_pos"], a["rot"], a["pos"], a["pos_ld"], a["dx"], a["lddx"], a["dgq"], a["dgk"], a["ws"], a["n"])

    need = L.kf_qkv_heads_backward_bytes(2, 8, 10, 2, 8)
    assert need > 0
    for bad in BAD_HEADS + (dict(x=None), dict(x=P(0x10002)), dict(dx=None), dict(dx=P(0x40001)), dict(lddx=111), dict(dx=A, lddx=120), dict(dx=P(0x100000)),
                            dict(dgq=P(0x10002)), dict(gq=None), dict(gk=None), dict(dgk=A), dict(ws=None), dict(ws=P(0x10008)), dict(n=need - 1)):
        assert call(**bad) == Bd.KF_EINVAL, bad
    for q in (_h(0x100002), _h(batch=-1), _h(row=-8)):
        assert call(dq=q) == Bd.KF_EINVAL
    assert L.kf_qkv_heads_backward_bytes(0, 8, 1, 1, 8) == 0 == L.kf_qkv_heads_backward_bytes(2, 8, 1, 1, 600)
    t = L.kf_rope_table
    for bad in ((0, 8, 1e4, A), (5, 7, 1e4, A), (5, 0, 1e4, A), (5, 514, 1e4, A), (5, 8, 0.0, A), (5, 8, -1.0, A), (5, 8, INF, A), (5, 8, NAN, A), (5, 8, 1e4, None),
                (5, 8, 1e4, P(0x10004))):
        assert t(None, *bad) == Bd.KF_EINVAL, bad


def test_dropout_refusals(L):
    ok = dict(xt=1, yt=0, rows=4, d=8, x=A, ldx=8, res=None, ldr=8, p=0.1, seed=1, ds=None, site=0, y=P(0x20000), ldy=8)

    def call(**kw):
        a = dict(ok, **kw)
        return L.kf_dropout(None, a["xt"], a["yt"], a["rows"], a["d"], a["x"], a["ldx"], a["res"], a["ldr"], a["p"], a["seed"], a["ds"], a["site"], a["y"], a["ldy"])

    def back(**kw):
        a = dict(ok, **kw)
        return L.kf_dropout_backward(None, a["xt"], a["yt"], a["rows"], a["d"], a["x"], a["ldx"], a["p"], a["seed"], a["ds"], a["site"], a["y"], a["ldy"])

    for f in (call, back):
        for bad in (dict(xt=3), dict(yt=-1), dict(xt=1, yt=2), dict(rows=-1), dict(d=0), dict(d=(1 << 28) + 1, ldx=1 << 29, ldy=1 << 29), dict(ldx=7), dict(ldy=7),
                    dict(p=-0.1), dict(p=1.1), dict(p=NAN), dict(site=1 << 31), dict(ds=P(0x10004)), dict(x=None), dict(y=None), dict(x=P(0x10001)),
                    dict(y=P(0x20001)), dict(y=A), dict(rows=1 << 58, ldx=1 << 10)):
            assert f(**bad) == Bd.KF_EINVAL, bad
        assert f(rows=0, x=None, y=None) == Bd.KF_OK
    for bad in (dict(res=P(0x10002)), dict(res=P(0x30000), ldr=7), dict(res=P(0x20000), ldr=9), dict(xt=0, y=A, ldy=9)):
        assert call(**bad) == Bd.KF_EINVAL, bad


def test_dropout_norm_refusals(L):
    ok = dict(norm=0, ht=0, yt=1, rows=4, d=8, x=A, ldx=8, res=P(0x20000), ldr=8, p=0.1, ds=None, site=0, g=A, b=A, eps=1e-5, h=P(0x30000), ldh=8, y=P(0x40000),
              ldy=8, st=A)

    def call(**kw):
        a = dict(ok, **kw)
        return L.kf_dropout_norm(None, a["norm"], a["ht"], a["yt"], a["rows"], a["d"], a["x"], a["ldx"], a["res"], a["ldr"], a["p"], 1, a["ds"], a["site"], a["g"],
                                 a["b"], a["eps"], a["h"], a["ldh"], a["y"], a["ldy"], a["st"])

    for bad in (dict(norm=2), dict(ht=1, yt=0), dict(ht=3), dict(rows=-1), dict(d=0), dict(ldx=7), dict(ldr=7), dict(ldh=7), dict(ldy=7), dict(p=2.0), dict(p=NAN),
                dict(site=1 << 31), dict(ds=P(0x10001)), dict(norm=1), dict(eps=-1.0), dict(eps=NAN), dict(x=None), dict(res=None), dict(h=None), dict(y=None),
                dict(g=None), dict(b=P(0x10001)), dict(st=P(0x10004)), dict(h=P(0x20000), ldh=9), dict(h=A), dict(h=P(0x40000)), dict(y=A), dict(y=P(0x20000))):
        assert call(**bad) == Bd.KF_EINVAL, bad
    assert call(rows=0, x=None, res=None, h=None, y=None, g=None, b=None, st=None) == Bd.KF_OK
    ok2 = dict(norm=0, ht=0, yt=1, rows=4, d=8, dy=A, lddy=8, h=P(0x20000), ldh=8, g=A, st=A, dres=None, ldr=8, p=0.1, site=0, dh=P(0x30000), lddh=8,
               dx=P(0x40000), lddx=8, dg=A, db=A, ws=A, n=1 << 20)

    def back(**kw):
        a = dict(ok2, **kw)
        return L.kf_dropout_norm_backward(None, a["norm"], a["ht"], a["yt"], a["rows"], a["d"], a["dy"], a["lddy"], a["h"], a["ldh"], a["g"], a["st"], a["dres"],
                                          a["ldr"], a["p"], 1, None, a["site"], a["dh"], a["lddh"], a["dx"], a["lddx"], a["dg"], a["db"], a["ws"], a["n"])

    need = L.kf_layer_norm_backward_bytes(4, 8)
    for bad in (dict(norm=5), dict(yt=4), dict(rows=-1), dict(d=0), dict(lddy=7), dict(ldh=7), dict(lddh=7), dict(lddx=7), dict(dres=A, ldr=7), dict(p=-1.0),
                dict(site=1 << 31), dict(norm=1), dict(dy=None), dict(h=None), dict(dh=None), dict(dx=None), dict(g=None), dict(st=None), dict(st=P(0x10004)),
                dict(dres=P(0x10002)), dict(dh=P(0x20000)), dict(dh=A), dict(dh=P(0x40000)), dict(dx=A), dict(dx=P(0x20000)), dict(dres=P(0x30000), ldr=9),
                dict(dres=P(0x40000)), dict(ws=None), dict(ws=P(0x10004)), dict(n=need - 1), dict(dg=P(0x10001)), dict(db=P(0x10001))):
        assert back(**bad) == Bd.KF_EINVAL, bad


def test_policy_refusals(L):
    ok = dict(t=1, rows=3, V=100, x=A, ld=100, tok=A, adv=A, old=A, ref=A, w=A, lo=0.8, hi=1.2, beta=0.1, c=0.1, rl=A, lp=A, ra=A, kl=A, h=A, loss=A,
              d=P(0x40000), ldd=100)

    def call(**kw):
        a = dict(ok, **kw)
        return L.kf_policy_loss(None, a["t"], a["rows"], a["V"], a["x"], a["ld"], a["tok"], a["adv"], a["old"], a["ref"], a["w"], a["lo"], a["hi"], a["beta"], a["c"],
                                a["rl"], a["lp"], a["ra"], a["kl"], a["h"], a["loss"], a["d"], a["ldd"])

    for bad in (dict(t=3), dict(rows=-1), dict(V=0), dict(V=(1 << 28) + 1, ld=1 << 29, ldd=1 << 29), dict(ld=99), dict(ldd=99), dict(lo=-0.1), dict(lo=1.1), dict(hi=0.9),
                dict(lo=NAN), dict(hi=NAN), dict(beta=NAN), dict(beta=INF), dict(c=INF), dict(c=1e30), dict(x=None), dict(tok=None), dict(adv=None), dict(rl=None),
                dict(ref=None), dict(ref=None, kl=None), dict(ref=None, beta=0.0), dict(x=P(0x10001)), dict(tok=P(0x10002)), dict(adv=P(0x10001)), dict(old=P(0x10002)),
                dict(ref=P(0x10001)), dict(w=P(0x10001)), dict(rl=P(0x10001)), dict(lp=P(0x10001)), dict(ra=P(0x10002)), dict(kl=P(0x10001)), dict(h=P(0x10001)),
                dict(loss=P(0x10001)), dict(d=P(0x40001)), dict(d=A, ldd=101), dict(rows=1 << 57)):
        assert call(**bad) == Bd.KF_EINVAL, bad
    assert call(rows=0, x=None, tok=None, adv=None, rl=None, loss=None, d=None) == Bd.KF_OK


def test_binding_refuses_host_tensors_and_bad_shapes():
    x, g = torch.zeros(2, 4, 48), torch.ones(8)
    i64 = torch.zeros(2, 4, dtype=torch.int64)
    for call in (lambda: Bd.qkv_heads(x, 2, 2), lambda: Bd.qkv_heads(x[0], 2, 2), lambda: Bd.qkv_heads(x, 5), lambda: Bd.qkv_heads(x, 2, 2, q_gain=torch.ones(7)),
                 lambda: Bd.qkv_heads(x, 2, 2, table=g), lambda: Bd.qkv_heads(x, 2, 2, positions=i64), lambda: Bd.qkv_heads(x, 2, 2, positions=i64[0, :3].int()),
                 lambda: Bd.qkv_heads(x.transpose(0, 1), 2, 2), lambda: Bd.qkv_heads_backward(x, x, x), lambda: Bd.rope_table(4, 7, device="cpu"),
                 lambda: Bd.rope_table(4, 8, device="cpu"), lambda: Bd.dropout(x, 0.1, 1), lambda: Bd.dropout(x, 0.1, 1, residual=x[0]),
                 lambda: Bd.dropout(x, 0.1, torch.zeros(2, dtype=torch.int64)), lambda: Bd.dropout(x, 0.1, torch.zeros(1)), lambda: Bd.dropout(x.transpose(0, 1), 0.1, 1),
                 lambda: Bd.dropout(x, 0.1, 1, residual=x.bfloat16(), out_dtype=torch.float32), lambda: Bd.dropout_norm(x[0], x[0], g), lambda: Bd.dropout_norm(x, x[0], g),
                 lambda: Bd.dropout_norm_backward(x[0], x, g, g), lambda: Bd.policy_loss(x, i64, g), lambda: Bd.policy_loss(x, i64.int(), g[:7]),
                 lambda: Bd.policy_loss(x, None, g), lambda: Bd.policy_loss(x, i64.int(), g, weights=torch.ones(7)),
                 lambda: Bd.policy_loss(x, i64.int(), g, grad=False, out=x), lambda: Bd.qkv_heads_backward(*[torch.zeros(1, 2, 3, 8)] * 3, q_gain=g)):
        with pytest.raises(ValueError):
            call()


def test_binding_refuses_what_32_bits_do_not_hold():
    """Sizes that the C entries take as 32 bits (tensors without memory)."""
    big = lambda *s: torch.empty(*s, device="meta", dtype=torch.bfloat16)
    for call in (lambda: Bd.dropout(big(2 ** 32 + 100), 0.1, 1), lambda: Bd.dropout(big(3, 2 ** 31), 0.1, 1), lambda: Bd.qkv_heads(big(1, 2 ** 32 + 8, 3), 1),
                 lambda: Bd.qkv_heads(big(2 ** 16, 2 ** 14 + 1, 3), 1), lambda: Bd.qkv_heads_backward(*[big(1, 1, 2 ** 32 + 8, 1)] * 3),
                 lambda: Bd.qkv_heads(big(1, 8, 6), 1, table=torch.empty(2 ** 32 + 8, 1, 2, device="meta")), lambda: Bd.rope_table(2 ** 32 + 8, 2, device="meta"),
                 lambda: Bd.policy_loss(big(1, 2 ** 32 + 8), torch.zeros(1, dtype=torch.int32), torch.zeros(1)), lambda: Bd.layer_norm(big(2 ** 32 + 8), big(1)),
                 lambda: Bd.dropout(big(4, 8), 0.1, 1, site=2 ** 31), lambda: Bd.dropout(big(4, 8), 0.1, 1, site=-1), lambda: Bd.dropout(big(4, 8), 0.1, 1, site=2 ** 32 + 1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        Bd.dropout(big(4, 8), 0.1, 1.5)
    assert Bd._seed(np.int64(-1), 0, None) == Bd._seed(-1, 0, None) == (2 ** 64 - 1, None)


def test_philox_against_published_vectors():
    n = 0
    for line in open(GOLDEN):
        if line.strip() and not line.startswith("#"):
            v = [int(t, 16) for t in line.split() if all(ch in "0123456789abcdefABCDEF" for ch in t)]
            c, k, want = v[:4], v[4:6], v[6:10]
            assert [int(t) for t in S.philox(c, k)] == want
            n += 1
    assert n >= 3


# ------------------------------- the references' gradients against differences
def _directional(f, args, grads, seed):
    g = torch.Generator().manual_seed(seed)
    v = [torch.randn(a.shape, generator=g, dtype=torch.float64) for a in args]
    e = 1e-5
    d = (f(*[a + e * w for a, w in zip(args, v)]) - f(*[a - e * w for a, w in zip(args, v)])) / (2 * e)
    s = sum((a * b).sum() for a, b in zip(grads, v))
    assert abs(float(d - s)) <= 1e-7 * (1 + abs(float(s))) * len(v) * 10


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    kept = dict(R.HALF)
    R.HALF[torch.float64] = R.TINY[torch.float64] = 0.0
    try:
        B, L, Hq, Hkv, dh = 2, 5, 3, 2, 8
        x, gq, gk = rnd(B, L, 7 * dh), rnd(dh), rnd(dh)
        d = [rnd(B, h, L, dh) for h in (Hq, Hkv, Hkv)]
        a = torch.arange(L, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(3) / 3)
        table = torch.stack([torch.cos(a), torch.sin(a)], -1)
        for gains in ((gq, gk), (None, None)):
            (dx, _), a, b = S.heads_grad(*d, x, Hq, Hkv, dh, table, None, *gains, 1e-5, torch.float64)

            def f(x, gq, gk):
                q = (gq, gk) if gains[0] is not None else gains
                return sum((o[0] * w).sum() for o, w in zip(S.heads(x, Hq, Hkv, dh, table, None, *q, 1e-5, torch.float64), d))
            dg = [a[0], b[0]] if gains[0] is not None else [torch.zeros(dh, dtype=torch.float64)] * 2
            _directional(f, [x, gq, gk], [dx] + dg, 5)
        # turning keeps lengths, and by the opposite angle takes it back
        q, c, s = rnd(B, 3, L, dh), *S._angles(table, None, B, L, dh)
        t = S.turn(q, c, s)[0]
        assert torch.allclose(t.norm(dim=-1), q.norm(dim=-1)) and torch.allclose(S.turn(t, c, s, -1)[0], q)
        z, tok = rnd(6, 30) * 2, torch.tensor([3, -1, 29, 0, 7, 8], dtype=torch.int32)
        lp = torch.log_softmax(z, -1).gather(1, tok.long().clamp(min=0)[:, None])[:, 0]
        old, ref, adv, w = lp + torch.tensor([0.5, 0.0, -0.5, 0.1, 0.6, -0.1]), lp + 0.3 * rnd(6), torch.tensor([1.0, 1, 1, -1, -1, 2]), torch.tensor([1.0, 1, 0.5, 2, 1, 0])
        r = S.policy(z, tok, adv, old, ref, w, 0.8, 1.2, 0.3, 0.1)
        assert r["on"].tolist() == [True, False, True, True, True, False] and r["cut"][r["on"]].tolist() == [False, True, False, True]
        _directional(lambda t: S.policy(t, tok, adv, old, ref, w, 0.8, 1.2, 0.3, 0.1)["loss"], [z], [r["d_logits"]], 7)
    finally:
        R.HALF.clear()
        R.HALF.update(kept)
        R.TINY.pop(torch.float64, None)


def test_share_of_the_mask():
    """16 bits an element: each of p's shares in the long run, elements unlike their neighbours."""
    for p in (0.1, 0.5):
        k = S.kept(400, 1000, p, 5, 3).double()
        q = 1 - S.threshold(p) / 65536
        n = k.numel()
        assert abs(float(k.sum()) - q * n) <= 6 * math.sqrt(n * q * (1 - q))
        for step in (1, 2, 8):
            both = float((k[:, step:] * k[:, :-step]).mean())
            assert abs(both - q * q) <= 6 * math.sqrt(q * q * (1 - q * q) / n) + 1e-3
    assert S.kept(3, 9, 0.0, 1, 1).all() and not S.kept(3, 9, 1.0, 1, 1).any()
    assert np.array_equal(S.kept(5, 9, 0.3, 1, 1)[2:], S.kept(3, 9, 0.3, 1, 1, 2))
