"""Argument checks of the training step's operators (no GPU: every call here is refused before a
launch, or is an empty problem), and the 64-bit references against differences."""
import ctypes
import math

import pytest

from paper_2606_10820_amd import binding as Bd
from tests import train_ref as R

torch = pytest.importorskip("torch")
P = ctypes.c_void_p
A = P(0x10000)  # 256-byte aligned, never dereferenced
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    return Bd.lib()


def test_norm_refusals(L):
    ok = dict(norm=0, xt=0, yt=0, rows=4, d=8, x=A, ldx=8, g=A, b=A, eps=1e-5, y=P(0x20000), ldy=8, st=A)

    def call(**kw):
        a = dict(ok, **kw)
        return L.kf_layer_norm(None, a["norm"], a["xt"], a["yt"], a["rows"], a["d"], a["x"], a["ldx"], a["g"], a["b"],
                               a["eps"], a["y"], a["ldy"], a["st"])

    for bad in (dict(norm=2), dict(norm=-1), dict(xt=3), dict(yt=-1), dict(xt=1, yt=0), dict(xt=1, yt=2), dict(xt=2, yt=1),
                dict(rows=-1), dict(d=0), dict(d=(1 << 28) + 1, ldx=1 << 29, ldy=1 << 29), dict(ldx=7), dict(ldy=7),
                dict(rows=1 << 58, ldx=1 << 10), dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF), dict(norm=1),
                dict(x=None), dict(y=None), dict(g=None), dict(x=P(0x10002)), dict(y=P(0x10002)), dict(g=P(0x10001)),
                dict(b=P(0x10002)), dict(st=P(0x10004)), dict(yt=1, y=A), dict(y=A, ldy=9)):
        assert call(**bad) == Bd.KF_EINVAL, bad
    assert call(rows=0, x=None, y=None, g=None, b=None, st=None) == Bd.KF_OK


def test_norm_backward_refusals(L):
    ok = dict(norm=0, xt=0, yt=0, rows=4, d=8, x=A, ldx=8, g=A, st=A, dy=A, lddy=8, res=None, ldr=8, dx=P(0x30000), ldd=8,
              dg=A, db=A, ws=A, n=1 << 20)

    def call(**kw):
        a = dict(ok, **kw)
        return L.kf_layer_norm_backward(None, a["norm"], a["xt"], a["yt"], a["rows"], a["d"], a["x"], a["ldx"], a["g"], a["st"],
                                        a["dy"], a["lddy"], a["res"], a["ldr"], a["dx"], a["ldd"], a["dg"], a["db"], a["ws"], a["n"])

    for bad in (dict(norm=7), dict(xt=1), dict(yt=5), dict(rows=-2), dict(d=0), dict(ldx=7), dict(lddy=0), dict(ldd=7),
                dict(res=A, ldr=7), dict(norm=1), dict(x=None), dict(dy=None), dict(dx=None), dict(g=None), dict(st=None),
                dict(st=P(0x10004)), dict(res=P(0x10002)), dict(dx=A), dict(res=P(0x30000), ldr=9), dict(ws=None),
                dict(ws=P(0x10008)), dict(n=0), dict(dg=P(0x10001)), dict(db=P(0x10002))):
        assert call(**bad) == Bd.KF_EINVAL, bad
    need = L.kf_layer_norm_backward_bytes(4, 8)
    assert need > 0 and call(n=need - 1) == Bd.KF_EINVAL
    assert L.kf_layer_norm_backward_bytes(0, 8) == 0 and L.kf_layer_norm_backward_bytes(4, 0) == 0


def test_logprobs_refusals(L):
    ok = dict(t=0, rows=3, V=100, x=A, ld=100, tok=A, top=5, lp=A, h=A, lse=A, ids=A, tl=A)

    def call(**kw):
        a = dict(ok, **kw)
        return L.kf_token_logprobs(None, a["t"], a["rows"], a["V"], a["x"], a["ld"], a["tok"], a["top"], a["lp"], a["h"], a["lse"], a["ids"], a["tl"])

    for bad in (dict(t=3), dict(t=-1), dict(rows=-1), dict(V=0), dict(V=(1 << 28) + 1, ld=1 << 29), dict(ld=99), dict(top=-1), dict(top=65),
                dict(V=4, top=5), dict(x=None), dict(x=P(0x10002)), dict(tok=P(0x10002)), dict(lp=P(1)), dict(h=P(2)),
                dict(lse=P(3)), dict(ids=None), dict(tl=None), dict(tl=P(0x10002)), dict(rows=1 << 57)):
        assert call(**bad) == Bd.KF_EINVAL, bad
    assert call(rows=0, x=None, ids=None, tl=None) == Bd.KF_OK

    def back(**kw):
        a = dict(t=1, rows=3, V=100, x=A, ld=100, tok=A, u=A, c=None, lp=None, h=None, lse=None, d=P(0x40000), ldd=100, **{})
        a.update(kw)
        return L.kf_token_logprobs_backward(None, a["t"], a["rows"], a["V"], a["x"], a["ld"], a["tok"], a["u"], a["c"], a["lp"], a["h"], a["lse"], a["d"], a["ldd"])

    for bad in (dict(t=9), dict(rows=-1), dict(V=-5), dict(ld=99), dict(ldd=99), dict(x=None), dict(d=None), dict(d=P(0x40001)),
                dict(u=P(0x10002)), dict(c=P(0x10001)), dict(d=A, ldd=101)):
        assert back(**bad) == Bd.KF_EINVAL, bad
    assert back(rows=0, x=None, d=None) == Bd.KF_OK


def test_clip_refusals(L):
    def arr(*gs):
        return (Bd.KfGrad * max(len(gs), 1))(*[Bd.KfGrad(*g) for g in gs])

    good = (0x10000, 0x20000, 10, 0, 0)
    assert L.kf_grad_plan_bytes(1, arr(good)) > L.kf_grad_plan_bytes(0, None) > 0
    for bad in ((0, 0x20000, 10, 0, 0), (0x10002, 0x20000, 10, 0, 0), (0x10000, 0x20001, 10, 1, 1), (0x10000, 0x20000, -1, 0, 0),
                (0x10000, 0x20000, 10, 3, 0), (0x10000, 0x20000, 10, 0, 1), (0x10000, 0x20000, 10, 1, 2), (0x10000, 0x10000, 10, 1, 0),
                (0x10000, 0x20000, (1 << 48) + 1, 0, 0)):
        assert L.kf_grad_plan_bytes(2, arr(good, bad)) == 0, bad
        assert L.kf_grad_plan_init(None, 2, arr(good, bad), A, 1 << 30, ctypes.byref(Bd.KfGradPlan())) == Bd.KF_EINVAL
    assert L.kf_grad_plan_bytes(-1, arr(good)) == 0 and L.kf_grad_plan_bytes(1, None) == 0
    plan = Bd.KfGradPlan()
    n = L.kf_grad_plan_bytes(1, arr(good))
    assert L.kf_grad_plan_init(None, 1, arr(good), A, n - 1, ctypes.byref(plan)) == Bd.KF_EINVAL
    assert L.kf_grad_plan_init(None, 1, arr(good), P(0x10010), n, ctypes.byref(plan)) == Bd.KF_EINVAL
    assert L.kf_grad_plan_init(None, 1, arr(good), A, n, None) == Bd.KF_EINVAL
    # a dst on another dst, on another src, half over its own src, a tensor twice in place
    for clash in ((good, (0x30000, 0x20010, 10, 0, 0)), (good, (0x30000, 0x10020, 4, 0, 0)), ((0x10000, 0x10010, 10, 0, 0),),
                  ((0x10000, 0x10000, 10, 0, 0),) * 2):
        a = arr(*clash)
        assert L.kf_grad_plan_init(None, len(clash), a, A, 1 << 30, ctypes.byref(plan)) == Bd.KF_EINVAL, clash
    fake = Bd.KfGradPlan(0x10000, 1, 1)
    assert L.kf_grad_norm(None, None, A) == Bd.KF_EINVAL
    assert L.kf_grad_norm(None, ctypes.byref(fake), None) == Bd.KF_EINVAL
    assert L.kf_grad_norm(None, ctypes.byref(Bd.KfGradPlan(0, 1, 1)), A) == Bd.KF_EINVAL
    for m in (-1.0, NAN):
        assert L.kf_grad_clip(None, ctypes.byref(fake), m, A) == Bd.KF_EINVAL
    assert L.kf_grad_clip(None, ctypes.byref(Bd.KfGradPlan(0x10000, 1, 0)), 1.0, A) == Bd.KF_EINVAL  # no dst


def test_attention_backward_refusals(L):
    ok = dict(mask=0, B=2, H=3, N=8, k=4, dh=64, scale=0.125)

    def fwd(ptrs=(A,) * 5, **kw):
        a = dict(ok, **kw)
        return L.kf_training_attention_lse(None, a["mask"], a["B"], a["H"], a["N"], a["k"], a["dh"], *ptrs, a["scale"])

    def bwd(ptrs=(A,) * 9, ws=A, n=1 << 40, **kw):
        a = dict(ok, **kw)
        return L.kf_training_attention_backward(None, a["mask"], a["B"], a["H"], a["N"], a["k"], a["dh"], *ptrs, a["scale"], ws, n)

    for bad in (dict(mask=2), dict(k=0), dict(B=-1), dict(N=-3), dict(dh=48), dict(scale=INF), dict(scale=NAN), dict(scale=0.0), dict(scale=-0.2), dict(scale=1e-21), dict(scale=1e21),
                dict(mask=1, N=1 << 22, k=4), dict(N=4000, k=2000, dh=32, B=1, H=1)):
        assert fwd(**bad) == Bd.KF_EINVAL, bad
        assert bwd(**bad) == Bd.KF_EINVAL, bad
        if "scale" not in bad:
            a = dict(ok, **bad)
            assert L.kf_training_attention_backward_bytes(a["mask"], a["B"], a["H"], a["N"], a["k"], a["dh"]) == 0
    for i in range(5):
        assert fwd(ptrs=(A,) * i + (P(0x10008),) + (A,) * (4 - i)) == Bd.KF_EINVAL
    for i in range(9):
        assert bwd(ptrs=(A,) * i + (None,) + (A,) * (8 - i)) == Bd.KF_EINVAL
    need = L.kf_training_attention_backward_bytes(0, 2, 3, 8, 4, 64)
    assert need > 0 and bwd(n=need - 1) == Bd.KF_EINVAL and bwd(ws=None) == Bd.KF_EINVAL
    for empty in (dict(B=0), dict(H=0), dict(N=0)):
        assert fwd(ptrs=(None,) * 5, **empty) == Bd.KF_OK
        assert bwd(ptrs=(None,) * 9, ws=None, n=0, **empty) == Bd.KF_OK


def test_binding_refuses_host_tensors_and_bad_shapes():
    x, g = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(ValueError):
        Bd.layer_norm(x, g)
    with pytest.raises(ValueError):
        Bd.layer_norm(x, torch.ones(7))
    with pytest.raises(ValueError):
        Bd.layer_norm(x.t(), torch.ones(4))
    with pytest.raises(ValueError):
        Bd.token_logprobs(torch.zeros(2, 5), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        Bd.GradClip([])
    with pytest.raises(ValueError):
        Bd.GradClip([torch.zeros(4, 4).t()[1:]])


# ------------------------------- the references' gradients against differences
def _directional(f, args, grads, seed):
    """sum(grad . v) against a central difference of f along random directions v (fp64)."""
    g = torch.Generator().manual_seed(seed)
    v = [torch.randn(a.shape, generator=g, dtype=torch.float64) for a in args]
    e = 1e-5
    d = (f(*[a + e * w for a, w in zip(args, v)]) - f(*[a - e * w for a, w in zip(args, v)])) / (2 * e)
    s = sum((a * b).sum() for a, b in zip(grads, v))
    assert abs(float(d - s)) <= 1e-7 * (1 + abs(float(s))) * len(v) * 10


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    HALF64 = dict(R.HALF)
    R.HALF[torch.float64] = R.TINY[torch.float64] = 0.0
    try:
        x, gain, shift, dy = rnd(5, 12), rnd(12), rnd(12), rnd(5, 12)
        for rms in (False, True):
            (dx, dg, db), _ = R.norm_grad(dy, x, gain, 1e-5, rms)
            f = lambda a, b, c: (R.norm(a, b, None if rms else c, 1e-5, rms)[0] * dy).sum()
            _directional(f, [x, gain, shift], [dx, dg, torch.zeros_like(db) if rms else db], 5)
        z, tok, u, c = rnd(4, 30) * 3, torch.tensor([3, -1, 29, 0]), rnd(4), rnd(4)
        z[1, 7] = -math.inf
        d, _ = R.logprobs_grad(z, tok, u, c)

        def loss(a):
            r = R.logprobs(a, tok)
            return (r["logp"] * u + r["entropy"] * c).sum()
        keep = torch.isfinite(z)
        _directional(lambda a: loss(torch.where(keep, a, z)), [z.nan_to_num(neginf=0.0)], [d * keep], 7)
        import oracle as O
        for kind in ("single", "double"):
            mask = torch.from_numpy(O.training_mask(kind, 4, 3)).bool()
            q, k, v, do = rnd(mask.shape[0], 8), rnd(mask.shape[1], 8), rnd(mask.shape[1], 8), rnd(mask.shape[0], 8)
            grads, _ = R.attention_grad(q, k, v, do, mask, 0.3)
            _directional(lambda a, b, c: (R.attention(a, b, c, mask, 0.3)[0] * do).sum(), [q, k, v], grads, 9)
    finally:
        R.HALF.clear()
        R.HALF.update(HALF64)
        R.TINY.pop(torch.float64, None)
