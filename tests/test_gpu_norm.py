"""GPU parity of LayerNorm and RMSNorm with their gradients against 64-bit references (bounds:
tests/train_ref.py), over widths on both sides of every kernel's edge, odd widths, strides and
misaligned rows."""
import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
EPS = 1e-5
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (F32, BF), (F32, HF), (BF, BF), (HF, HF)]
IDS = lambda v: str(v).replace("torch.", "")


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _inputs(rows, d, xt, yt, seed=0, offset=0.5):
    g = torch.Generator().manual_seed(seed + 17 * rows + d)
    rnd = lambda *s: torch.randn(*s, generator=g)
    x = (rnd(rows, d) + offset * rnd(rows, 1)).to(xt)
    return x, 1 + 0.2 * rnd(d), 0.1 * rnd(d), rnd(rows, d).to(yt), rnd(rows, d).to(xt)


def _both(Bd, x, gain, shift, dy, dres, rms, yt, where=""):
    """Forward and backward on the GPU against the references, for CPU tensors (device tensors keep
    the strides of the CPU ones' storage when they are given as (device, cpu) pairs)."""
    dev = lambda t: t if t is None or t.is_cuda else t.cuda()
    shift = None if rms else shift
    X, DY, DR = dev(x), dev(dy), dev(dres)
    y, stats = Bd.layer_norm(X, dev(gain), dev(shift), EPS, rms, yt)
    dx, dg, db = Bd.layer_norm_backward(DY, X, dev(gain), stats, rms, DR)
    torch.cuda.synchronize()
    x, dy, dres = (t.cpu() if t is not None else None for t in (X, DY, DR))
    ref, mu, r = R.norm(x, gain, shift, EPS, rms)
    (rdx, rdg, rdb), (bx, bg, bb) = R.norm_grad(dy, x, gain, EPS, rms, dres)
    got = dict(y=R.worst(y, ref, R.norm_bound(x, gain, shift, EPS, rms, yt)), dx=R.worst(dx, rdx, bx), dgain=R.worst(dg, rdg, bg))
    K = (x.shape[-1] / 64 + 32) * R.U
    got["mean"] = R.worst(stats[:, 0], mu.reshape(-1), K * x.double().abs().mean(-1).reshape(-1) + 1e-30)
    got["rstd"] = R.worst(stats[:, 1], r.reshape(-1), 2 * K * r.reshape(-1))
    if rms:
        assert db is None
    else:
        got["dshift"] = R.worst(db, rdb, bb)
    print(where, tuple(x.shape), {k: round(v, 3) for k, v in got.items()}, flush=True)
    assert all(v <= 1.0 for v in got.values()), got
    return y, dx, dg, db


@pytest.mark.parametrize("rms", [False, True], ids=["layer", "rms"])
@pytest.mark.parametrize("pair", PAIRS, ids=lambda p: f"{IDS(p[0])}-{IDS(p[1])}")
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (1, 64), (5, 63), (7, 100), (33, 128), (9, 256), (13, 257), (6, 512), (10, 520), (131, 768),
                                    (12, 771), (65, 1024), (9, 1028), (4, 1536), (5, 2048), (3, 2049), (4, 4096), (3, 5000), (2, 8192), (2, 8200), (2, 16384), (2, 20001)])
def test_parity(Bd, rows, d, pair, rms):
    _both(Bd, *_inputs(rows, d, *pair, seed=PAIRS.index(pair)), rms, pair[1])


@pytest.mark.parametrize("rows", [0, 1, 2, 3, 4, 5, 63, 64, 513, 2047, 4099])
def test_row_counts(Bd, rows):
    """The strips of the column sums with and without rows of their own; an empty batch has zero sums."""
    for d, pair in ((96, PAIRS[1]), (40, PAIRS[3])):
        if rows:
            _both(Bd, *_inputs(rows, d, *pair), False, pair[1])
            continue
        x, gain, shift, dy, _ = (t.cuda() for t in _inputs(0, d, *pair))
        y, stats = Bd.layer_norm(x, gain, shift, out_dtype=pair[1])
        dx, dg, db = Bd.layer_norm_backward(dy, x, gain, stats)
        assert y.shape == dx.shape == (0, d) and not dg.any() and not db.any()


@pytest.mark.parametrize("pair", [PAIRS[1], PAIRS[3]], ids=["fp32-bf16", "bf16-bf16"])
@pytest.mark.parametrize("d,ld,off", [(768, 800, 0), (768, 768, 1), (768, 771, 0), (768, 776, 3), (100, 104, 4), (1024, 1025, 1), (4096, 4100, 2)])
def test_strides_and_alignment(Bd, pair, d, ld, off):
    """Rows ld apart that start off elements into their storage: what lies between rows is not read
    (NaN there) and, in out, not written."""
    rows = 11
    x, gain, shift, dy, dres = _inputs(rows, d, *pair)

    def strided(t):
        buf = torch.full((rows * ld + off,), float("nan"), dtype=t.dtype, device="cuda")
        v = buf[off:].view(rows, ld)[:, :d] if ld * rows + off <= buf.numel() else None
        v.copy_(t)
        return v
    X, DY, DR = strided(x), strided(dy), strided(dres)
    y, dx, dg, db = _both(Bd, X, gain, shift, DY, DR, False, pair[1], f"ld {ld} off {off}")
    out = torch.full((rows * ld + off,), 7.0, dtype=pair[1], device="cuda")
    o = out[off:].view(rows, ld)[:, :d]
    Bd.layer_norm(X, gain.cuda(), shift.cuda(), EPS, False, pair[1], out=o)
    torch.cuda.synchronize()
    assert torch.equal(o, y)
    assert (out[:off] == 7).all() and (out[off:].view(rows, ld)[:, d:] == 7).all()


def test_shapes_of_more_dimensions(Bd):
    x, gain, shift, dy, _ = _inputs(24, 96, F32, BF)
    a, s = Bd.layer_norm(x.cuda(), gain.cuda(), shift.cuda(), out_dtype=BF)
    b, s3 = Bd.layer_norm(x.view(2, 3, 4, 96).cuda(), gain.cuda(), shift.cuda(), out_dtype=BF)
    assert b.shape == (2, 3, 4, 96) and torch.equal(a, b.view(24, 96)) and torch.equal(s, s3)
    one, _ = Bd.layer_norm(x[5].cuda(), gain.cuda(), shift.cuda(), out_dtype=BF)
    assert one.shape == (96,) and torch.equal(one, a[5])
    with pytest.raises(ValueError):
        Bd.layer_norm(x.view(2, 12, 96).transpose(0, 1).cuda(), gain.cuda())


def test_in_place_and_no_shift(Bd):
    x, gain, shift, dy, dres = (t.cuda() for t in _inputs(37, 256, BF, BF))
    y, _ = Bd.layer_norm(x, gain, shift)
    z = x.clone()
    Bd.layer_norm(z, gain, shift, out=z)
    assert torch.equal(y, z)
    y0, _ = Bd.layer_norm(x, gain)
    ref = R.norm(x.cpu(), gain.cpu(), None, EPS, False)[0]
    assert R.worst(y0, ref, R.norm_bound(x.cpu(), gain.cpu(), None, EPS, False, BF)) <= 1


def test_residual_gradient_in_place(Bd):
    """dx over dres through the C ABI, and null dgain / dshift without a workspace."""
    L = Bd.lib()
    x, gain, shift, dy, dres = (t.cuda() for t in _inputs(50, 384, F32, BF))
    y, stats = Bd.layer_norm(x, gain, shift, out_dtype=BF)
    dx, dg, db = Bd.layer_norm_backward(dy, x, gain, stats, dres=dres)
    buf = dres.clone()
    s = torch.cuda.current_stream().cuda_stream
    p = lambda t: t.data_ptr()
    rc = L.kf_layer_norm_backward(s, 0, 0, 1, 50, 384, p(x), 384, p(gain), p(stats), p(dy), 384, p(buf), 384, p(buf), 384, None, None, None, 0)
    assert rc == 0
    torch.cuda.synchronize()
    assert torch.equal(buf, dx)


def test_large_offset(Bd):
    """A row whose offset is 1000 times its spread: squares of deviations, not of values."""
    x, gain, shift, dy, dres = _inputs(16, 512, F32, F32, offset=0.0)
    _both(Bd, x + 1000.0, gain, shift, dy, None, False, F32)


def test_values_that_are_not_finite(Bd):
    """A row with an infinity or NaN is NaN; its neighbours and their gradients are not touched."""
    x, gain, shift, dy, _ = _inputs(9, 200, F32, F32)
    x[3, 10], x[6, 199] = float("inf"), float("nan")
    y, stats = Bd.layer_norm(x.cuda(), gain.cuda(), shift.cuda())
    good = [i for i in range(9) if i not in (3, 6)]
    ref = R.norm(x[good], gain, shift, EPS, False)[0]
    assert R.worst(y[good], ref, R.norm_bound(x[good], gain, shift, EPS, False, F32)) <= 1
    assert torch.isnan(y[[3, 6]]).all()
    dx, _, _ = Bd.layer_norm_backward(dy.cuda(), x.cuda(), gain.cuda(), stats)
    (rdx, _, _), (b, _, _) = R.norm_grad(dy[good], x[good], gain, EPS, False)
    assert R.worst(dx[good], rdx, b) <= 1


def test_constant_rows(Bd):
    """Zero variance: r = eps^-1/2, y = shift, dx finite."""
    x = torch.full((4, 130), 3.0)
    _, gain, shift, dy, _ = _inputs(4, 130, F32, F32)
    _both(Bd, x, gain, shift, dy, None, False, F32)
    _both(Bd, torch.zeros(4, 130), gain, shift, dy, None, True, F32)


def test_many_rows(Bd):
    """More rows than the grid, offsets past 2^31 bytes."""
    rows, d = 600_001, 1024
    x = torch.empty(rows, d, dtype=BF, device="cuda").normal_()
    gain = torch.rand(d, device="cuda")
    dy = torch.empty(rows, d, dtype=BF, device="cuda").normal_()
    y, stats = Bd.layer_norm(x, gain, rms=True)
    dx, dg, _ = Bd.layer_norm_backward(dy, x, gain, stats, rms=True)
    torch.cuda.synchronize()
    pick = [0, 1, 300_000, rows - 2, rows - 1]
    xs, g, dys = x[pick].cpu(), gain.cpu(), dy[pick].cpu()
    assert R.worst(y[pick], R.norm(xs, g, None, EPS, True)[0], R.norm_bound(xs, g, None, EPS, True, BF)) <= 1
    (rdx, _, _), (b, _, _) = R.norm_grad(dys, xs, g, EPS, True)
    assert R.worst(dx[pick], rdx, b) <= 1
    part = torch.zeros(d, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(part)
    for i in range(0, rows, 50_000):
        t = dy[i:i + 50_000].double() * x[i:i + 50_000].double() * stats[i:i + 50_000, 1:].double()
        part += t.sum(0)
        size += t.abs().sum(0)
    assert float(((dg.double() - part).abs() / (size * R.U * 2000)).max()) <= 1  # at most 2000 rows in a strip's row


def test_same_result_on_every_run(Bd):
    x, gain, shift, dy, dres = (t.cuda() for t in _inputs(3000, 768, F32, BF))
    first = None
    for _ in range(3):
        y, stats = Bd.layer_norm(x, gain, shift, out_dtype=BF)
        res = (y, stats, *Bd.layer_norm_backward(dy, x, gain, stats, dres=dres))
        first = first or res
        assert all(torch.equal(a, b) for a, b in zip(first, res))


def test_difference_quotient(Bd):
    """The gradient against differences of the framework's own forward pass (fp32): along v of
    size e, the loss dy.y moves by e dx.v + O(e^3), its own rounding U sqrt(n) |dy| |y| aside."""
    x, gain, shift, dy, _ = (t.cuda() for t in _inputs(40, 300, F32, F32))
    y, stats = Bd.layer_norm(x, gain, shift)
    dx, dg, db = Bd.layer_norm_backward(dy, x, gain, stats)
    g = torch.Generator(device="cuda").manual_seed(1)
    v, vg, vb = (torch.randn(t.shape, generator=g, device="cuda") for t in (x, gain, shift))
    e = 2.0 ** -8
    f = lambda s: (Bd.layer_norm(x + s * e * v, gain + s * e * vg, shift + s * e * vb)[0].double() * dy.double()).sum()
    got = float(f(1) - f(-1)) / (2 * e)
    want = float((dx.double() * v).sum() + (dg.double() * vg).sum() + (db.double() * vb).sum())
    size = float((dx.double() * v).abs().sum() + (dg.double() * vg).abs().sum())
    # third derivative along v: y is a ratio whose terms are of size 1, so 6 e^2 of the sum of magnitudes
    assert abs(got - want) <= size * (6 * e * e) + 4 * R.U / e * float((dy.double().abs() * y.double().abs()).sum())
