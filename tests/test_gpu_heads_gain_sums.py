"""Gradients of the norms' gains over more tokens than one pass of a launch takes, against sums in 64 bits
formed on the GPU, with a bound from the order in which the kernel adds."""
import pytest

from tests import step_ref as S
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF = torch.float32, torch.bfloat16
EPS = 1e-5


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _sums(x, heads, first, dh, d, table):
    """sum of w x r and of its terms' magnitudes, [dh] each, for heads first .. first + heads - 1 of rows
    x [B][L][W] with gradients d [B][heads][L][dh]."""
    B, L, _ = x.shape
    total = torch.zeros(2, dh, dtype=torch.float64, device="cuda")
    for l0 in range(0, L, 16384):
        l = slice(l0, min(L, l0 + 16384))
        t = x[:, l].view(B, l.stop - l0, -1, dh)[:, :, first:first + heads].transpose(1, 2).double()
        xh = t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS)
        w = d[:, :, l].double()
        m = w.abs()
        if table is not None:
            c = torch.ones(1, 1, l.stop - l0, (dh + 1) // 2, dtype=torch.float64, device="cuda")
            s = torch.zeros_like(c)
            n = table.shape[1]
            c[..., :n], s[..., :n] = table[l, :, 0].double(), table[l, :, 1].double()
            w, m = S.turn(w, c, s, -1)
        total[0] += (w * xh).sum((0, 1, 2))
        total[1] += (m * xh.abs()).sum((0, 1, 2))
    return total.cpu()


def _chain(tokens, H_all):
    """Additions one after another, at most, that a term of a gain's gradient goes through.  Up to 2048
    workgroups of four wavefronts share the tokens and groups of heads; of H_all heads of three kinds there
    are at most H_all / 4 + 3 groups.  A lane adds its columns over up to four heads of each of its tokens,
    of which a wavefront takes one at least at once.  Then 6 levels of lanes, 3 wavefronts, and the strips
    by 32: a share of 2048 / 32 = 64, and 31."""
    blocks = 2048 // (H_all // 4 + 3)
    return 4 * (tokens // (blocks * 4) + 1) + 6 + 3 + 64 + 31


@pytest.mark.parametrize("kind", [(F32, BF), (BF, BF)], ids=["fp32-bf16", "bf16-bf16"])
@pytest.mark.parametrize("B,L,Hq,Hkv,dh,rot", [(3, 33367, 2, 1, 32, 32), (1, 100003, 2, 2, 77, 64), (2, 40001, 4, 1, 96, 0)])
@pytest.mark.parametrize("same_sign", [True, False], ids=["positive", "signed"])
def test_many_tokens(Bd, B, L, Hq, Hkv, dh, rot, kind, same_sign):
    """With the heads' own values as gradients every term is about the gain times a square: a strip or a
    pass that is lost shows.  With random ones the sums cancel, and the order of the additions shows.
    A term's own error: as in tests/step_ref.py."""
    g = torch.Generator(device="cuda").manual_seed(L)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = rnd(B, L, (Hq + 2 * Hkv) * dh).to(kind[0])
    table = Bd.rope_table(L, rot) if rot else None
    gq, gk = 1 + 0.2 * rnd(dh), 1 + 0.2 * rnd(dh)
    ones = torch.ones(dh, device="cuda")
    if same_sign:
        d = Bd.qkv_heads(x, Hq, Hkv, table, None, ones, ones, EPS, kind[1])
    else:
        d = [rnd(B, h, L, dh).to(kind[1]) for h in (Hq, Hkv, Hkv)]
    _, dgq, dgk = Bd.qkv_heads_backward(*d, x, table, None, gq, gk, EPS)
    for got, heads, first, grad in ((dgq, Hq, 0, d[0]), (dgk, Hkv, Hq, d[1])):
        want, size = _sums(x, heads, first, dh, grad, table)
        b = (_chain(B * L, Hq + 2 * Hkv) + 2 * S.C_NORM + 16) * R.U * size
        worst = R.worst(got, want, b)
        # a workgroup's share of one pass (four wavefronts of 8 terms or more a column) stands out from the bound
        print((B, L, Hq, Hkv, dh), round(worst, 4), float((b / size).max() * B * L * heads), flush=True)
        assert worst <= 1
        assert not same_sign or float((b / size).max()) * B * L * heads < 4 * 8


def test_past_32_bits(Bd):
    Hq, Hkv, dh, L = 18, 16, 64, 690_000
    x = torch.empty(1, L, (Hq + 2 * Hkv) * dh, dtype=BF, device="cuda")
    assert x.numel() > 2 ** 31
    x.normal_()
    table, g = Bd.rope_table(L, 64), torch.ones(dh, device="cuda")
    d = Bd.qkv_heads(x, Hq, Hkv, table, None, g, g)
    _, dgq, dgk = Bd.qkv_heads_backward(*d, x, table, None, g, g)
    for got, heads, first, grad in ((dgq, Hq, 0, d[0]), (dgk, Hkv, Hq, d[1])):
        want, size = _sums(x, heads, first, dh, grad, table)
        b = (_chain(L, Hq + 2 * Hkv) + 2 * S.C_NORM + 16) * R.U * size
        print(R.worst(got, want, b), flush=True)
        assert R.worst(got, want, b) <= 1


def test_positions_outside_the_table(Bd):
    """NaN in the turned columns of the gains' gradients and in that row's gradients, nowhere else."""
    B, L, H, dh, rot = 2, 40, 2, 64, 32
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, gain = rnd(B, L, 3 * H * dh), 1 + 0.2 * rnd(dh)
    d = [rnd(B, H, L, dh) for _ in range(3)]
    pos = torch.arange(L, dtype=torch.int32, device="cuda").expand(B, L).contiguous()
    pos[1, 7] = 50
    table = Bd.rope_table(50, rot)
    dx, dgq, dgk = Bd.qkv_heads_backward(*d, x, table, pos, gain, gain)
    for dg in (dgq, dgk):
        assert torch.isnan(dg[:rot]).all() and torch.isfinite(dg[rot:]).all()
    bad = torch.zeros(B, L, 3 * H * dh, dtype=torch.bool)
    bad[1, 7, :2 * H * dh] = True
    assert torch.equal(torch.isnan(dx).cpu(), bad)
