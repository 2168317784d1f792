"""Dropout of rows of odd width that follow each other, past one pass of a launch (4096 workgroups of 256
threads, eight elements each): the mask is that of (row, column) in every pass, against the generator in
numpy (bounds: tests/step_ref.py)."""
import pytest

from tests import step_ref as S
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF = torch.float32, torch.bfloat16
PASS = 4096 * 256 * 8
SEED, SITE, P = 0x9E3779B97F4A7C15, 6, 0.3


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _places(rows, d, passes):
    """First rows of stretches of four that hold the ends of passes, and the last one."""
    return [0] + [max(0, k * PASS // d - 1) for k in passes if k * PASS // d + 3 <= rows] + [rows - 4]


@pytest.mark.parametrize("rows,d", [(40961, 771), (300001, 33), (1048577, 9)])
@pytest.mark.parametrize("kind", [(BF, F32), (F32, BF), (BF, BF)], ids=lambda p: "-".join(str(t).replace("torch.", "") for t in p))
def test_passes(Bd, rows, d, kind):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, d, generator=g, device="cuda").to(kind[0])
    res = (3 * torch.randn(rows, d, generator=g, device="cuda")).to(kind[1])
    y = Bd.dropout(x, P, SEED, SITE, res)
    plain = Bd.dropout(x, P, SEED, SITE, out_dtype=kind[1])
    dx = Bd.dropout_backward(res, P, SEED, SITE, kind[0])
    places = _places(rows, d, range(1, rows * d // PASS + 1))
    assert len(places) >= 3
    for r in places:
        at = slice(r, r + 4)
        for got, a, b, t in ((y, x, res, kind[1]), (plain, x, None, kind[1]), (dx, res, None, kind[0])):
            ref, bound = S.dropout(a[at].cpu(), P, SEED, SITE, None if b is None else b[at].cpu(), t, r)
            assert R.worst(got[at], ref, bound + 1e-300) <= 1, (r, b is None)
    # the same rows apart, an element at a time
    wide = torch.zeros(rows, d + 1, dtype=kind[0], device="cuda")[:, :d]
    wide.copy_(x)
    assert torch.equal(Bd.dropout(wide, P, SEED, SITE, res), y)


def test_past_32_bits(Bd):
    rows, d = 2_800_003, 771
    assert rows * d > 2 ** 31
    x = torch.ones(rows, d, dtype=BF, device="cuda")
    Bd.dropout(x, P, SEED, SITE, out=x)
    for r in _places(rows, d, (1, 2, 255, 256, 257)):
        assert torch.equal(x[r:r + 4].cpu() != 0, S.kept(4, d, P, SEED, SITE, r)), r
