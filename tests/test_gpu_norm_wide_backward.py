"""Gradients of the gain and shift of the widest rows: a launch holds fewer than 2^32 threads, which a
workgroup of 1024 for each 32 of 2^27 column sums is."""
import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("d", [(1 << 20) + 5, (1 << 26) + 3])
def test_column_sums(Bd, d):
    """Two rows of given statistics: dshift is a sum of two values, dgain of two products of three
    factors (four roundings of each)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(2, d, generator=g, device="cuda").to(BF) for _ in range(2))
    gain = torch.ones(d, device="cuda")
    stats = torch.tensor([[0.25, 0.5], [-0.125, 2.0]], device="cuda")
    dx, dgain, dshift = Bd.layer_norm_backward(dy, x, gain, stats)
    torch.cuda.synchronize()
    assert torch.equal(dshift, dy[0].float() + dy[1].float())
    term = lambda i: dy[i].double() * (x[i].double() - stats[i, 0].double()) * stats[i, 1].double()
    ref, size = term(0) + term(1), term(0).abs() + term(1).abs()
    # the difference x - mu is rounded once, relative to itself
    assert float(((dgain.double() - ref).abs() / (6 * R.U * size + 1e-30)).max()) <= 1
    assert torch.isfinite(dx).all()
