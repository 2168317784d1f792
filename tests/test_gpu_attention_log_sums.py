"""The log sums that training attention keeps for its backward pass are those of the exponentials
themselves, not of their bf16 roundings: against 64 bits with fp32's bound."""
import pytest

import oracle as O
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
KIND = {0: "single", 1: "double"}


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


# both kernels (16 and 32 query rows a wavefront) at each d_head; rows of one key to some hundred
CASES = [(m, *c) for m in (0, 1) for c in [
    (1, 2, 1, 1, 32), (2, 2, 2, 1, 64), (1, 2, 5, 3, 128), (3, 5, 16, 4, 32), (2, 3, 37, 3, 64), (1, 2, 70, 5, 128), (1, 2, 130, 2, 64),
    (64, 12, 30, 3, 32), (64, 12, 30, 3, 64), (64, 12, 30, 3, 128), (128, 8, 100, 1, 64)]]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_B%d_H%d_N%d_k%d_dh%d" % (KIND[c[0]], *c[1:]))
@pytest.mark.parametrize("std", [1.0, 3.0])
def test_log_sums(Bd, case, std):
    """A score is off by (d_head + 8) U sum|q k| (products and sums) and three roundings of its size
    (scale, the base's factor, the difference); an exponential by 2 U of itself; a sum of n by n U; then
    a logarithm and two roundings of the result."""
    mask, B, H, N, k, dh = case
    rows, keys = Bd.training_attention_shapes(mask, N, k)
    g = torch.Generator(device="cuda").manual_seed(N + dh)
    mk = lambda n, s: (s * torch.randn(B, H, n, dh, generator=g, device="cuda")).bfloat16()
    q, k_, v = mk(rows, std), mk(keys, std), mk(keys, 1.0)
    o, lse = Bd.training_attention_lse(mask, q, k_, v, N, k)
    assert torch.equal(o, Bd.training_attention(mask, q, k_, v, N, k))
    M = torch.from_numpy(O.training_mask(KIND[mask], N, k)).bool()
    scale = dh ** -0.5
    for b, h in {(0, 0), (B - 1, H - 1), (B // 2, H // 3)}:
        a, c, w = q[b, h].cpu(), k_[b, h].cpu(), v[b, h].cpu()
        _, want, _ = R.attention(a, c, w, M, scale)
        size = (a.double().abs() @ c.double().abs().t() * scale).masked_fill(~M, 0).amax(-1)
        n = M.sum(-1).double()
        bound = R.U * ((dh + 8 + 3) * size + n + 16 + 4 * want.abs()) + 1e-7
        got = R.worst(lse[b, h], want, bound)
        print(case, std, round(got, 3), flush=True)
        assert got <= 1
