"""P and dS enter dV and dK as two bf16 terms whatever the number of heads: the same head alone and among
many, both walks' block sizes, against 64 bits with a bound that one term of 8 bits does not meet."""
import pytest

import oracle as O
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
KIND = {0: "single", 1: "double"}
BF = torch.bfloat16


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _bounds(q, k_, v, do, M, scale):
    """((dk, dv), bounds).  h: half a bf16 step, of the results.  A score, with the log sum that is taken
    from it, is off by (d_head + 11) U of its products' sizes and of the log sum, in either pass; an
    exponential by 4 U; a log sum by n U more, n the keys a row sees; two terms leave h^2 of P and of dS; sums over
    rows (rows U).  dP - D by (d_head + 8) U of its products' sizes; the D of the other walk is that whose
    row sum of dS is zero, up to the log sum's error times what O's rounding, 2 h, put it off by, and that
    sum's own roundings (n U)."""
    h, U = R.HALF[BF], R.U
    o, lse, p = R.attention(q, k_, v, M, scale)
    q, k_, v, do = (t.double() for t in (q, k_, v, do))
    T = lambda t: t.transpose(-1, -2)
    dh, n, rows = q.shape[-1], M.sum(-1, keepdim=True).double(), q.shape[0]
    dp = do @ T(v)
    D = (do * o).sum(-1, keepdim=True)
    ds = p * (dp - D)
    size = scale * (q.abs() @ T(k_.abs()))
    e = 2 * (dh + 11) * U * (size + size.masked_fill(~M, 0).amax(-1, keepdim=True) + lse.abs()[:, None]) + (n + 16 + 4 * lse.abs()[:, None]) * U
    mag = do.abs() @ T(v.abs())
    top = mag.masked_fill(~M, 0).amax(-1, keepdim=True)
    pe = p * (e + h * h + rows * U)
    de = (dh + 8) * U * (mag + 2 * top) + (3 * h * e.masked_fill(~M, 0).amax(-1, keepdim=True) + n * U) * top
    se = ds.abs() * (e + h * h + rows * U) + p * de
    dk, dv = T(ds) @ q * scale, T(p) @ do
    return (dk, dv), (1.02 * (scale * (T(se) @ q.abs()) + h * dk.abs()) + 1e-30, 1.02 * (T(pe) @ do.abs() + h * dv.abs()) + 1e-30)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("mask,N,k", [(0, 30, 3), (0, 129, 2), (1, 1, 1), (1, 45, 4)])
def test_same_terms_alone_and_among_many_heads(Bd, mask, N, k, dh):
    rows, keys = Bd.training_attention_shapes(mask, N, k)
    g = torch.Generator().manual_seed(N + dh)
    one = [torch.randn(1, n, dh, generator=g).to(BF) for n in (rows, keys, keys, rows)]
    M, scale = torch.from_numpy(O.training_mask(KIND[mask], N, k)).bool(), dh ** -0.5
    ref, bound = _bounds(*[t[0] for t in one], M, scale)
    for heads in (1, 60, 150, 400):  # one walk's block sizes and the other's
        q, k_, v, do = (t.cuda().expand(heads, -1, -1)[None].contiguous() for t in one)
        o, lse = Bd.training_attention_lse(mask, q, k_, v, N, k)
        _, dk, dv = Bd.training_attention_backward(mask, q, k_, v, o, lse, do, N, k)
        assert all((t[0] == t[0, :1]).all() for t in (dk, dv))  # the heads are alike
        got = [R.worst(t[0, heads // 2], r, b) for t, r, b in zip((dk, dv), ref, bound)]
        print(mask, N, k, dh, heads, [round(x, 3) for x in got], flush=True)
        assert max(got) <= 1, heads
