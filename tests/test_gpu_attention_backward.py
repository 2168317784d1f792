"""GPU parity of the training-mask attention's gradients and row sums against the 64-bit formula
(bounds: tests/train_ref.py, from the roundings of P, dS, O and the results to bf16)."""
import numpy as np
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


def _inputs(B, H, rows, keys, dh, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    mk = lambda n, s: (torch.randn(B, H, n, dh, generator=g) * s).to(BF)
    return mk(rows, std), mk(keys, std), mk(keys, 1.0), mk(rows, 1.0)


def _run(Bd, mask, q, k_, v, do, N, k, scale=None):
    o, lse = Bd.training_attention_lse(mask, q, k_, v, N, k, scale)
    return (o, lse, *Bd.training_attention_backward(mask, q, k_, v, o, lse, do, N, k, scale))


def _check(got, q, k_, v, do, M, scale, where):
    """got = (o, lse, dq, dk, dv) for the heads in q .. do (CPU)."""
    _, lse, _ = R.attention(q, k_, v, M, scale)
    ref, bound = R.attention_grad(q, k_, v, do, M, scale)
    score = (q.shape[-1] + 8) * R.U * abs(scale) * (q.double().abs() @ k_.double().abs().transpose(-1, -2)).amax(-1)
    res = dict(lse=R.worst(got[1], lse, R.HALF[BF] + score + 8 * R.U * lse.abs() + 1e-6))
    for name, g, r, b in zip(("dq", "dk", "dv"), got[2:], ref, bound):
        res[name] = R.worst(g, r, b)
    print(where, {n: round(x, 3) for n, x in res.items()}, flush=True)
    assert all(x <= 1 for x in res.values()), (where, res)


# (mask, B, H, N, k, d_head, std): rows and keys on both sides of the 32-, 64- and 128-row edges, N = 1,
# k = 1, groups that straddle tiles (odd k), groups longer than a tile, every d_head, peaked rows
CASES = [(m, *c) for m in (0, 1) for c in [
    (2, 3, 37, 3, 64, 1.0), (1, 2, 50, 1, 32, 1.0), (1, 2, 64, 4, 128, 1.0), (2, 2, 1, 4, 64, 1.0), (1, 1, 1, 1, 32, 1.0),
    (1, 3, 129, 2, 64, 2.0), (1, 1, 200, 4, 64, 1.0), (1, 2, 70, 5, 64, 1.0), (1, 1, 127, 1, 64, 1.0), (1, 1, 128, 1, 128, 1.0),
    (1, 2, 43, 3, 32, 1.0), (2, 1, 32, 7, 64, 1.0), (1, 1, 9, 40, 64, 1.0), (1, 1, 3, 150, 32, 1.0), (3, 5, 16, 4, 32, 1.0),
    (1, 1, 257, 2, 128, 1.0), (1, 2, 320, 1, 64, 3.0), (1, 1, 31, 8, 128, 2.0)]]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_B%d_H%d_N%d_k%d_dh%d_s%g" % (KIND[c[0]], *c[1:]))
def test_parity(Bd, case):
    mask, B, H, N, k, dh, std = case
    rows, keys = Bd.training_attention_shapes(mask, N, k)
    print(case, rows, keys, flush=True)
    t = _inputs(B, H, rows, keys, dh, N + k, std)
    M = torch.from_numpy(O.training_mask(KIND[mask], N, k)).bool()
    dev = [x.cuda() for x in t]
    got = _run(Bd, mask, *dev, N, k)
    plain = Bd.training_attention(mask, *dev[:3], N, k)
    torch.cuda.synchronize()
    assert torch.equal(got[0], plain)  # the same output, bit for bit
    _check(got, *t, M, dh ** -0.5, str(case))


@pytest.mark.parametrize("scale", [1e-6, 0.4, 1.0])
def test_scales(Bd, scale):
    t = _inputs(1, 2, 60, 60, 32, 5)
    M = torch.from_numpy(O.training_mask("single", 20, 2)).bool()
    got = _run(Bd, 0, *[x.cuda() for x in t], 20, 2, scale)
    torch.cuda.synchronize()
    _check(got, *t, M, scale, f"scale {scale}")


@pytest.mark.parametrize("mask,B,H,N,k,dh", [(0, 4, 12, 512, 4, 64), (1, 2, 8, 512, 4, 64), (1, 2, 4, 300, 3, 128), (0, 64, 12, 128, 4, 64),
                                             (0, 1, 1, 2000, 1, 64), (1, 1, 2, 1024, 4, 32)])
def test_larger_shapes(Bd, mask, B, H, N, k, dh):
    """Training shapes; heads at both ends and in the middle against the formula."""
    rows, keys = Bd.training_attention_shapes(mask, N, k)
    g = torch.Generator(device="cuda").manual_seed(N)
    mk = lambda n: torch.randn(B, H, n, dh, generator=g, device="cuda").to(BF)
    t = [mk(rows), mk(keys), mk(keys), mk(rows)]
    got = _run(Bd, mask, *t, N, k)
    torch.cuda.synchronize()
    assert all(torch.isfinite(x).all() for x in got)
    M = torch.from_numpy(O.training_mask(KIND[mask], N, k)).bool()
    for b, h in {(0, 0), (B - 1, H - 1), (B // 2, H // 3)}:
        _check([x[b, h].cpu() for x in got], *[x[b, h].cpu() for x in t], M, dh ** -0.5, f"b {b} h {h}")


@pytest.mark.parametrize("mask,N,k,dh", [(0, 40, 1, 64), (0, 100, 1, 32), (0, 20, 3, 128), (0, 1, 8, 64), (1, 31, 4, 64), (1, 5, 1, 32), (1, 16, 2, 128)])
def test_equal_answers_have_no_score_gradient(Bd, mask, N, k, dh):
    """Values that differ but give every key the same dO.V (pairs of columns swapped, dO equal on a pair):
    dS is zero everywhere, although O is rounded.  What stays of D after its correction is O's rounding,
    2^-8 of A = sum |dO||V|, times what the forward's sum of bf16 probabilities leaves of 1 - sum P, 2^-8;
    beside it two fp32 sums of d_head products and the row sum."""
    rows, keys = Bd.training_attention_shapes(mask, N, k)
    B, H = 2, 3
    q, k_, _, _ = _inputs(B, H, rows, keys, dh, N)
    g = torch.Generator().manual_seed(N + dh)
    pair = torch.randn(B, H, 1, dh // 2, 2, generator=g).to(BF)
    swap = torch.rand(B, H, keys, dh // 2, 1, generator=g) < 0.5
    v = torch.where(swap, pair.flip(-1), pair).reshape(B, H, keys, dh).contiguous()
    do = torch.randn(B, H, rows, dh // 2, 1, generator=g).to(BF).expand(-1, -1, -1, -1, 2).reshape(B, H, rows, dh).contiguous()
    _, _, dq, dk, _ = _run(Bd, mask, *[x.cuda() for x in (q, k_, v, do)], N, k)
    torch.cuda.synchronize()
    M, scale = torch.from_numpy(O.training_mask(KIND[mask], N, k)).bool(), dh ** -0.5
    P = (q.double() @ k_.double().transpose(-1, -2) * scale).masked_fill(~M, -torch.inf).softmax(-1)
    A = (do.double().abs() @ v.double().abs().transpose(-1, -2)).amax(-1, keepdim=True)
    e = P * A * (2 ** -16 + (4 * dh + M.sum(-1, keepdim=True) + 32) * R.U) * 1.01
    res = [float((x.double().cpu().abs() / (b + 1e-30)).max()) for x, b in
           ((dq, scale * e @ k_.double().abs()), (dk, scale * e.transpose(-1, -2).contiguous() @ q.double().abs()))]
    print(mask, N, k, dh, res, flush=True)
    assert max(res) <= 1.01  # the results' own rounding


def test_gradients_that_vanish(Bd):
    """The first context row sees itself alone: P = 1, its dq is zero up to the rounding of scores
    and D; zero dO gives zero gradients."""
    N, k = 40, 2
    t = [x.cuda() for x in _inputs(1, 2, N + N * k, N + N * k, 64, 1)]
    o, lse, dq, dk, dv = _run(Bd, 0, *t, N, k)
    # dP - D: two fp32 sums of the same 64 products
    lim = 64 * 2 * R.U * float((t[3][:, :, 0].float().abs() * t[2][:, :, 0].float().abs()).sum(-1).max()) * float(t[1][:, :, 0].float().abs().max())
    assert float(dq[:, :, 0].float().abs().max()) <= lim
    z = Bd.training_attention_backward(0, *t[:3], o, lse, torch.zeros_like(o), N, k)
    assert not any(x.any() for x in z)


def test_same_result_on_every_run_and_neighbours_untouched(Bd):
    """Three runs bit for bit; results at the end of a larger buffer leave what follows alone."""
    import ctypes
    mask, B, H, N, k, dh = 1, 1, 3, 45, 3, 64
    rows, keys = Bd.training_attention_shapes(mask, N, k)
    q, k_, v, do = (x.cuda() for x in _inputs(B, H, rows, keys, dh, 2))
    o, lse, *first = _run(Bd, mask, q, k_, v, do, N, k)
    L, p = Bd.lib(), lambda t: ctypes.c_void_p(t.data_ptr())
    n = L.kf_training_attention_backward_bytes(mask, B, H, N, k, dh)
    for _ in range(3):
        bufs = [torch.full((x.numel() + 4096,), 7.0, dtype=BF, device="cuda") for x in first]
        ws = torch.full((n // 4 + 64,), 7.0, device="cuda")
        rc = L.kf_training_attention_backward(torch.cuda.current_stream().cuda_stream, mask, B, H, N, k, dh, p(q), p(k_), p(v), p(o),
                                              p(lse), p(do), p(bufs[0]), p(bufs[1]), p(bufs[2]), dh ** -0.5, p(ws), n)
        assert rc == 0
        torch.cuda.synchronize()
        for a, b in zip(first, bufs):
            assert torch.equal(a.reshape(-1), b[:a.numel()]) and (b[a.numel():] == 7).all()
        assert (ws[n // 4:] == 7).all()


def test_empty_problem(Bd):
    L = Bd.lib()
    for mask in (0, 1):
        assert L.kf_training_attention_lse(None, mask, 0, 2, 8, 4, 64, *[None] * 5, 0.125) == 0
        assert L.kf_training_attention_backward(None, mask, 2, 2, 0, 4, 64, *[None] * 9, 0.125, None, 0) == 0
