"""Gradient of masked logits (minus infinity, the type's lowest value) for entropy weights of any size,
against 64 bits (bounds: tests/train_ref.py): a probability of zero has a gradient of zero."""
import math

import pytest

from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


def _rows(V, t):
    """Masked rows, spread and peaked (the sum of exponentials at its least, 1)."""
    g = torch.Generator().manual_seed(V)
    x = 2.5 * torch.randn(10, V, generator=g)
    low = torch.finfo(t).min
    x[0, ::2] = -math.inf
    x[1, 1::2] = low
    x[2] = -math.inf
    x[2, V // 2] = 1.5  # one id left
    x[3] = low
    x[3, 7] = 0.0
    x[4, 3:] = -math.inf
    x[4, 0] += 40.0  # peaked: the others of the three have a probability near zero
    x[5, ::2] = low
    x[5, V - 1] = 60.0
    x[6] = low  # nothing but the lowest value: all alike
    x[7, V - 9:] = -math.inf
    x[7, :3] = low
    x[8] = -math.inf  # nothing
    tok = torch.randint(0, V, (10,), generator=g, dtype=torch.int32)
    tok[0], tok[1], tok[2], tok[3], tok[4], tok[5], tok[9] = 0, 1, V // 2, 5, 0, V - 1, -1
    u = torch.randn(10, generator=g)
    sign = torch.tensor([1.0, -1.0] * 5)
    return x.to(t), tok, u, sign


@pytest.mark.parametrize("t", [F32, BF, HF], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("V", [70, 1000, 3000, 30522, 140001])
def test_entropy_weights_of_any_size(Bd, V, t):
    x, tok, u, sign = _rows(V, t)
    X, T, U = x.cuda(), tok.cuda(), u.cuda()
    # fp16 holds gradients up to 65504: |p (log p + H)| < 4
    for c in (0.0, 1.5, 2.0, 64.0, 1e4) + ((65536.0, 1e30) if t != HF else ()):
        for given in (u, None):
            d, _ = Bd.token_logprobs_backward(X, T, U if given is not None else None, (c * sign).cuda())
            ref, b = R.logprobs_grad(x, tok, given, c * sign)
            got = R.worst(d, ref, b)
            print(V, t, c, given is not None, round(got, 3), flush=True)
            assert got <= 1, (c, given is not None)
    ref, b = R.logprobs_grad(x, tok, u, None)
    assert R.worst(Bd.token_logprobs_backward(X, T, U)[0], ref, b) <= 1
