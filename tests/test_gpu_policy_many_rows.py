"""The policy loss of more rows than a launch has workgroups (2^20, of 16 rows each where rows are narrow):
rows of the second pass, ignored ones among them, against 64 bits (bounds: tests/step_ref.py)."""
import math

import pytest

from tests import step_ref as S
from tests import train_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32, BF = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("grad", [True, False], ids=["gradient", "loss"])
@pytest.mark.parametrize("rows,V,t,first", [(2 ** 20 + 1501, 4105, BF, 2 ** 20), (2 ** 24 + 70_003, 17, F32, 2 ** 24)], ids=["256 threads", "16 lanes"])
def test_second_pass(Bd, rows, V, t, first, grad):
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.empty(rows, V, dtype=t, device="cuda")
    x.normal_(generator=g)
    rnd = lambda: torch.randn(rows, generator=g, device="cuda")
    tok = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    adv, old = rnd(), 0.3 * rnd() - math.log(V)
    ref, w = old + 0.3 * rnd(), 0.5 + rnd().abs()
    tok[3::7], w[5::11] = -1, 0.0
    at = torch.tensor([*range(12), *range(first - 12, first + 12), *range(first + 1400, first + 1412), *range(rows - 12, rows)], device="cuda")
    keep = [v[at].cpu() for v in (x, tok, adv, old, ref, w)]
    # no clipping: at a border of it the two sides may differ by a whole row's gradient
    r = Bd.policy_loss(x, tok, adv, old, ref, w, clip_low=1.0, clip_high=math.inf, kl_coef=0.125, entropy_coef=0.0625, grad=grad, out=x if grad else None)
    want = S.policy(*keep, 0.0, math.inf, 0.125, 0.0625)
    names = ["row_loss", "logp", "ratio", "entropy", "kl"] + (["d_logits"] if grad else [])
    got = {n: R.worst(getattr(r, n)[at], want[n], want[n + "_b"]) for n in names}
    print({n: round(v, 3) for n, v in got.items()}, flush=True)
    assert all(v <= 1 for v in got.values()), got
    off = ~want["on"]
    assert off.sum() >= 8 and not any(getattr(r, n)[at].cpu()[off].any() for n in names)
    rl = r.row_loss.double()
    assert abs(float(r.loss) - float(rl.sum())) <= R.U * abs(float(r.loss)) + 2.0 ** -40 * float(rl.abs().sum())
