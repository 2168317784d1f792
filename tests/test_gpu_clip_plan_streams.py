"""A clipping plan used on another stream than its own and dropped while that one still runs: its
table's memory is not handed out before the call has read it."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def Bd():
    from paper_2606_10820_amd import binding
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return binding


@pytest.mark.parametrize("named", [False, True])
def test_plan_dropped_under_a_call(Bd, named):
    grads = [torch.full((1000 + i,), 0.25 * (i + 1), device="cuda") for i in range(40)]
    out = [torch.zeros_like(g) for g in grads]
    plan = Bd.GradClip(grads, out)
    size, table = plan.buf.numel(), range(plan.buf.data_ptr(), plan.buf.data_ptr() + plan.buf.numel())
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        torch.cuda._sleep(20_000_000)  # the call waits behind it
        norm = plan.clip(1.0, stream=other if named else None)
        done = torch.cuda.Event()
        done.record()
    del plan
    fresh = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(16)]
    assert not done.query()  # still running when they were handed out
    assert not any(t.data_ptr() in table for t in fresh)
    for t in fresh:
        t.fill_(0)
    torch.cuda.synchronize()
    want = float(torch.stack([(g.double() ** 2).sum() for g in grads]).sum().sqrt())
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for g, o in zip(grads, out):
        assert torch.allclose(o, g / want, rtol=2.0 ** -21, atol=0)
