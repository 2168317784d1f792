"""A clipping plan's table outlives the calls that read it, whichever stream they run on: the caching
allocator is told of every stream but the one the table was allocated on (no GPU: the library, the
streams and the allocator's notes are stand-ins)."""
from types import SimpleNamespace

import pytest

from paper_2606_10820_amd import binding as Bd

torch = pytest.importorskip("torch")


@pytest.fixture
def fake(monkeypatch):
    """.now: the current stream; .noted: (address, stream's handle) told to the allocator."""
    f = SimpleNamespace(now=SimpleNamespace(cuda_stream=11), noted=[])

    def on(device, stream, used):  # _on's contract, without a device
        if stream is not None and stream.cuda_stream != f.now.cuda_stream:
            for t in used:
                t.record_stream(stream)
            return stream.cuda_stream, Bd._NOTHING
        return f.now.cuda_stream, Bd._NOTHING

    ok = lambda *a: 0
    monkeypatch.setattr(Bd, "_on", on)
    monkeypatch.setattr(Bd, "lib", lambda: SimpleNamespace(kf_grad_plan_bytes=lambda n, a: 1024, kf_grad_plan_init=ok,
                                                           kf_grad_norm=ok, kf_grad_clip=ok))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: f.noted.append((t.data_ptr(), s.cuda_stream)), raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: f.now)
    return f


@pytest.mark.parametrize("call", [lambda p, s: p.clip(1.0, stream=s), lambda p, s: p.norm(stream=s)], ids=["clip", "norm"])
@pytest.mark.parametrize("given", [False, True], ids=["current", "given"])
def test_table_used_on_another_stream(fake, given, call):
    """Another stream that is the current one, or is named in the call too."""
    plan = Bd.GradClip([torch.zeros(5)])
    call(plan, None)
    assert fake.noted == []  # its own stream
    other = SimpleNamespace(cuda_stream=22)
    fake.now = other
    call(plan, other if given else None)
    assert (plan.buf.data_ptr(), 22) in fake.noted


def test_table_used_on_a_named_stream(fake):
    grads = [torch.zeros(5), torch.zeros(7)]
    plan = Bd.GradClip(grads)
    plan.clip(1.0, stream=SimpleNamespace(cuda_stream=33))
    assert {(t.data_ptr(), 33) for t in (plan.buf, *grads)} <= set(fake.noted)


def test_table_built_on_a_named_stream(fake):
    """The current stream is then the other one."""
    s = SimpleNamespace(cuda_stream=44)
    plan = Bd.GradClip([torch.zeros(5)], stream=s)
    fake.noted.clear()
    plan.clip(1.0, stream=s)
    assert all(at != 11 for _, at in fake.noted)
    plan.clip(1.0)
    assert (plan.buf.data_ptr(), 11) in fake.noted
