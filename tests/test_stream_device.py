"""A stream of another device than the tensors' is refused, also where both are default streams, whose
handles are equal (no GPU: torch's view of the devices is a stand-in)."""
from types import SimpleNamespace

import pytest

from paper_2606_10820_amd import binding as Bd

torch = pytest.importorskip("torch")


def test_stream_of_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(Bd, "_current_device", lambda: 0)
    monkeypatch.setattr(Bd, "_current_raw", lambda i: 0)
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    for handle in (0, 7):
        with pytest.raises(ValueError, match="another device"):
            Bd._on(here, SimpleNamespace(cuda_stream=handle, device=there), ())
    raw, ctx = Bd._on(here, SimpleNamespace(cuda_stream=0, device=here), ())
    assert raw == 0 and ctx is Bd._NOTHING
