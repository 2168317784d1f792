"""qkv_heads' out as one tensor of three, [3][B][H][L][d_head]."""
import pytest

from paper_2606_10820_amd import binding as Bd

torch = pytest.importorskip("torch")


def test_refused_like_any_other():
    """For what is wrong with the call, not for being a tensor (host tensors here)."""
    x, out = torch.zeros(2, 4, 48), torch.zeros(3, 2, 2, 4, 8)
    with pytest.raises(ValueError, match="on a GPU"):
        Bd.qkv_heads(x, 2, out=out)


@pytest.mark.gpu
def test_stacked():
    x = torch.randn(2, 9, 6 * 32, device="cuda").bfloat16()
    want = Bd.qkv_heads(x, 2)
    for stream in (None, torch.cuda.Stream()):
        out = torch.full((3, 2, 2, 9, 32), 7.0, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        q, k, v = Bd.qkv_heads(x, 2, out=out, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, torch.stack(want)) and q.data_ptr() == out.data_ptr() and torch.equal(v, want[2])
    with pytest.raises(ValueError):
        Bd.qkv_heads(x, 2, out=out[:2])
