"""Training attention of more workgroups than one launch holds is refused before anything is launched: a
launch's threads are counted in 32 bits, 2^24 - 1 workgroups of 256, and what is past them would be
dropped without an error.  No GPU: refusals, and the size query on both sides of the limit."""
import ctypes

import pytest

from paper_2606_10820_amd import binding as Bd

torch = pytest.importorskip("torch")
A = ctypes.c_void_p(0x10000)  # never dereferenced
LIMIT = 1 << 24


def _refused(mask, B, H, N, k, dh, forward=True):
    L = Bd.lib()
    got = [L.kf_training_attention_lse(None, mask, B, H, N, k, dh, *[A] * 5, 0.125),
           L.kf_training_attention_backward(None, mask, B, H, N, k, dh, *[A] * 9, 0.125, A, 1 << 60)]
    if forward:
        got.append(L.kf_training_attention(None, mask, B, H, N, k, dh, *[A] * 4, 0.125))
    return all(rc == Bd.KF_EINVAL for rc in got) and L.kf_training_attention_backward_bytes(mask, B, H, N, k, dh) == 0


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("mask,N,k,blocks", [(0, 1, 1, 1), (0, 1, 127, 1), (0, 100, 2, 3), (0, 1, 400, 4), (1, 1, 1, 1), (1, 40, 3, 2), (1, 128, 4, 8)])
def test_forward(mask, N, k, blocks, dh):
    """`blocks`: of a head, 128 rows each (at these many heads every call has those, or shorter ones)."""
    for B, H in ((-(-LIMIT // blocks), 1), (1 << 12, -(-LIMIT // (blocks << 12))), (1 << 15, 1 << 15)):
        assert _refused(mask, B, H, N, k, dh), (B, H)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("mask,N,k,blocks", [(0, 1, 1, 2), (0, 200, 1, 4), (0, 1, 400, 5), (1, 1, 1, 3), (1, 129, 4, 12)])
def test_gradients(mask, N, k, blocks, dh):
    """`blocks`: of a head, 128 keys each, the context's and each noise region's by themselves.  Accepted
    below that where the forward call's blocks, of 64 query rows at the shortest, fit as well."""
    L, heads = Bd.lib(), -(-LIMIT // blocks)
    assert _refused(mask, heads, 1, N, k, dh, forward=False)
    assert _refused(mask, 1 << 12, -(-heads // (1 << 12)), N, k, dh, forward=False)
    rows = Bd.training_attention_shapes(mask, N, k)[0]
    below = (LIMIT - 1) // max(blocks, -(-rows // 64))
    assert L.kf_training_attention_backward_bytes(mask, below, 1, N, k, dh) == 16 * below * rows
