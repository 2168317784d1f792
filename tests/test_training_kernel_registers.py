"""Register spills of the training step's kernels, from the code objects' own metadata: none beyond the
known ones (attention's dQ walk at d_head 128, which holds Q, dO and dQ of 32 rows in a wavefront, and two
registers of the log probabilities of fp32 rows in eight vectors a lane)."""
import os

import pytest

from tests.test_kernel_registers import LIB, READELF, _kernels

KNOWN = {"training_attention_dq_kernelILi128E": 8, "logprobs_kernelIfLi64ELi8ELb0E": 2, "logprobs_kernelIfLi256ELi8ELb0E": 2}
TRAINING = ("training_attention", "logprobs_kernel", "norm_", "grad_")


@pytest.mark.skipif(not (os.path.exists(LIB) and os.path.exists(READELF)), reason="needs the built library and llvm-readelf")
def test_training_kernels_do_not_spill(tmp_path):
    kernels = [k for k in _kernels(tmp_path) if any(n in k[0] for n in TRAINING)]
    assert len(kernels) > 100
    for name, spilled in kernels:
        assert spilled <= next((v for n, v in KNOWN.items() if n in name), 0), name
