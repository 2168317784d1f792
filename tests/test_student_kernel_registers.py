"""Registers of the student's operators, from the code objects' own metadata: no spills, and no scratch
memory (an array that a run-time choice indexes goes there: dropout of odd widths took 1.6 times as long)."""
import os
import re
import struct
import subprocess

import pytest

from tests.test_kernel_registers import LIB, MAGIC, READELF, _kernels

OURS = ("heads_kernel", "heads_grad_kernel", "heads_gain_kernel", "rope_table_kernel", "dropout_kernel", "dropout_flat_kernel", "DropNormArgs", "DropNormGradArgs",
        "PolicyArgs", "policy_sum_kernel")


def _scratch(tmp_path):
    """{name: bytes of scratch memory a lane} of every kernel in the library."""
    data, found, at = open(LIB, "rb").read(), {}, 0
    while (at := data.find(MAGIC, at)) >= 0:
        p = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            off, size, n = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + n].decode()
            p += 24 + n
            if "gfx950" in target:
                f = tmp_path / f"s{at}.co"
                f.write_bytes(data[at + off:at + off + size])
                notes = subprocess.run([READELF, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
                names = re.findall(r"^    \.name: +(\S+)", notes, re.M)
                sizes = re.findall(r"\.private_segment_fixed_size: +(\d+)", notes)
                assert len(names) == len(sizes)
                found.update(zip(names, map(int, sizes)))
        at += len(MAGIC)
    return found


@pytest.mark.skipif(not (os.path.exists(LIB) and os.path.exists(READELF)), reason="needs the built library and llvm-readelf")
def test_student_kernels_keep_to_registers(tmp_path):
    ours = [k for k in _kernels(tmp_path) if any(n in k[0] for n in OURS)]
    assert len(ours) > 150 and all(any(n in k[0] for k in ours) for n in OURS)
    assert [k for k in ours if k[1]] == []
    assert {n: b for n, b in _scratch(tmp_path).items() if b and any(o in n for o in OURS)} == {}
