"""Registers, scratch and LDS of the gated-delta layer's kernels, from the
library's own code objects: a spilled register in the chain over blocks waits
for the loads in flight, which no parity test shows."""
import os

import msgpack
import pytest

from paper_2608_02560_amd import build
from test_kernel_resources import _code_objects, _notes, _pick


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(build.LIB):
        build.build()
    with open(build.LIB, "rb") as f:
        data = f.read()
    return {k[".name"]: k for elf in _code_objects(data) for note in _notes(elf)
            for k in msgpack.unpackb(note)["amdhsa.kernels"]}


def test_delta_kernels(kernels):
    """Two waves a SIMD for a workgroup of eight, nothing in scratch, the LDS of a CU."""
    got = _pick(kernels, r"12delta_kernelILi(64|128)E")
    assert len(got) == 24
    for name, k in got.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_count"] <= 256, name
        assert k[".group_segment_fixed_size"] <= 160 * 1024, name


def test_memory_bound_kernels(kernels):
    for pattern, most in ((r"11conv_kernelI", 128), (r"12score_kernelI", 128), (r"17delta_step_kernelI", 144)):
        for name, k in _pick(kernels, pattern).items():
            assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_count"] <= most, (name, k[".vgpr_count"])
