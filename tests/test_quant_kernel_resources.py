"""Registers and spills of the 4-bit cache's kernels, from ptxas with the library's own flags: every instance keeps to what
its launch is planned for, and none spills more than two words.  Compiles on the CPU; skipped where nvcc is missing."""

import re

import pytest

from tests.test_kernel_resources import resources  # noqa: F401  (a fixture)

# instances, and the registers a thread that their CTAs' number on an SM leaves (65536 over its threads)
INSTANCES = {
    "verify kernel, one CTA of 512 threads": (r"_ZN2bd15quant_tc_kernelILi(64|128)E", 10, 128),
    "its merge, 128 threads": (r"_ZN2bd18quant_merge_kernelILi(64|128)E", 2, 128),
    "mma.sync kernel, 8 rows, 512 threads an SM": (r"_ZN2bd17quant_attn_kernelILi(64|128)ELi1E", 8, 128),
    "mma.sync kernel, 16 rows": (r"_ZN2bd17quant_attn_kernelILi(64|128)ELi2E", 4, 255),
    "rows written": (r"_ZN2bd18quant_write_kernelILi(64|128)E", 4, 64),
    "rows read": (r"_ZN2bd17quant_read_kernelILi(64|128)E", 4, 64),
}
MAX_SPILL_BYTES = 8


@pytest.mark.parametrize("what", sorted(INSTANCES))
def test_instances_keep_to_their_registers(resources, what):  # noqa: F811
    pattern, number, registers = INSTANCES[what]
    hits = {n: k for n, k in resources.items() if re.match(pattern, n)}
    assert len(hits) == number, sorted(hits)
    bad = {n: k for n, k in hits.items() if k["regs"] > registers or k["spill"] > MAX_SPILL_BYTES}
    assert not bad, bad
