"""Registers and spills of the paged cache's kernels, from ptxas with the library's own flags: every instance keeps to what its
launch is planned for, and none spills more than a few words.  Compiles on the CPU; skipped where nvcc is missing."""

import re

import pytest

from tests.test_kernel_resources import resources  # noqa: F401  (a fixture)

# instances, their number, the registers a thread that their CTAs' number on an SM leaves, bytes that may be spilled
INSTANCES = {
    "rows appended, four CTAs of 256 threads an SM": (r"_ZN2bd19paged_append_kernelILi(64|128)E", 4, 64, 0),
    "rows read": (r"_ZN2bd17paged_read_kernelILi(64|128)E", 2, 64, 0),
    "verify kernel, clusters, two CTAs of 256 threads an SM": (r"_ZN2bd19paged_verify_kernelILi(64|128)ELi1ELb1E", 2, 128, 0),
    "verify kernel, stream, two CTAs of 192 threads an SM at head_dim 64": (r"_ZN2bd19paged_verify_kernelILi64ELi[13]ELb0E", 2, 168, 0),
    "verify kernel, stream, head_dim 128": (r"_ZN2bd19paged_verify_kernelILi128ELi1ELb0E", 1, 255, 0),
    "tcgen05 verify kernel over pages, 352 threads": (r"_ZN2bd16verify_tc_kernelILi(64|128)ELi[12]ELb0ELi[12]E", 6, 168, 32),
    "drafter pass over pages": (r"_ZN2bd12draft_kernelILi(64|128)ELi\d+ELb[01]ELb1E", 20, 204, 32),
}


@pytest.mark.parametrize("what", sorted(INSTANCES))
def test_instances_keep_to_their_registers(resources, what):  # noqa: F811
    pattern, number, registers, spill = INSTANCES[what]
    hits = {n: k for n, k in resources.items() if re.match(pattern, n)}
    assert len(hits) == number, sorted(hits)
    bad = {n: k for n, k in hits.items() if k["regs"] > registers or k["spill"] > spill}
    assert not bad, bad
