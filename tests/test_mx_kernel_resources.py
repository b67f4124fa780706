"""Registers of the block-scaled kernels, from the compiler's figures that the build leaves next to the library: none uses scratch
memory but the largest 4-bit tiles, a few dwords outside their loop (every value of the loop is in registers: a reload there
would wait for all requests before it), and no workgroup asks for more LDS than there is."""
import os

import pytest

OUTSIDE_THE_LOOP = {"mx_ring_kernel<1, 1, 256, 256, 2, 4, 2, unsigned short>": 64, "mx_ring_kernel<1, 1, 256, 256, 2, 4, 2, float>": 64}


def test_block_scaled_kernels_do_not_spill():
    from paper_2401_11469_amd import build
    if not os.path.exists(build.RESOURCES):
        pytest.skip("no resource table (library not built by build.py here)")
    rows = [l.rstrip("\n").split(" | ") for l in open(build.RESOURCES) if not l.startswith("#")]
    for kind, least in (("mx_rows_kernel<", 6), ("mx_gather_kernel<", 30), ("mx_long_kernel<", 6), ("mx_cols_kernel<", 12), ("mx_values_kernel<", 12),
                        ("mx_kernel<", 8), ("mx_ring_kernel<", 16), ("mx_few_kernel<", 24)):
        mine = [r for r in rows if r[0].startswith(kind)]
        assert len(mine) >= least, (kind, len(mine))
        for name, vgpr, agpr, scratch, occ, lds in mine:
            assert int(scratch) <= OUTSIDE_THE_LOOP.get(name, 0), (name, scratch)
            assert int(lds) <= 160 * 1024, (name, lds)
