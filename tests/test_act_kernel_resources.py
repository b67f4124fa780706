"""Registers of the kernels around a block's products, from the compiler's figures that the build leaves next to the library: none uses
scratch memory but the joins' backward kernels of more than 4096 columns (no room for a row and its sums), and no workgroup asks for more LDS than
there is."""
import os
import re

import pytest


def wide_join(name):
    m = re.match(r"join_(back_)?kernel<[a-z ]+, (\d+), (\d+)", name)
    return bool(m) and int(m[2]) * int(m[3]) > 512


def test_kernels_around_the_products_do_not_spill():
    from paper_2401_11469_amd import build
    if not os.path.exists(build.RESOURCES):
        pytest.skip("no resource table (library not built by build.py here)")
    rows = [l.rstrip("\n").split(" | ") for l in open(build.RESOURCES) if not l.startswith("#")]
    for kind, least in (("act_fast_kernel<", 12), ("act_slice_kernel<", 3), ("act_reduce_kernel", 1), ("act_kernel<", 20), ("f32_act_kernel<", 20),
                        ("act_few_rows_kernel<", 24), ("act_few_cols_kernel<", 9), ("act_back_kernel<", 3), ("dropout_kernel<", 2), ("sum_slabs_kernel<", 2), ("join_sums_kernel<", 2),
                        ("join_kernel<", 40), ("join_back_kernel<", 100)):
        mine = [r for r in rows if r[0].startswith(kind)]
        assert len(mine) >= least, (kind, len(mine))
        for name, vgpr, agpr, scratch, occ, lds in mine:
            assert int(scratch) == 0 or wide_join(name), (name, scratch)
            assert int(lds) <= 160 * 1024, (name, lds)
