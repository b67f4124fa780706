"""The generator against its authors' published outputs for a counter and a key whose words all differ, so that a swapped word shows, and the place of
each half of a draw: key = seed, counter = (column group, row, offset)."""
import pytest

import act_util as au

PI = ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0])
ONES = ([0xffffffff] * 4, [0xffffffff] * 2)


@pytest.mark.parametrize("rounds,counter_and_key,want", [
    (7, ONES, "5207ddc2 45165e59 4d8ee751 8c52f662"),
    (7, PI, "4dfccaba 190a87f0 c47362ba b6b5242a"),
    (10, ONES, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
    (10, PI, "d16cfe09 94fdcceb 5001e420 24126ea1"),
])
def test_published_outputs(rounds, counter_and_key, want):
    assert " ".join(f"{v:08x}" for v in au.philox(*counter_and_key, rounds)) == want


def test_halves_of_large_rows_and_unlike_words():
    """Row, seed and offset as in the block above: each half is where the published order puts it."""
    (_, row, low, high), (k0, k1) = PI
    h = au.halves(k0 | k1 << 32, low | high << 32, 2, 24, first_row=row)
    for r in range(2):
        for c in range(24):
            w = au.philox([c // 8, row + r, low, high], [k0, k1])[c % 8 // 2]
            assert h[r, c] == (w >> 16 if c % 2 else w & 0xFFFF)
