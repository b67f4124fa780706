"""Which kernels a forward product with bias, activation and so on is sent to, asked of the built library on the CPU (launch_util.py)."""
import pytest

from launch_util import launches

NARROW = "act_kernel<Plain, true, Plain, false, 32, 256>"


def names(tmp_path, calls):
    return [[n.split("(")[0] for n, _ in c] for c in launches(tmp_path, calls)]


@pytest.mark.parametrize("M,N", [(8192, 2064), (8192, 2112), (16384, 1056)])
def test_columns_behind_a_panel_of_a_short_contraction(tmp_path, M, N):
    """Fewer kept columns than the 16-byte loads of the 32 x 32 tiles take (8) stay off those tiles: row 0 would be read from before its first
    element, which is that of the caller's workspace."""
    kept = [1, 2, 5, 7, 8, 9, 64]
    for n, got in zip(kept, names(tmp_path, [dict(M=M, K=96, N=N, n_keep=n, mode_k=True, kn=True, scratch=True) for n in kept])):
        assert got[1] == "act_fast_kernel<RingP, RingQM, 256, 256, 2, 4>", got
        assert got[2] == (NARROW if n >= 8 else "act_fast_kernel<DmaP, DmaQM, 128, 128, 2, 2>"), (n, got)


def test_no_short_contraction_reaches_loads_of_eight(tmp_path):
    """Any size, layout and mode: Plain along the contraction needs eight indices there."""
    calls = [dict(M=M, K=K, N=N, n_keep=n, mode_k=True, kn=kn, scratch=scratch)
             for M in (1, 4, 5, 16, 17, 40, 300, 4096, 8192) for K in (7, 8, 96, 97) for N in (3, 8, 65, 1000, 1032, 2056, 2064, 4104, 8200)
             for n in (1, 4, 7) for kn in (True, False) for scratch in (True, False)]
    for c, got in zip(calls, names(tmp_path, calls)):
        assert got and not any("Plain, true" in g for g in got), (c, got)


@pytest.mark.parametrize("C,pieces", [(1096, 1), (1264, 1), (1336, 1), (1280, 2), (1344, 2), (1400, 2)])
def test_slices_by_the_rules_of_the_plain_product(tmp_path, C, pieces):
    """216 tiles of 128 x 128: the contraction is cut in two with scratch where it is whole stages of 64 or at least 1344 long."""
    call = dict(M=1536, K=C, N=2304, n_keep=None, mode_k=False, kn=False)
    one, two = names(tmp_path, [dict(call, scratch=False), dict(call, scratch=True)])
    assert one == ["act_fast_kernel<DmaP, DmaP, 64, 128, 1, 4>"]
    assert two == (one if pieces == 1 else ["act_slice_kernel<DmaP, DmaP>", "act_reduce_kernel"])
