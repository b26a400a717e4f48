"""Runs of rows whose column sums a gated gradient adds up first, seen by the workspace that their sums take."""
import ctypes as C

import pytest

from paper_1909_07588_b200 import build, laq

PLACES = {False: 3 * 148, True: 2 * 148}        # blocks of 256 columns that the SMs hold at once; True: 8-bit projections at odd places


@pytest.fixture(scope="module")
def lib():
    build.build()
    return laq.load_library()


def _runs(lib, M, F, odd=False):
    c = laq.laq_gated_call()
    c.dtype, c.activation, c.M, c.F, c.K = 1, 3, M, F, 8
    c.dh, c.ld_dh, c.z, c.ld_z, c.db = 4096, F, 4096, 2 * F, 4096
    if odd:
        q = laq.laq_blocks(4097, 2 * F, 4096, 2 * F // 128, 1)
        c.z, c.z_blocks = None, C.pointer(q)
    return lib.laq_gated_workspace_bytes(C.byref(c), 1) // (2 * F * 4)


@pytest.mark.parametrize("M, F, odd", [(8192, 4096, False), (8192, 57344, False), (1 << 20, 4096, False), (1 << 20, 128, False), (20_000, 120_064, False),
                                       (4096, 37_888 + 256, True), (8192, 38_400, False), (100_000, 1024, True)])
def test_runs_fill_the_gpu_and_stay_short(lib, M, F, odd):
    runs, cols = _runs(lib, M, F, odd), -(-F // 256)
    per = -(-M // runs)
    assert per <= 2048
    rounds = -(-cols * runs // PLACES[odd])
    assert cols * runs >= 0.65 * rounds * PLACES[odd]


def test_runs_of_ordinary_sizes(lib):
    """As many as the SMs hold, of 32 rows at least."""
    assert _runs(lib, 8192, 4096) == 27 and _runs(lib, 64, 4096) == 2 and _runs(lib, 1, 32) == 1 and _runs(lib, 0, 32) == 0
