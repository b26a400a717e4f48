"""The pitch of a matrix of one row is of no account: an 8-bit product of it needs no copy."""
import ctypes as C

from paper_1909_07588_b200 import build, laq

A = 1 << 20


def _need(M, N, K, x_at=A, w_at=2 * A, w_pitch=None):
    c = laq.laq_linear_call()
    c.dtype, c.M, c.N, c.K, c.flags = 1, M, N, K, 1                # by tiles, which want rows at multiples of 16 bytes
    x = laq.laq_blocks(x_at, K, 3 * A, -(-K // 128), 1)
    w = laq.laq_blocks(w_at, w_pitch or K, 4 * A, -(-K // 128), 128)
    return laq.load_library().laq_linear_blocks_workspace_bytes(C.byref(c), C.byref(x), C.byref(w), 0)


def test_one_row_is_not_copied():
    build.build()
    up = lambda n: -(-n // 256) * 256
    assert _need(1, 48, 200, w_pitch=208) == 0 and _need(1, 1, 200) == 0 and _need(1, 1, 7) == 0
    assert _need(2, 48, 200, w_pitch=208) == up(2 * 208) and _need(1, 48, 200) == up(48 * 208)
    assert _need(1, 1, 200, x_at=A + 1) == 256 and _need(1, 1, 200, w_at=2 * A + 8) == 256
