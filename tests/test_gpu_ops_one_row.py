"""The 8-bit product of single rows and single columns whose lengths are no multiples of 16."""
import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_blocks import _check8, _pair
from tests.test_gpu_ops_linear import DTYPES, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(1, 100, 7), (1, 48, 200), (1, 4096, 1000), (1, 300, 4095), (1, 1, 129), (2, 1, 200), (8, 1, 1000), (300, 1, 777), (40, 1, 7)])
def test_single_rows(M, N, K, dtype):
    dt = DTYPES[dtype]
    x, w = _pair(M, N, K)
    b, r = _randn(N, seed=3, dtype=dt), _randn(M, N, seed=4, dtype=dt)
    for act in ("none", "silu"):
        _check8(x, w, b, act, r, dt)
    # rows that stand alone between others, with NaN behind them
    among = lambda p: torch.nn.functional.pad(p.codes.view(torch.uint8), (16, 3, 1, 1), value=0x7f).view(torch.float8_e4m3fn)[1:-1, 16:16 + K]
    _check8(ops.Packed8(among(x), x.scales), ops.Packed8(among(w), w.scales), b, "silu", r, dt)
    y = ops.linear8(x, w, b, dtype=dt)
    if M > 8:                          # by tiles
        odd = ops.linear8(ops.Packed8(among(x), x.scales), ops.Packed8(among(w), w.scales), b, dtype=dt)
        assert torch.equal(odd, y)
    ops.check_status()


def test_a_wait_that_runs_out_on_one_row():
    x, w = _pair(1, 300, 1000)
    ops.linear8(x, w, flags=ops.LINEAR_STARVE)
    with pytest.raises(Exception, match="bounded wait"):
        ops.check_status()
    _check8(x, w, None, "none", None, torch.bfloat16)
    ops.check_status()
