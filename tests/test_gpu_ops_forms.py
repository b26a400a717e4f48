"""The gated block and the 8-bit product in every form that their plans give them: pairs of SMs, lone ones, transposed tiles, each width,
whole and split sums.  tests/test_ops_plans.py asks the plans for the forms that stand beside the sizes here."""
import math

import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_blocks import _check8, _pair
from tests.test_gpu_ops_gated import _check
from tests.test_gpu_ops_linear import DTYPES, _randn

pytestmark = pytest.mark.gpu

# M, F, K: (form, columns of a tile, blocks that share a sum)
GATED = {
    (4097, 5504, 2048): ("pair", 256, 1), (4097, 5501, 2047): ("pair", 256, 1), (6359, 207, 2391): ("pair", 256, 1),
    (155, 2415, 2154): ("pair", 128, 1), (160, 2432, 2152): ("pair", 128, 1),
    (300, 72, 40): ("lone", 64, 1), (1094, 8, 916): ("lone", 64, 8), (1218, 9, 1035): ("lone", 64, 4),
    (1024, 768, 2048): ("lone", 128, 1), (73, 1664, 1848): ("lone", 128, 4), (66, 1564, 1503): ("lone", 128, 4),
    (2500, 1100, 600): ("lone", 192, 1), (40, 5688, 3590): ("lone", 192, 2), (39, 1069, 14456): ("lone", 192, 8),
    (2304, 4352, 136): ("lone", 256, 1), (146, 9427, 8): ("lone", 256, 1), (77, 3376, 3064): ("lone", 256, 4), (141, 782, 6907): ("lone", 256, 8),
    (6, 5369, 9): ("transposed", 16, 1), (40, 24, 1000): ("transposed", 16, 8), (551, 8, 1232): ("transposed", 32, 4), (48, 1125, 2804): ("transposed", 64, 4),
    (2192, 46, 9717): ("transposed", 96, 4), (8013, 34, 7097): ("transposed", 112, 2), (1603, 652, 11092): ("transposed", 128, 1),
    (4551, 81, 8954): ("transposed", 128, 2),
}
# M, N, K
LINEAR8 = {
    (4097, 2304, 128): ("pair", 256, 1), (3000, 2304, 100): ("pair", 256, 1), (5000, 4000, 1100): ("pair", 256, 1),
    (155, 4797, 921): ("pair", 128, 1), (160, 4800, 1100): ("pair", 128, 1),
    (300, 72, 40): ("lone", 64, 1), (40, 10298, 9): ("lone", 128, 1), (5, 10298, 8): ("lone", 128, 1),
    (40, 13, 1500): ("transposed", 16, 4), (595, 10, 1288): ("transposed", 32, 4), (1445, 9, 2941): ("transposed", 64, 4), (38, 10289, 6752): ("transposed", 64, 1),
    (2463, 9, 3468): ("transposed", 96, 4), (71, 9975, 13139): ("transposed", 96, 1), (3346, 8, 6020): ("transposed", 112, 4),
    (7191, 11, 8512): ("transposed", 112, 2), (3820, 9, 6464): ("transposed", 128, 4), (8938, 10, 5324): ("transposed", 128, 2),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, F, K", sorted(GATED))
def test_gated(M, F, K, dtype):
    dt = DTYPES[dtype]
    x, w, b = _randn(M, K, seed=1, dtype=dt), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5), _randn(2 * F, seed=3, dtype=dt)
    x[M // 2] = 0
    x[M - 1] *= 2.0 ** -8
    _check(x, w, None, "silu")
    _check(x, w, b, "gelu")
    far = b.clone()
    far[F // 2], far[F], far[2 * F - 1] = math.inf, -math.inf, math.nan
    for bias in (None, b, far):
        h, z = ops.gated(x, w, bias, activation="relu", preact=True)
        h8, z8 = ops.gated(x, w, bias, activation="relu", preact="packed")
        want = ops.pack8(z)
        assert torch.equal(h8.view(torch.int16), h.view(torch.int16)) and torch.equal(ops.gated(x, w, bias, activation="relu").view(torch.int16), h.view(torch.int16))
        assert torch.equal(z8.scales, want.scales) and torch.equal(z8.codes.view(torch.uint8), want.codes.view(torch.uint8))
    # among other numbers, which stay as they are
    big = _randn(M + 2, F + 6, seed=5, dtype=dt)
    before, inside = big.clone(), big[1:1 + M, 3:3 + F]
    got, _ = _check(x, w, b, "silu", out=inside)
    assert got is inside
    mark = torch.ones_like(big, dtype=torch.bool)
    mark[1:1 + M, 3:3 + F] = False
    assert torch.equal(big[mark], before[mark])
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", sorted(LINEAR8))
def test_linear8(M, N, K, dtype):
    dt = DTYPES[dtype]
    x, w = _pair(M, N, K)
    if M <= 32:                        # in order so few rows go by other kernels
        x = ops.Packed8(torch.nn.functional.pad(x.codes.view(torch.uint8), (1, 2)).view(torch.float8_e4m3fn)[:, 1:-2], x.scales)
    b, r = _randn(N, seed=3, dtype=dt), _randn(M, N, seed=4, dtype=dt)
    _check8(x, w, None, "none", None, dt, preact=False)
    y = _check8(x, w, b, "gelu", r, dt)
    big = _randn(M + 2, N + 6, seed=5, dtype=dt)
    before, inside = big.clone(), big[1:1 + M, 3:3 + N]
    assert torch.equal(ops.linear8(x, w, b, activation="gelu", residual=r, dtype=dt, out=inside), y)
    mark = torch.ones_like(big, dtype=torch.bool)
    mark[1:1 + M, 3:3 + N] = False
    assert torch.equal(big[mark], before[mark])
    over = r.clone()
    assert torch.equal(ops.linear8(x, w, b, activation="gelu", residual=over, dtype=dt, out=over), y)
    # a code that is no number spoils its row, or its column, and no other
    x.codes.view(torch.uint8)[M // 2, K - 1] = 0x7f
    w.codes.view(torch.uint8)[N // 2, 0] = 0xff
    got = ops.linear8(x, w, b, activation="gelu", residual=r, dtype=dt)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[M // 2] = True
    bad[:, N // 2] = True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], y[~bad])
    ops.check_status()
