"""Gradients whose two products share a launch, with tiles of both widths, of either product first, and with results that allow vectors,
pairs and single numbers.  tests/test_ops_plans.py asks the plans for the widths that stand beside the sizes here."""
import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_linear import DTYPES, _product_bound, _randn, _within

pytestmark = pytest.mark.gpu

# M, N, K: columns of a tile; 0: two launches
SIZES = {(3000, 3000, 3001): 256, (5000, 5001, 256): 256, (4500, 4504, 1024): 256, (2900, 3000, 3002): 256, (300, 512, 1024): 128, (1030, 1030, 515): 128,
         (64, 64, 64): 128, (33, 31, 17): 128, (1817, 176, 1808): 128, (200, 200, 4096): 128, (8192, 300, 2048): 0, (8192, 8192, 136): 0, (128, 1024, 256): 0}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", sorted(SIZES))
def test_both_products(M, N, K, dtype):
    dt = DTYPES[dtype]
    half, tiny = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    x, w, dy = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt, scale=K ** -0.5), _randn(M, N, seed=3, dtype=dt, scale=N ** -0.5)
    both = ops.linear_backward(dy, x, w)
    for name, a, b, n in (("dx", dy.double(), w.double(), N), ("dw", dy.T.double(), x.double(), M)):
        alone = ops.linear_backward(dy, x, w, **{k: k == name for k in ("dx", "dw", "db")})[name]
        assert torch.equal(both[name], alone)
        want = a @ b
        bound = _product_bound(a, b, n)
        _within(both[name], want, bound + half * (want.abs() + bound) + tiny, "%s %d x %d x %d" % (name, M, N, K))
    if N % 2 == 0:                     # the gated block's: its dz here is [dh | dh g], of gates of one and no activation
        F = N // 2
        z = torch.cat([_randn(M, F, seed=4, dtype=dt), torch.ones(M, F, device="cuda", dtype=dt)], dim=1)
        dh = dy[:, :F]
        g = ops.gated_backward(dh, x, w, z, activation="none")
        dz = torch.cat([dh, (dh.float() * z[:, :F].float()).to(dt)], dim=1)
        alike = ops.linear_backward(dz, x, w)
        for name, a, b, n in (("dx", dz.double(), w.double(), N), ("dw", dz.T.double(), x.double(), M)):
            want = a @ b
            bound = _product_bound(a, b, n)
            _within(g[name], want, bound + half * (want.abs() + bound) + tiny, name)
            assert SIZES[M, N, K] == 0 or torch.equal(g[name], alike[name])
    ops.check_status()
