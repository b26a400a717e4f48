"""Gradients of gated blocks of more columns than the SMs hold blocks for at once, and of very many rows."""
import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_linear import U, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M, F, packed", [(700, 57_344, False), (90, 60_001, False), (300, 38_401, True), (200_000, 264, False), (70_001, 130, True)])
def test_column_sums(M, F, packed):
    """A thread adds up 256 products one after another at most (u of the sum of magnitudes for each), eight threads a run (8 u), and 32
    threads of the runs (their number over 32, and 5 u); a product of three has 2 u, an up or a gate without an activation none."""
    dh, z = _randn(M, F, seed=1, dtype=torch.bfloat16), _randn(M, 2 * F, seed=2, dtype=torch.bfloat16)
    w, x = torch.zeros(2 * F, 8, device="cuda", dtype=torch.bfloat16), torch.zeros(M, 8, device="cuda", dtype=torch.bfloat16)
    if packed:
        z = ops.pack8(z)
    db = ops.gated_backward(dh, x, w, z, activation="none", dx=False, dw=False)["db"].double()
    z = ops.unpack8(z) if packed else z
    for c0 in range(0, F, 8192):
        c1 = min(c0 + 8192, F)
        d = dh[:, c0:c1].double()
        for at, v in ((c0, z[:, F + c0:F + c1].double()), (F + c0, z[:, c0:c1].double())):
            want, size = (d * v).sum(0), (d * v).abs().sum(0)
            assert bool(((db[at:at + c1 - c0] - want).abs() <= (256 + 8 + M / 32 / 32 + 5 + 2) * U * size + 1e-30).all())
    ops.check_status()
