"""A gradient of the gated block has the same bits whichever of its results are asked for."""
import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_linear import DTYPES, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, F, K", [(128, 512, 256), (300, 1024, 1024), (1024, 64, 64), (2048, 1024, 256), (16, 512, 256), (4096, 512, 1024),
                                     (2048, 1024, 128), (301, 1021, 777)])
def test_each_result_by_itself(M, F, K, dtype):
    """Sizes at which one of the products, by itself, has its sum split over several blocks, and one at which none has."""
    dt = DTYPES[dtype]
    x, w, dh, z = _randn(M, K, seed=1, dtype=dt), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5), _randn(M, F, seed=3, dtype=dt), _randn(M, 2 * F, seed=4, dtype=dt)
    for kept in (x, ops.pack8(x)):
        every = ops.gated_backward(dh, kept, w, z)
        for some in (("dx",), ("dw",), ("db",), ("dx", "dw"), ("dx", "db"), ("dw", "db")):
            got = ops.gated_backward(dh, kept, w, z, **{k: k in some for k in every})
            assert set(got) == set(some)
            for k in some:
                assert torch.equal(got[k], every[k]), (some, k)
    ops.check_status()
