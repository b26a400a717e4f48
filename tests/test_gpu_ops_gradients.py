"""Both products of a gradient in one launch: bit for bit what each of them gives by itself, whatever their sizes and addresses."""
import pytest
import torch

from paper_1909_07588_b200 import laq, ops
from tests.test_gpu_ops_linear import DTYPES, _product_bound, _randn, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(3000, 1000, 1500), (2500, 2504, 1032), (4097, 4096, 1030), (1111, 3333, 777), (8192, 300, 2048), (3000, 3000, 3001)])
def test_together_and_apart(M, N, K, dtype):
    dt = DTYPES[dtype]
    half, tiny = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    x, w, dy = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt, scale=K ** -0.5), _randn(M, N, seed=3, dtype=dt, scale=N ** -0.5)
    both = ops.linear_backward(dy, x, w)
    dx, dw = ops.linear_backward(dy, x, w, dw=False, db=False)["dx"], ops.linear_backward(dy, x, w, dx=False, db=False)["dw"]
    assert torch.equal(both["dx"], dx) and torch.equal(both["dw"], dw)
    for got, a, b, n in ((dx, dy, w, N), (dw, dy.T, x, M)):
        want = a.double() @ b.double()
        bound = _product_bound(a.double(), b.double(), n)
        _within(got, want, bound + half * (want.abs() + bound) + tiny, "%d x %d x %d" % (M, N, K))
    ops.check_status()


def test_bounded_wait():
    M, N, K = 3000, 3000, 2048
    x, w, dy = _randn(M, K, seed=1, dtype=torch.bfloat16), _randn(N, K, seed=2, dtype=torch.bfloat16), _randn(M, N, seed=3, dtype=torch.bfloat16)
    before = ops.linear_backward(dy, x, w)
    ops.check_status()
    ops.linear_backward(dy, x, w, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    after = ops.linear_backward(dy, x, w)
    for k in before:
        assert torch.equal(after[k], before[k])
    ops.check_status()
