"""Values in 8 bits that fp16 cannot hold, and gradients that leave its range: what the calls say of them."""
import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_blocks import values
from tests.test_gpu_ops_linear import _product_bound, _randn, _within

pytestmark = pytest.mark.gpu


def _far(rows, cols, seed, scale, tiles=False):
    p = ops.pack8(_randn(rows, cols, seed=seed, dtype=torch.float32), tiles=tiles)
    p.scales.mul_(scale)
    return p


@pytest.mark.parametrize("scale", [2.0 ** 18, 2.0 ** -20, 2.0 ** -40])
def test_gradient_takes_what_unpack8_gives(scale):
    M, N, K = 70, 40, 200
    x, w, dy = _far(M, K, 1, scale), _far(N, K, 2, 1 / scale, tiles=True), _randn(M, N, seed=3, dtype=torch.float16)
    restored = ops.unpack8(x, dtype=torch.float16)
    want = values(x).clamp(-65504, 65504).to(torch.float16)
    assert torch.equal(restored, want) and not torch.equal(restored.double(), values(x))
    got, plain = ops.linear_backward(dy, x, w), ops.linear_backward(dy, restored, ops.unpack8(w, dtype=torch.float16))
    for k in got:
        assert torch.equal(got[k].view(torch.int16 if got[k].dtype == torch.float16 else torch.int32), plain[k].view(torch.int16 if plain[k].dtype == torch.float16 else torch.int32)), k
    # bfloat16 holds every value: there it is the gradient of what linear8 computes
    dy = dy.bfloat16()
    got = ops.linear_backward(dy, x, w)
    half = 2.0 ** -8
    for name, a, b, n in (("dx", dy.double(), values(w), N), ("dw", dy.double().T, values(x), M)):
        bound = _product_bound(a, b, n)
        _within(got[name], a @ b, bound + half * ((a @ b).abs() + bound), name)


def test_gated_gradient_beyond_fp16():
    """dh and z of a few hundred: dh z is not a number of fp16.  db, summed before the rounding, is."""
    M, F, K = 40, 24, 48
    dh, z = torch.full((M, F), 300.0, device="cuda").half(), torch.full((M, 2 * F), 400.0, device="cuda").half()
    x, w = torch.ones(M, K, device="cuda").half(), torch.ones(2 * F, K, device="cuda").half()
    got = ops.gated_backward(dh, x, w, z, activation="none")
    assert bool(got["dx"].isinf().all()) and bool(got["dw"].isinf().all()) and bool((got["db"] == 300.0 * 400.0 * M).all())
    got = ops.gated_backward(dh.bfloat16(), x.bfloat16(), w.bfloat16(), z.bfloat16(), activation="none")
    assert bool(got["dx"].isfinite().all()) and bool(got["dw"].isfinite().all())
