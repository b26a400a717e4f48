"""Long sums of the gated block are added up with rounding.  The tensor cores cut an ulp, 2^-23, at most off a sum for every 16 terms: 640 terms, the most
at a time, lose (40 + 16) 2^-23 of a sum of positive numbers at most, however many there are, and each of the n chunks' additions 2^-24.  A number
in fp16 is not the rounded exact one only where that lies as near, e of its size, to the middle between two of them, which are 2^-11 to 2^-10
of their size apart: 2 e 2^11 of them at most, where cuts throughout put a third to a half there."""
import pytest
import torch

from paper_1909_07588_b200 import ops
from tests.test_gpu_ops_linear import _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M, F, K", [(2304, 2048, 65536), (2305, 2041, 40000), (1024, 1000, 65536)])
def test_sums_of_one_sign(M, F, K):
    x, w = _randn(M, K, seed=1, dtype=torch.float16).abs(), _randn(2 * F, K, seed=2, dtype=torch.float16, scale=1 / K).abs()
    _, z = ops.gated(x, w, activation="none", preact=True)
    e = (40 + 16 + K / 640 / 2) * 2.0 ** -23
    wrong = 0
    for r in range(0, M, 512):
        want = x[r:r + 512].double() @ w.double().T
        assert float(((z[r:r + 512].double() - want).abs() / want).max()) <= 2.0 ** -11 + e
        wrong += int((z[r:r + 512] != want.to(torch.float16)).sum())
    assert wrong <= 2 * e * 2 ** 11 * z.numel()
    ops.check_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K", [640, 641, 704, 1000, 1024, 1025, 1300, 2500])
def test_packed_is_pack8_of_the_other(K, dtype):
    """Whatever the sums' length: with and without Z, in 16 bits and in 8, a call adds up the same numbers in the same order."""
    for M, F in ((2300, 1408), (6500, 2560), (130, 128), (5000, 384), (4097, 5504)):
        x, w, b = _randn(M, K, seed=1, dtype=dtype), _randn(2 * F, K, seed=2, dtype=dtype, scale=K ** -0.5), _randn(2 * F, seed=3, dtype=dtype)
        for bias in (None, b):
            h, z = ops.gated(x, w, bias, activation="gelu", preact=True)
            h8, z8 = ops.gated(x, w, bias, activation="gelu", preact="packed")
            want = ops.pack8(z)
            assert torch.equal(ops.gated(x, w, bias, activation="gelu").view(torch.int16), h.view(torch.int16)) and torch.equal(h8.view(torch.int16), h.view(torch.int16))
            assert torch.equal(z8.scales, want.scales) and torch.equal(z8.codes.view(torch.uint8), want.codes.view(torch.uint8)), (M, F)
    ops.check_status()
