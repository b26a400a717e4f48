"""How precise the operators are where it is easy to lose precision: peaked rows, long sums, low temperatures.

u = 2^-24.  A rounding to nearest is off by at most u of the value and, over many values, by u / sqrt(3) of it (root mean
square); n independent ones by sqrt(n) of that."""
import math

import pytest
import torch

from paper_1909_07588_b200 import ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _peaked(T, V, dt, seed):
    """Rows like a trained model's: a broad body and one peak in each."""
    x = torch.empty(T, V, dtype=dt, device="cuda")
    g = _gen(seed)
    for r in range(0, T, 200):
        b = torch.randn(min(200, T - r), V, generator=g, device="cuda") * 2.5
        b[torch.arange(b.shape[0], device="cuda"), torch.randint(0, V, (b.shape[0],), generator=g, device="cuda")] += 12.0
        x[r:r + 200] = b.to(dt)
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V", [(1400, 131072), (300, 131072), (64, 100003), (3000, 2001)])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_entropy_of_peaked_rows(T, V, dtype, tau):
    """The entropy is log2 s - m, m = u / s the mean of d = (x - ref) c.  Root mean square over rows, in units of what a row's
    independent roundings make of it:
      n additions on the way to s and u (16 within a batch, a batch for every 512 threads' vectors, a rest of 3, the joins' 14),
      sqrt(n / 3) u of s, and of sum |d| 2^d: log2(e) and sqrt(2) |d| of that, with |d| at most 8, what a reference may
      lag, and 1 and log2(e) H for the body;
      the exponentials' 4 u, u for each of d's, of the logarithm's and the quotient's rounding, with the same weights: 6 u;
      c off by u at most: u times the variance of x / tau under p."""
    dt = DTYPES[dtype]
    x = _peaked(T, V, dt, V)
    got = ops.token_logprobs(x, temperature=tau)["entropy"].double()
    H, var = torch.empty_like(got), torch.empty_like(got)
    for r in range(0, T, 100):
        s = x[r:r + 100].double() / tau
        logp = torch.log_softmax(s, dim=1)
        p = logp.exp()
        H[r:r + 100] = -(p * logp).sum(dim=1)
        var[r:r + 100] = (p * logp * logp).sum(dim=1) - H[r:r + 100] ** 2
    n = 16 + V / (512 * (16 / dt.itemsize)) + 3 + 14
    size = math.log2(math.e) + math.sqrt(2) * (8 + 1 + math.log2(math.e) * H)
    unit = U * (math.log(2) * (math.sqrt(n / 3) + 6) * size + var)
    assert float(((got - H) / unit).square().mean().sqrt()) <= 1


def _chunked(n, chunk=16384):
    """What a sum of n positive terms in chunks may lose of itself: a step for 16 of a chunk's terms, each cut by less than an ulp, and
    a rounding for every chunk (and for a split's parts)."""
    return chunk / 16 * 2.0 ** -23 + (n / chunk + 10) * U


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("M, N, K", [(1 << 20, 64, 136), (70001, 257, 129), (262144, 512, 256)])
def test_weight_gradient_over_many_rows(M, N, K, dtype, act):
    """Same-sign terms: a sum that is cut at every step would lose n 10^-9 of itself, 8e-4 over 2^20 rows."""
    dt = DTYPES[dtype]
    dy = (torch.rand(M, N, generator=_gen(1), device="cuda") * (1024.0 / M)).to(dt)
    x = torch.rand(M, K, generator=_gen(2), device="cuda").to(dt)
    w = torch.zeros(N, K, device="cuda", dtype=dt)
    z = None if act == "none" else torch.ones(M, N, device="cuda", dtype=dt)
    want = sum(dy[r:r + 65536].double().T @ x[r:r + 65536].double() for r in range(0, M, 65536))
    got = ops.linear_backward(dy, x, w, z=z, activation=act, dx=False, db=False)["dw"].double()
    half = torch.finfo(dt).eps / 2
    assert float(((got - want).abs() / want).max()) <= _chunked(M) + half * (1 + _chunked(M))
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(33, 72, (1 << 20) + 24), (512, 512, 131080), (300, 1000, 65537), (7, 20, 70000)])
def test_long_rows(M, N, K, dtype):
    """The forward product and the input's gradient over a long axis, with everything that the epilogue does."""
    dt = DTYPES[dtype]
    half, c = torch.finfo(dt).eps / 2, _chunked(K)
    x = torch.rand(M, K, generator=_gen(1), device="cuda").to(dt)
    w = (torch.rand(N, K, generator=_gen(2), device="cuda") * (16.0 / K)).to(dt)
    b, r = torch.rand(N, generator=_gen(3), device="cuda").to(dt), torch.rand(M, N, generator=_gen(4), device="cuda").to(dt)
    want = x.double() @ w.double().T
    y, z = ops.linear(x, w, b, activation="relu", residual=r, preact=True)
    zw = want + b.double()
    assert float(((z.double() - zw).abs() / zw).max()) <= c + 2 * U + half * (1 + c + 2 * U)
    yw = zw + r.double()
    assert float(((y.double() - yw).abs() / yw).max()) <= c + 4 * U + half * (1 + c + 4 * U)
    # dX = dZ W has the layer's outputs as its terms: K of them, with x in the place of dZ
    got = ops.linear_backward(x, torch.zeros(M, N, device="cuda", dtype=dt), w.T.contiguous(), dw=False, db=False)["dx"].double()
    assert float(((got - want).abs() / want).max()) <= c + half * (1 + c)
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(8192, 64, 128), (16384, 200, 784), (65536, 256, 512), (1 << 19, 40, 72)])
def test_fp32_weight_gradient_is_summed_in_chunks(M, N, K, dtype):
    """fp32 dW of same-sign terms within what chunks of 512 terms may lose, 4e-6 for a chunk's cuts and 6e-8 a chunk.  One
    uncut sum loses more from 8192 rows on with fp16 operands, from 65536 with bf16 ones."""
    dt = DTYPES[dtype]
    dy = torch.rand(M, N, generator=_gen(1), device="cuda").to(dt)
    x = torch.rand(M, K, generator=_gen(2), device="cuda").to(dt)
    want = sum(dy[r:r + 65536].double().T @ x[r:r + 65536].double() for r in range(0, M, 65536))
    got = ops.linear_backward(dy, x, torch.zeros(N, K, device="cuda", dtype=dt), dx=False, db=False, dw_dtype=torch.float32)["dw"]
    off = ((got.double() - want) / want).abs()
    # the roundings of the chunks' additions are to nearest: sqrt(n / 3) of them, and four times that at the farthest
    assert float(off.max()) <= 32 * 2.0 ** -23 + U * (4 * math.sqrt((M / 512 + 10) / 3) + 1)
    ops.check_status()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [500, 3000, 40000])
@pytest.mark.parametrize("tau", [1.0, 1e-2, 1e-3, 1e-4])
def test_step_gradient_at_low_temperatures(V, dtype, tau):
    """Rows whose largest logit comes n times and whose others are 1 below: p is 1 / n there (and, but for tau = 1, 0 elsewhere).
    Differences of equal logits are exact, so what is left is the sum's V / 256 + 40 roundings, the exponential's and the
    logarithm's few, and the output's own; a reference near 20 / tau log2(e) rounded together with log2 s would be off by half
    a step of it, 0.5 % of p at tau = 1e-4."""
    dt = DTYPES[dtype]
    tops = [20.0, -20.25, 7.5, 30.0, -3.0, 0.0]
    x = torch.stack([torch.full((V,), t - 1.0, device="cuda") for t in tops])
    n = [1, 2, 3, 7, 50, V // 3]
    for r, (t, k) in enumerate(zip(tops, n)):
        x[r, torch.randperm(V, generator=_gen(r), device="cuda")[:k]] = t
    x = x.to(dt)
    tok = x.argmin(dim=1, keepdim=True).int()
    one = torch.full((6,), 1 / tau, device="cuda")
    got = ops.distill(x, tok, torch.zeros(6, 1, device="cuda"), temperature=tau, d_loss=one)
    want = torch.softmax(x.double() / tau, dim=1)
    want.scatter_add_(1, tok.long(), torch.full((6, 1), -1.0, device="cuda", dtype=torch.float64))
    half = torch.finfo(dt).eps / 2 if dt != torch.float32 else U
    # c's rounding shifts the lower logits by u / tau; the other type's of ref c + log2 s, where it is taken, 2^-13 of log2
    rel = half + (V / 256 + 60) * U + (2 * U / tau if tau == 1.0 else 0) + (2.0 ** -13 if dt != torch.float32 and tau >= 1e-2 else 0)
    off = (got["dlogits"].double() - want).abs()
    assert bool((off <= rel * want.abs() * (1 + rel) + 1e-7).all()), float((off / want.abs().clamp(min=1e-12)).max())


@pytest.mark.parametrize("M, N, K", [(16, 256, 70000), (300, 300, 70000), (2048, 1024, 66000)])
def test_starved_long_sum_runs_out_and_is_reported(M, N, K):
    """A split tile, single blocks and pairs whose sums are taken in chunks: every wait ends, and the same call works again."""
    from paper_1909_07588_b200 import laq
    x, w = torch.rand(M, K, generator=_gen(1), device="cuda").half(), (torch.rand(N, K, generator=_gen(2), device="cuda") / K).half()
    want = ops.linear(x, w)
    ops.check_status()
    ops.linear(x, w, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    ops.check_status()
    assert torch.equal(ops.linear(x, w), want)
    ops.check_status()


def test_long_sums_beside_each_other():
    """Long and short split sums on two streams at once, many times: each result as when alone."""
    dt = torch.bfloat16
    dy, x = torch.rand(131072, 1024, generator=_gen(1), device="cuda").to(dt), torch.rand(131072, 1024, generator=_gen(2), device="cuda").to(dt)
    w = torch.rand(1024, 1024, generator=_gen(3), device="cuda").to(dt)
    a, b = torch.rand(64, 4096, generator=_gen(4), device="cuda").to(dt), torch.rand(2048, 4096, generator=_gen(5), device="cuda").to(dt)
    long = lambda: ops.linear_backward(dy, x, w, dx=False, db=False)["dw"]
    short = lambda: ops.linear(a, b)
    want_long, want_short = long(), short()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    wrong = [torch.zeros((), dtype=torch.int64, device="cuda") for _ in streams]
    for _ in range(20):
        for s, n in zip(streams, wrong):
            with torch.cuda.stream(s):
                if s is streams[0]:
                    n += (long() != want_long).sum()
                else:
                    for _ in range(6):
                        n += (short() != want_short).sum()
    torch.cuda.synchronize()
    assert [int(n) for n in wrong] == [0, 0, 0]
    ops.check_status()
