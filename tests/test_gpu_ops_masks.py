"""Rows of logits under finite masks of any size: -1e4 to the type's lowest value, in parts of a row and in all of it.

The bounds leave the masks' size out (u = 2^-24).  A masked logit either is the largest of its row, where d = (x - ref) c is
a difference of neighbours, or is so far below the largest one that its share is 0 in 64 bits too.  What is left:
  a sum of V terms, each off by at most (5 R + 4) u with R over the logits that are not masked (5 * 1 for masks only, whose d
  is at most a quarter), and V / 256 + 36 additions: E;
  an entropy, a difference of the sum's logarithm and its moment: E (2 + 2 R);
  a logarithm's own roundings: 4 u of its value."""
import math

import pytest
import torch

from paper_1909_07588_b200 import ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = math.inf
MASKS = [-1e4, -1e6, -1e8, -1e9, -3e9, -1e10, -1e12, -1e20, -1e29, -1e30, None]         # None: the type's lowest value


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _masks(dtype):
    dt = DTYPES[dtype]
    return [torch.finfo(dt).min if m is None else m for m in MASKS if m is None or m > torch.finfo(dt).min]


def _rows(V, dt, m, seed=0):
    """(x, keep): rows with parts masked by m, and one with all of it; keep marks what is not masked."""
    x = (torch.randn(6, V, generator=_gen(seed), device="cuda") * 3).to(dt)
    j = torch.arange(V, device="cuda")
    keep = torch.ones(6, V, dtype=torch.bool, device="cuda")
    keep[0] = False                                  # nothing left
    keep[1] = j >= V * 3 // 4                        # the front
    keep[2] = j < (V + 3) // 4                       # the back
    keep[3] = j == V - 1
    keep[4] = torch.rand(V, generator=_gen(seed + 1), device="cuda") < 0.1
    keep[4, V // 2] = True
    return torch.where(keep, x, torch.full_like(x, m)), keep


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V", [(6, 5), (6, 100), (6, 2000), (6, 50001), (6, 140000), (1500, 9001)])
def test_forward_under_finite_masks(T, V, dtype):
    dt = DTYPES[dtype]
    for m in _masks(dtype):
        for tau in (1.0, 0.7):
            x, keep = _rows(V, dt, m, seed=V)
            live = x.double().div(tau).masked_fill(~keep, -INF)
            live[0] = x[0].double() / tau
            logp = live - torch.logsumexp(live, dim=1, keepdim=True)
            # the fp64 lse of the row of masks would itself round: all of its logits are equal
            logp[0] = -math.log(V)
            H = torch.where(logp > -INF, -logp.exp() * logp, 0.0).sum(dim=1)
            tokens = torch.stack([torch.nonzero(k)[-1, 0] if bool(k.any()) else torch.tensor(V // 3, device="cuda") for k in keep]).int()
            R = torch.where(keep, x.double().abs() / tau, 0.0).amax(dim=1).clamp(min=1)
            E = (5 * R + 40 + V / 256) * U
            want = logp.gather(1, tokens.long()[:, None])[:, 0]
            k = min(V, 4)
            order = torch.argsort(x.double(), dim=1, descending=True, stable=True)[:, :k].int()
            times = T // 6
            got = {n: v.view(times, 6, *v.shape[1:]) for n, v in
                   ops.token_logprobs(x.repeat(times, 1), tokens.repeat(times), top_k=k, temperature=tau).items()}
            for r in (0, times - 1):
                assert bool(((got["logprob"][r].double() - want).abs() <= E + 4 * U * want.abs()).all()), (m, tau)
                assert bool(((got["entropy"][r].double() - H).abs() <= E * (2 + 2 * R) + 4 * U * H).all()), (m, tau)
                lse = torch.logsumexp(live, dim=1)
                off = (got["lse"][r].double() - lse).abs()
                assert bool((off <= E + 4 * U * lse.abs())[lse.abs() < 3e38].all()), (m, tau)
                assert torch.equal(got["top_tokens"][r], order), (m, tau)
                first = logp.amax(dim=1)
                assert bool(((got["top_logprobs"][r, :, 0].double() - first).abs() <= E + 4 * U * first.abs()).all()), (m, tau)


@pytest.mark.parametrize("V", [300, 20000])
def test_forward_among_masks_that_differ(V):
    """Nothing left but masks a few steps of their own type apart: the formula, from exact differences."""
    for m in (-1e5, -1e8, -3e9, -1e10, -1e14):
        step = abs(float(torch.tensor(m).float() - torch.nextafter(torch.tensor(m), torch.tensor(0.0))))
        x = (m + torch.randint(0, 40, (4, V), generator=_gen(1), device="cuda").double() * step).float()
        d = x.double() - x.double().amax(dim=1, keepdim=True)
        logp = d - torch.logsumexp(d, dim=1, keepdim=True)
        H = -(logp.exp() * logp).sum(dim=1)
        tokens = x.argmax(dim=1).int()
        got = ops.token_logprobs(x, tokens)
        want = logp.amax(dim=1)
        # |d| below 150 has a share: 2 roundings of it, and what V / 256 + 40 additions add
        E = (2 * 150 + 40 + V / 256) * U
        assert bool(((got["logprob"].double() - want).abs() <= E + 4 * U * want.abs()).all()), m
        assert bool(((got["entropy"].double() - H).abs() <= E * (2 + 2 * math.log(V)) + 4 * U * H).all()), m


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [100, 1500, 50001])
def test_distill_under_finite_masks(V, dtype):
    """Loss and gradient of rows with masked parts are those of rows masked by -inf there."""
    dt = DTYPES[dtype]
    for m in _masks(dtype):
        x, keep = _rows(V, dt, m, seed=V)
        x, keep = x[1:].contiguous(), keep[1:]
        tok = torch.stack([torch.nonzero(k)[-1] for k in keep]).int()
        val = torch.zeros(5, 1, device="cuda")
        one = torch.ones(5, device="cuda")
        hard = x.masked_fill(~keep, -INF)
        for tau in (1.0, 2.0):
            want, got = (ops.distill(v, tok, val, temperature=tau, d_loss=one) for v in (hard, x))
            R = torch.where(keep, x.double().abs() / tau, 0.0).amax(dim=1).clamp(min=1)
            E = 2 * (5 * R + 40 + V / 256) * U
            assert bool(((got["loss"] - want["loss"]).double().abs() <= tau * tau * E + 8 * U * want["loss"].double()).all()), (m, tau)
            half = torch.finfo(dt).eps if dt != torch.float32 else 2 * U
            tiny = torch.finfo(dt).smallest_normal if dt != torch.float32 else 2.0 ** -120
            for dx in (got["dlogits"], ops.distill_backward(x, tok, val, got["lse"], one, temperature=tau)):
                off = (dx.double() - want["dlogits"].double()).abs()
                assert bool((off <= half * want["dlogits"].double().abs() + tau * (2 * E[:, None] + 6 * R[:, None] * U) + tiny).all()), (m, tau)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [100, 3000, 50001, 300000])
def test_gradients_of_rows_of_masks_alone(V, dtype):
    """Nothing left in a row: by -inf, and by finite masks whose lse fp32 does not hold to a unit, every gradient is 0, in the
    call with the loss (in one reading or, of the longest rows, in two) and in the call of its own.  Down to there the
    gradient is the formula's, up to what the rounding of lse, u |lse|, and of its product with log2(e) make of p."""
    dt = DTYPES[dtype]
    for m in [-INF, -1.0, -300.0] + _masks(dtype):
        for tau in (1.0, 0.5):
            x = torch.full((3, V), m, device="cuda").to(dt)
            x[1] = torch.randn(V, generator=_gen(1), device="cuda").to(dt)           # rows beside it are not concerned
            tok = torch.tensor([[0, 3], [1, 2], [V - 1, 5]], device="cuda").int()
            val = torch.tensor([[0.5, 0.25]] * 3, device="cuda")
            d = torch.tensor([1.5, 1.0, -0.5], device="cuda")
            step = ops.distill(x, tok, val, temperature=tau, d_loss=d)
            alone = ops.distill_backward(x, tok, val, step["lse"], d, temperature=tau)
            st = ops.token_logprobs(x, tok[:, 0].contiguous(), temperature=tau)
            pg = ops.token_logprobs_backward(x, tok[:, 0].contiguous(), st["lse"], st["entropy"], d, d, temperature=tau)
            s = float(x[0, 0]) / tau
            for r in (0, 2):
                if s + math.log(V) <= -2.0 ** 24:
                    assert not bool(step["dlogits"][r].any()) and not bool(alone[r].any()) and not bool(pg[r].any()), (m, tau)
                    continue
                if s <= -2.0 ** 20:
                    for dx in (step["dlogits"], alone, pg):
                        assert float(dx[r].abs().max()) <= 8 * 1.5 * max(tau, 1 / tau), (m, tau)
                    continue
                q = torch.softmax(val[r].double() / tau, dim=0)
                want = torch.full((V,), 1.0 / V, device="cuda", dtype=torch.float64)
                want[tok[r].long()] -= q
                want = want * tau * float(d[r])
                rel = 6 * U * (abs(s) + math.log(V)) + 60 * U + V / 256 * U
                rel = (torch.finfo(dt).eps / 2 if dt != torch.float32 else U) + 1.5 * rel
                tiny = torch.finfo(dt).smallest_normal
                for dx in (step["dlogits"], alone):
                    assert bool(((dx[r].double() - want).abs() <= rel * (want.abs() + 1.0 / V * abs(tau * float(d[r]))) + tiny).all()), (m, tau)
            assert bool(step["dlogits"][1].any()) and bool(alone[1].any()) and bool(pg[1].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [80, 1500, 30000, 300000])
@pytest.mark.parametrize("m", [-INF, -1e9, None])
def test_a_bad_column_shows_in_masked_rows_too(V, m, dtype):
    dt = DTYPES[dtype]
    x = torch.full((4, V), torch.finfo(dt).min if m is None else m, device="cuda").to(dt)
    x[3] = torch.randn(V, generator=_gen(1), device="cuda").to(dt)
    one = torch.ones(4, device="cuda")
    tok = torch.tensor([[3, V], [2, 5], [2 ** 31 - 1, -1], [1, 2]], device="cuda").int()
    val = torch.zeros(4, 2, device="cuda")
    step = ops.distill(x, tok, val, d_loss=one)
    alone = ops.distill_backward(x, tok, val, step["lse"], one)
    st = ops.token_logprobs(x, tok.amax(dim=1))
    pg = ops.token_logprobs_backward(x, tok.amax(dim=1), st["lse"], st["entropy"], one, one)
    assert step["loss"].isnan().tolist() == [True, False, True, False]
    assert st["logprob"].isnan().tolist() == [True, False, True, False]
    for dx in (step["dlogits"], alone, pg):
        assert bool(dx[[0, 2]].isnan().all()) and not bool(dx[1].any()) and bool(dx[3].isfinite().all())
