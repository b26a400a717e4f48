"""token_logprobs, distill and their gradients against the definitions in fp64.

Bounds (u = 2^-24, R = the largest finite |s| of the row, s = logit / temperature, n = vocabulary):
  a term exp(s_j - lse) is off, relatively, by at most the rounding of c = log2(e) / temperature and of one fused
  operation on numbers of up to 1.45 R each, 2 * 1.45 R u, by ex2's 2^-22 = 4 u, and by the rounding of the reference
  (1.45 R u): together (5 R + 4) u;
  a sum of n terms adds the roundings of the longest chain: n / 256 + 32 additions (two chains a thread, 128 threads or
  more, then the joins; rows of one warp have at most n / 32 / 2 <= n / 256 + 32 for n <= 4096);
  so lse, and a log probability, are off by at most E = (5 R + 8 + n / 256 + 32) u plus u |value| for its last rounding;
  the entropy's moment sum p d has |d| <= 2 R: E (2 + 2 R);
  a gradient's p carries (5 R + 4) u, its log p R u more; then the output's own rounding, eps / 2 of the value, and half
  a step of the smallest numbers of the type (its subnormals, which may also be flushed).
"""
import math

import pytest
import torch

from paper_1909_07588_b200 import laq, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = math.inf


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _logits(T, V, dtype, seed=0, scale=3.0):
    return (torch.randn(T, V, generator=_gen(seed), device="cuda") * scale).to(DTYPES[dtype])


def _range(s):
    return torch.where(s.isfinite(), s.abs(), 0.0).amax(dim=1)


def _sum_bound(s):
    return (5 * _range(s) + 40 + s.shape[1] / 256) * U


def _close(got, want, bound, what):
    got, want = got.double(), want.double()
    # what fp32 cannot hold rounds to an infinity: 2^128 (1 - 2^-25) lies halfway between its largest number and 2^128
    want = torch.where(want.abs() >= 2.0 ** 128 * (1 - 2.0 ** -25), want.sign() * INF, want)
    same = torch.where(want.isnan(), got.isnan(), torch.where(want.isinf(), got == want, torch.ones_like(want, dtype=torch.bool)))
    assert bool(same.all()), what
    fine = want.isfinite()
    excess = ((got - want).abs() - bound)[fine]
    assert excess.numel() == 0 or float(excess.max()) <= 0, "%s: off by %g more than it may" % (what, float(excess.max()))


def _exact(x, tokens, k, tau):
    """The definition in fp64, row by row conventions included."""
    s = x.double() / tau
    nan = s.isnan().any(dim=1) | (s == INF).any(dim=1)
    empty = (s == -INF).all(dim=1)
    lse = torch.logsumexp(s, dim=1)
    logp = torch.where(s == -INF, -INF, s - lse[:, None])
    p = torch.where(logp == -INF, 0.0, logp.exp())
    H = torch.where(empty, 0.0, torch.where(p > 0, -p * logp, 0.0).sum(dim=1))
    live = torch.ones_like(nan) if tokens is None else tokens >= 0
    out = dict(lse=torch.where(nan, math.nan, lse), entropy=torch.where(nan, math.nan, H))
    if tokens is not None:
        inside = tokens < x.shape[1]
        at = torch.where(live & inside, tokens, 0).long()
        lp = logp.gather(1, at[:, None])[:, 0]
        lp = torch.where(empty, -INF, lp)
        out["logprob"] = torch.where(nan | ~inside, math.nan, lp)
    for key in out:
        out[key] = torch.where(live, out[key], 0.0)
    if k:
        T, V = x.shape
        n = min(k, V)
        at = torch.argsort((x.double() + 0.0).nan_to_num(nan=INF), dim=1, descending=True, stable=True)[:, :n]
        value = logp.gather(1, at)
        gone = (value == -INF) | ~live[:, None] | nan[:, None]
        tt = torch.full((T, k), -1, dtype=torch.int32, device=x.device)
        tv = torch.full((T, k), -INF, dtype=torch.float64, device=x.device)
        tt[:, :n] = torch.where(gone, -1, at).int()
        tv[:, :n] = torch.where(gone, -INF, value)
        tv[nan & live] = math.nan
        out.update(top_tokens=tt, top_logprobs=tv)
    return out


def _check_forward(x, tokens=None, k=0, tau=1.0, **kw):
    got = ops.token_logprobs(x, tokens, top_k=k, temperature=tau, **kw)
    want = _exact(x, tokens, k, tau)
    assert set(got) == set(want)
    E = _sum_bound(x.double() / tau)
    R = _range(x.double() / tau)
    _close(got["lse"], want["lse"], E + U * want["lse"].abs() * 2, "lse")
    _close(got["entropy"], want["entropy"], E * (2 + 2 * R), "entropy")
    if tokens is not None:
        _close(got["logprob"], want["logprob"], E + 2 * U * want["logprob"].abs(), "logprob")
    if k:
        assert torch.equal(got["top_tokens"], want["top_tokens"])
        _close(got["top_logprobs"], want["top_logprobs"], (E[:, None] + 2 * U * want["top_logprobs"].abs()), "top_logprobs")
    return got


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 10), (4, 33), (3, 517), (3, 1000), (2, 1024), (2, 1025), (3, 4097), (2, 8191), (1, 50001),
          (2, 131072), (700, 100), (2500, 2050), (1300, 8200), (40, 16385)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V", SHAPES)
def test_forward(T, V, dtype):
    x = _logits(T, V, dtype, seed=V)
    tokens = torch.randint(0, V, (T,), generator=_gen(1), device="cuda").int()
    if T > 2:
        tokens[1] = -1
    for k, tau in ((0, 1.0), (1, 0.7), (5, 2.0), (32, 1.0)):
        _check_forward(x, tokens, k, tau)
    _check_forward(x, None, 3, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [61, 1500, 20011])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_forward_of_strided_rows(V, dtype, offset):
    whole = _logits(6, V + 9, dtype, seed=offset)
    x = whole[:, offset:offset + V]
    tokens = torch.tensor([0, V - 1, 5, -1, 7, V // 2], dtype=torch.int32, device="cuda")
    _check_forward(x, tokens, 8)
    _check_forward(whole[::2, offset:offset + V], tokens[::2].contiguous(), 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [40, 900, 3000, 30001, 140000])
def test_alternatives_among_equal_logits(V, dtype):
    rows = [torch.zeros(V), torch.full((V,), -3.0), torch.arange(V) % 3 * 1.0, (torch.arange(V) % 7 == 3) * 1.0,
            torch.arange(V) * 1e-3, -torch.arange(V) * 1e-3, torch.where(torch.arange(V) >= V - 3, 2.0, 1.0),
            torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)]
    x = torch.stack(rows).to("cuda").to(DTYPES[dtype])
    for k in (1, 8, 32):
        _check_forward(x, None, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V", [(1184, 33001), (1300, 2111), (1250, 16421)])
def test_forward_of_many_rows(T, V, dtype):
    """Rows of small blocks, each with rows of its own kind among them: equal logits, masks, nothing left, not a number."""
    x = _logits(T, V, dtype, seed=T)
    j = torch.arange(V, device="cuda")
    x[3] = 1.0
    x[4] = (j % 3).to(x.dtype)
    x[5] = torch.where(j >= V - 3, 2.0, 1.0).to(x.dtype)
    x[6] = -INF
    x[7, : V - 5] = -INF
    x[8, 5:] = -INF
    x[9] = torch.finfo(x.dtype).min
    x[10, 17] = math.nan
    x[11] = torch.where(j % 128 == 127, 0.01 * (j // 128 % 89), -1.0).to(x.dtype)
    x[12, :-1] = -INF
    tokens = torch.randint(0, V, (T,), generator=_gen(5), device="cuda").int()
    tokens[::7] = -1
    for k, tau in ((0, 1.0), (3, 0.7), (32, 1.0)):
        _check_forward(x, tokens, k, tau)
        _check_forward(x[:, 1:V - 1], None, k, tau)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_alternatives_of_many_long_rows(dtype):
    x = _logits(8, 140000, dtype, seed=8)
    x[1] = 0.5
    x[2] = torch.where(torch.arange(140000, device="cuda") % 1024 < 8, 3.0, 1.0).to(x.dtype)
    for k in (1, 20, 32):
        want = _check_forward(x, None, k)
        got = ops.token_logprobs(x.repeat(150, 1), None, top_k=k)
        assert torch.equal(got["top_tokens"], want["top_tokens"].repeat(150, 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives_that_few_threads_own(dtype):
    """All large logits lie in vectors that one thread (of 256, of 128, of one warp) reads."""
    for V, period in ((140000, 256), (16384, 256), (16384, 128), (4096, 32)):
        ev = 16 // DTYPES[dtype].itemsize
        x = _logits(2, V, dtype, scale=0.1)
        j = torch.arange(V, device="cuda")
        own = (j // ev) % period == 0
        x[0] = torch.where(own, 5 + 0.01 * (j // ev // period % 97), x[0].float()).to(x.dtype)
        x[1] = torch.where(own, 5.0, x[1].float()).to(x.dtype)
        _check_forward(x, None, 32)
        _check_forward(x.repeat(700, 1), None, 32)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [50, 2000, 30001])
def test_masks(V, dtype):
    x = _logits(9, V, dtype)
    low = torch.finfo(x.dtype).min
    x[0] = -INF                                      # nothing left
    x[1] = -INF
    x[1, V - 2] = 1.5                                # one entry left
    x[2] = low                                       # masked by the type's lowest value throughout: uniform
    x[3] = low
    x[3, 7] = -2.0
    x[4, ::2] = -INF
    x[5, 3] = math.nan
    x[6, 3] = INF
    x[7] = math.nan                                  # a padded row: nothing of it matters
    tokens = torch.tensor([3, V - 2, 4, 7, 2, 1, 3, -1, 5], dtype=torch.int32, device="cuda")
    got = _check_forward(x, tokens, 6)
    assert got["top_tokens"][7].tolist() == [-1] * 6 and float(got["lse"][7]) == 0.0
    assert float(got["logprob"][4]) == -INF
    # every x is the reference itself in row 2: exp is 1 there and only the sum and the logarithm round
    assert abs(float(got["logprob"][2]) + math.log(V)) <= (40 + V / 256 + 2 * math.log(V)) * U
    # gradients: rows without anything left, and padded rows, get zeros
    g, h = torch.randn(9, generator=_gen(3), device="cuda"), torch.randn(9, generator=_gen(4), device="cuda")
    for out in (None, x.clone()):
        src = x if out is None else out
        dx = ops.token_logprobs_backward(src, tokens, got["lse"], got["entropy"], g, h, out=out)
        assert not bool(dx[0].any()) and not bool(dx[7].any())
        assert bool(dx[5].isnan().all()) and bool(dx[6].isnan().all())
        assert not bool(dx[[1, 3, 4, 8]].isnan().any())
        assert float(dx[1].float().abs().max()) <= 2.0 ** -20 * float(g[1].abs() + h[1].abs())      # p = 1: nothing to gain
        assert not bool(dx[4, 4::2].any())           # masked entries other than the token


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_outside_the_vocabulary(dtype):
    for V in (100, 5000):
        x = _logits(4, V, dtype)
        tokens = torch.tensor([1, V, 2 ** 31 - 1, V - 1], dtype=torch.int32, device="cuda")
        got = _check_forward(x, tokens, 2)
        dx = ops.token_logprobs_backward(x, tokens, got["lse"], d_logprob=torch.ones(4, device="cuda"))
        assert bool(dx[1:3].isnan().all()) and not bool(dx[[0, 3]].isnan().any())


def _gradient_bound(want, terms, x, tau):
    """terms: the magnitudes that p and log p enter with; want: the exact gradient."""
    R = _range(x.double() / tau)[:, None]
    fi = torch.finfo(x.dtype)
    half = fi.eps / 2 if x.dtype != torch.float32 else U
    return half * want.abs() + (6 * R + 8) * U * terms + max(fi.smallest_normal * fi.eps if x.dtype != torch.float32 else 0.0, 2.0 ** -120)


def _exact_logprobs_gradient(x, tokens, lse, H, g, h, tau):
    s = x.double() / tau
    logp = s - lse.double()[:, None]
    p = logp.exp()
    logp = torch.where(p > 0, logp, 0.0)
    one = torch.zeros_like(p)
    live = tokens >= 0
    one[live, tokens[live].long()] = 1.0
    g, h, H = g.double()[:, None], h.double()[:, None], H.double()[:, None]
    want = (g * (one - p) - h * p * (logp + H)) / tau
    terms = (g.abs() * (p + one) + h.abs() * p * (logp.abs() + H.abs() + 1)) / tau
    return torch.where(live[:, None], want, 0.0), torch.where(live[:, None], terms, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V", [(1, 1), (3, 7), (4, 130), (2, 1024), (3, 1025), (2, 9001), (2, 70000), (2400, 300), (2500, 2050)])
def test_logprobs_gradient(T, V, dtype):
    x = _logits(T, V, dtype, seed=V + 1)
    tokens = torch.randint(0, V, (T,), generator=_gen(2), device="cuda").int()
    if T > 1:
        tokens[T - 1] = -1
    g, h = torch.randn(T, generator=_gen(3), device="cuda"), torch.randn(T, generator=_gen(4), device="cuda") * 0.3
    for tau in (1.0, 0.7):
        st = ops.token_logprobs(x, tokens, temperature=tau)
        want, terms = _exact_logprobs_gradient(x, tokens, st["lse"], st["entropy"], g, h, tau)
        bound = _gradient_bound(want, terms, x, tau)
        dx = ops.token_logprobs_backward(x, tokens, st["lse"], st["entropy"], g, h, temperature=tau)
        _close(dx, want, bound, "gradient")
        # into a strided place whose rows lie elsewhere within 16 bytes, and over the logits themselves
        place = torch.full((T, V + 11), 7.0, dtype=x.dtype, device="cuda")
        ops.token_logprobs_backward(x, tokens, st["lse"], st["entropy"], g, h, temperature=tau, out=place[:, 5:5 + V])
        _close(place[:, 5:5 + V], want, bound, "gradient in a strided place")
        assert bool((place[:, :5] == 7).all()) and bool((place[:, 5 + V:] == 7).all())
        over = x.clone()
        assert ops.token_logprobs_backward(over, tokens, st["lse"], st["entropy"], g, h, temperature=tau, out=over) is over
        assert torch.equal(over, dx)
        # one gradient at a time adds up to both (each part rounds for itself)
        a = ops.token_logprobs_backward(x, tokens, st["lse"], d_logprob=g, temperature=tau)
        b = ops.token_logprobs_backward(x, tokens, st["lse"], st["entropy"], d_entropy=h, temperature=tau)
        _close(a.double() + b.double(), want, 2 * bound + torch.finfo(x.dtype).eps * (a.double().abs() + b.double().abs()), "parts")


@pytest.mark.parametrize("what", ["logprob", "entropy"])
def test_logprobs_gradient_against_differences(what):
    """Central differences of the forward call: off by h^2 / 6 of the third derivative (below 6 for a softmax of unit
    temperature times |log p| + H < 16 here) and by the forward's error over h."""
    T, V, h = 3, 29, 2.0 ** -5
    x = _logits(T, V, "f32", scale=1.0)
    tokens = torch.tensor([0, 5, V - 1], dtype=torch.int32, device="cuda")
    st = ops.token_logprobs(x, tokens)
    one = torch.ones(T, device="cuda")
    dx = ops.token_logprobs_backward(x, tokens, st["lse"], st["entropy"], **{"d_" + what: one})
    bound = h * h * 6 * 16 / 6 + float(_sum_bound(x.double()).max()) * 12 / h
    for j in range(V):
        e = torch.zeros_like(x)
        e[:, j] = h
        d = (ops.token_logprobs(x + e, tokens)[what] - ops.token_logprobs(x - e, tokens)[what]) / (2 * h)
        assert float((d - dx[:, j]).abs().max()) <= bound


# --- distillation ----------------------------------------------------------------------------------------------------

def _teacher(T, K, V, seed=0, dup=True):
    g = _gen(seed)
    tok = torch.randint(0, V, (T, K), generator=g, device="cuda").int()
    val = torch.randn(T, K, generator=g, device="cuda") * 2
    if dup and K > 2:
        tok[:, 2] = tok[:, 0]
    return tok, val


def _exact_distill(x, tok, val, tau, d_loss):
    s = x.double() / tau
    lse = torch.logsumexp(s, dim=1)
    logp = s - lse[:, None]
    p = logp.exp()
    t = torch.where(tok >= 0, val.double() / tau, -INF)
    row = (t > -INF).any(dim=1)
    t = torch.where(row[:, None], t, 0.0)
    logq = t - torch.logsumexp(t, dim=1, keepdim=True)
    q = torch.where(row[:, None], logq.exp(), 0.0)
    at = tok.clamp(min=0).long()
    lp = logp.gather(1, at)
    each = torch.where(q > 0, q * (torch.where(q > 0, logq, 0.0) - lp), 0.0)
    loss = tau * tau * each.sum(dim=1)
    size = tau * tau * torch.where(q > 0, q * (torch.where(q > 0, logq, 0.0).abs() + lp.abs()), 0.0).sum(dim=1)
    target = torch.zeros_like(p).scatter_add_(1, at, q)
    want = torch.where(row[:, None], (p - target) * (tau * d_loss.double())[:, None], 0.0)
    terms = torch.where(row[:, None], (p + target) * (tau * d_loss.double().abs())[:, None], 0.0)
    return loss, torch.where(row, lse, 0.0), want, terms, size


def _check_distill(x, tok, val, tau, bwd=True):
    T = x.shape[0]
    d = torch.randn(T, generator=_gen(9), device="cuda")
    loss, lse, want, terms, size = _exact_distill(x, tok, val, tau, d)
    E = _sum_bound(x.double() / tau)
    R = torch.maximum(_range(x.double() / tau), _range(torch.where(tok >= 0, val, 0.0).double() / tau))
    # q: (2 R u + 4 u + 8 u for its own sum and quotient) of each share; a logarithm E
    lb = tau * tau * (E + (2 * R + 16) * U) + (2 * R + 24) * U * size
    fwd = ops.distill(x, tok, val, temperature=tau)
    assert set(fwd) == {"loss", "lse"}
    step = ops.distill(x, tok, val, temperature=tau, d_loss=d)
    for got in (fwd, step):
        _close(got["loss"], loss, lb, "loss")
        _close(got["lse"], lse, E + 2 * U * lse.abs(), "lse")
    # the step's p comes from the sums themselves: E more
    bound = _gradient_bound(want, terms * 2, x, tau) + E[:, None] * terms
    _close(step["dlogits"], want, bound, "gradient of the step")
    over = x.clone()
    res = ops.distill(over, tok, val, temperature=tau, d_loss=d, out=over)
    assert res["dlogits"] is over and torch.equal(over, step["dlogits"])
    if bwd:
        # the gradient alone goes by the lse it is given in fp32: u |lse| more
        b2 = bound + (U * lse.abs() * 3)[:, None] * terms
        dx = ops.distill_backward(x, tok, val, step["lse"], d, temperature=tau)
        _close(dx, want, b2, "gradient alone")
        over = x.clone()
        ops.distill_backward(over, tok, val, step["lse"], d, temperature=tau, out=over)
        assert torch.equal(over, dx)
    return step


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T, V, K", [(1, 1, 1), (3, 5, 8), (4, 33, 128), (2, 1024, 16), (3, 1025, 100), (2, 4100, 31), (2, 9001, 64),
                                     (1, 70000, 128), (2, 140000, 33), (900, 50, 7), (1200, 3000, 20), (600, 17000, 64), (3, 40001, 1)])
def test_distill(T, V, K, dtype):
    x = _logits(T, V, dtype, seed=V)
    tok, val = _teacher(T, K, V, seed=K)
    for tau in (1.0, 2.0):
        _check_distill(x, tok, val, tau)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_of_rows_too_long_for_one_pass(dtype):
    V = 140000 if dtype == "f32" else 270001
    x = _logits(2, V, dtype)
    tok, val = _teacher(2, 50, V)
    _check_distill(x, tok, val, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("V", [70, 1300, 20000])
def test_distill_with_missing_entries(V, dtype):
    T, K = 8, 12
    x = _logits(T, V, dtype)
    tok, val = _teacher(T, K, V)
    tok[0, 5:] = -1
    tok[1] = -1                       # no entries at all
    tok[2, ::2] = -1
    val[3, 4:] = -INF                 # masked entries
    val[4] = -INF                     # all of them: nothing to learn
    tok[5] = 7                        # one column, twelve times
    val[6, 0] = 500.0                 # the others underflow
    step = _check_distill(x, tok, val, 1.0)
    for i in (1, 4):
        assert float(step["loss"][i]) == 0 and float(step["lse"][i]) == 0 and not bool(step["dlogits"][i].any())
    # strided teacher, strided rows
    wide_t, wide_v = torch.full((T, K + 5), -1, dtype=torch.int32, device="cuda"), torch.zeros(T, K + 5, device="cuda")
    wide_t[:, 2:2 + K], wide_v[:, 2:2 + K] = tok, val
    wide_x = torch.zeros(T, V + 3, dtype=x.dtype, device="cuda")
    wide_x[:, 1:1 + V] = x
    again = ops.distill(wide_x[:, 1:1 + V], wide_t[:, 2:2 + K], wide_v[:, 2:2 + K], d_loss=torch.ones(T, device="cuda"))
    first = ops.distill(x, tok, val, d_loss=torch.ones(T, device="cuda"))
    E = _sum_bound(x.double())
    _close(again["loss"], first["loss"], 2 * E + 2 ** -18 * first["loss"].abs(), "loss of strided rows")
    _close(again["dlogits"], first["dlogits"], torch.finfo(x.dtype).eps * 2 * first["dlogits"].abs().double() + 64 * E[:, None], "strided rows")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [80, 1500, 30000])
def test_distill_masks_and_bad_columns(V, dtype):
    T, K = 6, 4
    x = _logits(T, V, dtype)
    tok, val = _teacher(T, K, V, dup=False)
    tok[:] = torch.tensor([3, 11, 20, 41], device="cuda", dtype=torch.int32)
    x[0, 11] = -INF                   # the teacher's column is masked for the student
    x[1] = -INF                       # the student has nothing left
    tok[2, 1] = V                     # outside the vocabulary
    tok[3, 1] = 2 ** 31 - 1
    x[4, 50] = math.nan
    d = torch.ones(T, device="cuda")
    step = ops.distill(x, tok, val, d_loss=d)
    grad = ops.distill_backward(x, tok, val, step["lse"], d)
    assert float(step["loss"][0]) == INF and float(step["loss"][1]) == INF
    assert bool(step["loss"][2:5].isnan().all()) and math.isfinite(float(step["loss"][5]))
    for dx in (step["dlogits"], grad):
        assert bool(dx[0].isfinite().all()) and not bool(dx[1].any()) and bool(dx[2:5].isnan().all()) and bool(dx[5].isfinite().all())


def test_distill_gradient_against_differences():
    T, V, K, h = 2, 23, 5, 2.0 ** -5
    x = _logits(T, V, "f32", scale=1.0)
    tok, val = _teacher(T, K, V)
    tau = 1.5
    one = torch.ones(T, device="cuda")
    dx = ops.distill(x, tok, val, temperature=tau, d_loss=one)["dlogits"]
    # the loss is tau^2 times a logsumexp of x / tau plus a linear function: third derivative below 6 / tau
    bound = h * h / tau + float(_sum_bound(x.double()).max()) * 8 * tau * tau / h
    for j in range(V):
        e = torch.zeros_like(x)
        e[:, j] = h
        d = (ops.distill(x + e, tok, val, temperature=tau)["loss"] - ops.distill(x - e, tok, val, temperature=tau)["loss"]) / (2 * h)
        assert float((d - dx[:, j]).abs().max()) <= bound


# --- how the calls are made --------------------------------------------------------------------------------------------

def test_no_rows():
    x = torch.empty(0, 50, dtype=torch.bfloat16, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    f = torch.empty(0, device="cuda")
    assert ops.token_logprobs(x, t, top_k=3)["top_tokens"].shape == (0, 3)
    assert ops.token_logprobs_backward(x, t, f, d_logprob=f).shape == (0, 50)
    tt, tv = torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda")
    assert ops.distill(x, tt, tv, d_loss=f)["dlogits"].shape == (0, 50)
    assert ops.distill_backward(x, tt, tv, f, f).shape == (0, 50)


def test_results_do_not_depend_on_the_run():
    x = _logits(64, 60001, "bf16")
    tokens = torch.randint(0, 60001, (64,), generator=_gen(5), device="cuda").int()
    tok, val = _teacher(64, 40, 60001)
    one = torch.ones(64, device="cuda")
    a, b = ops.token_logprobs(x, tokens, top_k=20), ops.distill(x, tok, val, d_loss=one)
    for _ in range(5):
        c, d = ops.token_logprobs(x, tokens, top_k=20), ops.distill(x, tok, val, d_loss=one)
        assert all(torch.equal(a[k], c[k]) for k in a) and all(torch.equal(b[k], d[k]) for k in b)


def test_streams_and_graphs():
    """A captured chain, replayed on new contents, on a stream of its own, beside eager calls on another."""
    T, V = 33, 5003
    x = _logits(T, V, "bf16", seed=1)
    tokens = torch.randint(0, V, (T,), generator=_gen(5), device="cuda").int()
    tok, val = _teacher(T, 16, V)
    one = torch.ones(T, device="cuda")
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()

    def chain():
        st = ops.token_logprobs(x, tokens, top_k=4)
        dx = ops.token_logprobs_backward(x, tokens, st["lse"], st["entropy"], one, one)
        ds = ops.distill(x, tok, val, d_loss=one)
        return [st["logprob"], st["top_tokens"], dx, ds["loss"], ds["dlogits"], ops.distill_backward(x, tok, val, ds["lse"], one)]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        captured = chain()
    for seed in (2, 3):
        x.copy_(_logits(T, V, "bf16", seed=seed))
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            graph.replay()
        with torch.cuda.stream(s2):
            eager = chain()
        given = ops.token_logprobs(x, tokens, top_k=4, stream=s2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))
        assert torch.equal(given["logprob"], captured[0])


def test_refusals():
    x = _logits(4, 100, "bf16")
    tokens = torch.zeros(4, dtype=torch.int32, device="cuda")
    f = torch.zeros(4, device="cuda")
    tok, val = _teacher(4, 3, 100)
    wrong = [
        lambda: ops.token_logprobs(x, tokens.long()),
        lambda: ops.token_logprobs(x, tokens[:3]),
        lambda: ops.token_logprobs(x, tokens.cpu()),
        lambda: ops.token_logprobs(x.double(), tokens),
        lambda: ops.token_logprobs(x.t(), tokens),
        lambda: ops.token_logprobs(x[None], tokens),
        lambda: ops.token_logprobs(x[0].expand(4, 100), tokens),
        lambda: ops.token_logprobs(x, tokens, top_k=33),
        lambda: ops.token_logprobs(x, tokens, top_k=-1),
        lambda: ops.token_logprobs(x[:, :0], tokens),
        lambda: ops.token_logprobs_backward(x, tokens, f, d_entropy=f),
        lambda: ops.token_logprobs_backward(x, tokens, f.double(), d_logprob=f),
        lambda: ops.token_logprobs_backward(x, tokens, f, d_logprob=f, out=torch.empty(4, 100, device="cuda")),
        lambda: ops.token_logprobs_backward(x, tokens, f, d_logprob=f, out=torch.empty(4, 99, dtype=x.dtype, device="cuda")),
        lambda: ops.distill(x, tok.long(), val),
        lambda: ops.distill(x, tok, val[:, :2]),
        lambda: ops.distill(x, tok[:3], val[:3]),
        lambda: ops.distill(x, tok.repeat(1, 50), val.repeat(1, 50)),
        lambda: ops.distill(x, tok, val, out=x),
        lambda: ops.distill(x, tok[:, :0], val[:, :0]),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)
    for call in (lambda: ops.token_logprobs(x, tokens, temperature=0.0),
                 lambda: ops.distill(x, tok, val, temperature=math.nan),
                 lambda: ops.token_logprobs_backward(x[:3], tokens[:3], f[:3], d_logprob=f[:3], out=x[1:]),
                 lambda: ops.distill(x[:3], tok[:3], val[:3], d_loss=f[:3], out=x[1:])):
        with pytest.raises(laq.LaqError) as e:
            call()
        assert e.value.status == laq.LAQ_EINVAL
