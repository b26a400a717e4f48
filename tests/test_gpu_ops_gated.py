"""The gated block and its gradient against fp64, its 8-bit activations, and a training step of a block.

Bounds as in tests/test_gpu_ops_linear.py (h_t a rounding to the type t, u = 2^-24, A the bound of a product):
  z is off by A =: a; the activation, 1.13-Lipschitz, of a gate by 1.13 a + 16 u |g| (1 + |g|) =: b; then
  h = act(g) u is off by (|act(g)| + b) a_u + b |u| + 2 u |h| and one rounding h_t |h|;
  dg = dh u act'(g) and du = dh act(g): slopes off by 32 u (1 + g^2) (|g| cut at 20), values by 16 u |g| (1 + |g|), and two
  products' roundings 2 u; each is rounded once, h_t |dz|, which the products carry.
"""
import math

import pytest
import torch

from paper_1909_07588_b200 import laq, ops
from tests.test_gpu_ops_blocks import values
from tests.test_gpu_ops_linear import ACTS, DTYPES, U, _act, _product_bound, _randn, _slope, _within

pytestmark = pytest.mark.gpu


def _check(x, w, bias, act, **kw):
    K, F = x.shape[1], w.shape[0] // 2
    dt = x.dtype
    half, tiny = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    xd, wd = x.double(), w.double()
    z = xd @ wd.T + (0 if bias is None else bias.double())
    zb = _product_bound(xd, wd.T, K) + 4 * U * (z.abs() + (0 if bias is None else bias.double().abs()))
    g, u, a, c = z[:, :F], z[:, F:], zb[:, :F], zb[:, F:]
    v = _act(g, act)
    b = 1.13 * a + 16 * U * g.abs() * (1 + g.abs())
    h = v * u
    hb = (v.abs() + b) * c + b * u.abs() + 2 * U * h.abs()
    got, gz = ops.gated(x, w, bias, activation=act, preact=True, **kw)
    _within(gz, z, zb + half * (z.abs() + zb) + tiny, "z " + act)
    _within(got, h, hb + half * (h.abs() + hb) + tiny, "h " + act)
    return got, gz


SHAPES = [(1, 1, 1), (1, 16, 8), (3, 5, 7), (1, 257, 129), (2, 2048, 64), (4, 50, 1000), (7, 100, 1000), (16, 200, 784), (33, 131, 72), (64, 64, 64),
          (100, 200, 784), (129, 129, 129), (130, 264, 1032), (257, 96, 200), (500, 10, 784), (512, 512, 512), (777, 500, 333),
          (1500, 300, 40), (1024, 768, 2048), (40, 2048, 4096), (5000, 24, 16), (2500, 1100, 600)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, F, K", SHAPES)
def test_forward(M, F, K, dtype):
    dt = DTYPES[dtype]
    x, w, b = _randn(M, K, seed=1, dtype=dt), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5), _randn(2 * F, seed=3, dtype=dt)
    for act in ACTS:
        h, z = _check(x, w, b, act)
        assert torch.equal(ops.gated(x, w, b, activation=act), h)
        h8, z8 = ops.gated(x, w, b, activation=act, preact="packed")
        want = ops.pack8(z)
        assert torch.equal(h8, h) and torch.equal(z8.scales, want.scales)
        assert torch.equal(z8.codes.view(torch.uint8), want.codes.view(torch.uint8))
    _check(x, w, None, "silu")
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, F, K", [(1000, 2048, 64), (2049, 1280, 136), (777, 4096, 72), (130, 128, 64)])
def test_projections_packed_where_they_are_made(M, F, K, dtype):
    """Tiles of whole blocks: bit for bit what pack8 makes of the 16-bit projections, with blocks of zeros, far values and values that
    are no numbers, and with and without a bias."""
    dt = DTYPES[dtype]
    x, w = _randn(M, K, seed=1, dtype=dt), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5)
    b = _randn(2 * F, seed=3, dtype=dt)
    x[3] = 0
    x[5] *= 2.0 ** 10
    x[M - 1] *= 2.0 ** -12
    w[128 % F:128 % F + 128] = 0
    odd = b.clone()
    odd[7], odd[F + 9], odd[2 * F - 1] = math.inf, -math.inf, math.nan
    for bias in (None, b, odd):
        h, z = ops.gated(x, w, bias, activation="gelu", preact=True)
        h8, z8 = ops.gated(x, w, bias, activation="gelu", preact="packed")
        want = ops.pack8(z)
        assert torch.equal(z8.scales, want.scales) and torch.equal(z8.codes.view(torch.uint8), want.codes.view(torch.uint8))
        assert torch.equal(h8.view(torch.int16), h.view(torch.int16))
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, F, K", [(1, 1, 1), (2, 3, 5), (1, 300, 120), (20, 40, 64), (100, 200, 784), (129, 129, 129), (300, 64, 1000),
                                     (600, 520, 136), (2048, 512, 1024), (4100, 16, 24), (64, 1024, 1024)])
def test_gradient(M, F, K, dtype):
    dt = DTYPES[dtype]
    half, tiny = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    x, w = _randn(M, K, seed=1, dtype=dt), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5)
    dh, z = _randn(M, F, seed=3, dtype=dt), _randn(M, 2 * F, seed=4, dtype=dt, scale=2.0)
    xd, wd, d = x.double(), w.double(), dh.double()
    g, u = z.double()[:, :F], z.double()[:, F:]
    for act in ACTS:
        v, s = _act(g, act), _slope(g, act)
        smooth = act in ("gelu", "silu")
        dz = torch.cat([d * u * s, d * v], dim=1)
        own = torch.cat([(d * u).abs() * 32 * U * (1 + g * g), d.abs() * 16 * U * g.abs() * (1 + g.abs())], dim=1) if smooth else 0 * dz
        dzb = own + 2 * U * dz.abs()
        rounded = half * (dz.abs() + dzb) + tiny + dzb
        bx = _product_bound(dz, wd, 2 * F) + 1.01 * (rounded @ wd.abs())
        bw = _product_bound(dz.T, xd, M) + 1.01 * (rounded.T @ xd.abs())
        got = ops.gated_backward(dh, x, w, z, activation=act)
        assert set(got) == {"dx", "dw", "db"}
        _within(got["dx"], dz @ wd, bx + half * ((dz @ wd).abs() + bx) + tiny, "dx " + act)
        _within(got["dw"], dz.T @ xd, bw + half * ((dz.T @ xd).abs() + bw) + tiny, "dw " + act)
        _within(got["db"], dz.sum(0), (M * U + 2 * U) * dz.abs().sum(0) + dzb.sum(0) + 1e-30, "db " + act)
        for k in got:
            only = ops.gated_backward(dh, x, w, z, activation=act, **{n: n == k for n in got})
            assert set(only) == {k} and torch.equal(only[k], got[k])
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, F, K", [(1, 1, 1), (3, 7, 130), (70, 64, 64), (129, 130, 200), (300, 512, 256), (1000, 257, 129)])
def test_gradient_from_packed_activations(M, F, K, dtype):
    """Exactly the gradient of the restored activations: those are numbers of the block's type."""
    dt = DTYPES[dtype]
    x, w = ops.pack8(_randn(M, K, seed=1, dtype=dt)), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5)
    dh, z = _randn(M, F, seed=3, dtype=dt), ops.pack8(_randn(M, 2 * F, seed=4, dtype=dt, scale=2.0))
    xr, zr = ops.unpack8(x, dtype=dt), ops.unpack8(z, dtype=dt)
    for act in ACTS:
        want = ops.gated_backward(dh, xr, w, zr, activation=act)
        for a, b in ((x, zr), (xr, z), (x, z)):
            got = ops.gated_backward(dh, a, w, b, activation=act)
            for k in want:
                assert torch.equal(got[k], want[k]), (act, k)
    ops.check_status()


def test_far_gates():
    """Values and slopes where exp overflows or g^3 does, and gates that are no numbers."""
    for dt in DTYPES.values():
        far = [0.0, -0.0, 5.0, -5.0, 19.5, -19.5, 21.0, -21.0, 100.0, -100.0, 3e4, -3e4] + ([1e30, -1e30] if dt == torch.bfloat16 else [])
        n = len(far)
        z = torch.tensor(far + [0.5] * n, device="cuda", dtype=dt).repeat(16, 1)
        x, w = torch.zeros(16, 16, device="cuda", dtype=dt), torch.zeros(2 * n, 16, device="cuda", dtype=dt)
        x[:, 0] = 1
        w[:, 0] = z[0]
        g = z[:, :n].double()
        for act in ("relu", "gelu", "silu"):
            h = ops.gated(x, w, activation=act).double()
            assert torch.allclose(h, 0.5 * _act(g, act), rtol=torch.finfo(dt).eps, atol=1e-6), act
            got = ops.gated_backward(torch.ones_like(z[:, :n]), x, w, z, activation=act, dx=False, dw=False)["db"].double() / 16
            assert torch.allclose(got[:n], 0.5 * _slope(g[0].clamp(-1e3, 1e3), act), rtol=1e-5, atol=1e-6), act
            assert torch.allclose(got[n:], _act(g[0], act), rtol=1e-5, atol=1e-6), act
        z[3, 2] = math.nan
        for act in ACTS:
            db = ops.gated_backward(torch.ones_like(z[:, :n]), x, w, z, activation=act, dx=False, dw=False)["db"]
            bad = torch.zeros(2 * n, dtype=torch.bool, device="cuda")
            bad[2], bad[n + 2] = act != "none", True       # without an activation the gate's slope is 1 whatever the gate
            assert torch.equal(db.isnan(), bad), act


@pytest.mark.parametrize("M, F, K", [(1, 40, 56), (3, 40, 1024), (70, 40, 56), (300, 136, 264)])
def test_strides_and_odd_addresses(M, F, K):
    dt = torch.bfloat16

    def inside(rows, cols, left, pad, seed):
        t = _randn(rows + 2, cols + left + pad, seed=seed, dtype=dt)
        return t, t[1:1 + rows, left:left + cols]

    for left, pad in ((0, 0), (8, 8), (1, 2), (3, 4)):
        _, x = inside(M, K, left, pad, 1)
        _, w = inside(2 * F, K, left, pad, 2)
        big, h = inside(M, F, left, pad, 3)
        b = _randn(2 * F + 1, seed=5, dtype=dt)[left % 2:2 * F + left % 2]
        before = big.clone()
        got, z = _check(x, w, b, "gelu", out=h)
        assert got is h
        mark = torch.ones_like(big, dtype=torch.bool)
        mark[1:1 + M, left:left + F] = False
        assert torch.equal(big[mark], before[mark])
        _, dh = inside(M, F, left, pad, 6)
        _, zz = inside(M, 2 * F, left, pad, 7)
        got = ops.gated_backward(dh, x, w, zz, activation="silu")
        want = ops.gated_backward(dh.contiguous(), x.contiguous(), w.contiguous(), zz.contiguous(), activation="silu")
        for k in want:
            assert torch.equal(got[k], want[k]), k
    ops.check_status()


def test_no_rows():
    x, w = torch.empty(0, 24, device="cuda").bfloat16(), _randn(16, 24, seed=1, dtype=torch.bfloat16)
    assert ops.gated(x, w).shape == (0, 8)
    h, z = ops.gated(x, w, preact="packed")
    assert h.shape == (0, 8) and z.shape == (0, 16)
    got = ops.gated_backward(torch.empty(0, 8, device="cuda").bfloat16(), x, w, z)
    assert got["dx"].shape == (0, 24) and not bool(got["dw"].any()) and not bool(got["db"].any())


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(act):
    """sum(h) against differences of the forward call in fp16, as a function of one gate and of one up (test_gpu_ops_linear.py has
    the bounds: h^2 / 6 of a third derivative below 2, a rounding of h over h)."""
    step = 2.0 ** -4
    v = torch.arange(-64, 65, device="cuda").half() * step
    n = v.numel()
    x = torch.zeros(8, 16, device="cuda").half()
    x[:, 0] = 1

    def value(gates, ups):
        w = torch.nn.functional.pad(torch.cat([gates, ups])[:, None], (0, 15))
        return ops.gated(x, w, activation=act)[0].double()

    ones = torch.ones_like(v)
    z = torch.cat([v, 1.5 * ones]).repeat(8, 1).contiguous()
    w = torch.zeros(2 * n, 16, device="cuda").half()
    db = ops.gated_backward(torch.ones(8, n, device="cuda").half(), x, w, z, activation=act, dx=False, dw=False)["db"].double() / 8
    up, down = value(v + step, 1.5 * ones), value(v - step, 1.5 * ones)
    bound = 1.5 * 2 * step * step / 6 + 2.0 ** -11 * torch.maximum(up.abs(), down.abs()) / step + 1e-6
    assert bool(((up - down) / (2 * step) - db[:n]).abs().le(bound).all())
    up, down = value(v, 2 * ones), value(v, ones)                # linear in the ups: roundings alone
    assert bool(((up - down) - db[n:]).abs().le(2.0 ** -11 * (up.abs() + down.abs()) + 1e-6).all())


def test_bounded_wait():
    x, w = _randn(300, 256, seed=1, dtype=torch.bfloat16), _randn(512, 256, seed=2, dtype=torch.bfloat16)
    before = ops.gated(x, w)
    ops.check_status()
    ops.gated(x, w, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    ops.gated_backward(_randn(300, 256, seed=3, dtype=torch.bfloat16), x, w, _randn(300, 512, seed=4, dtype=torch.bfloat16), flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError):
        ops.check_status()
    assert torch.equal(ops.gated(x, w), before)
    ops.check_status()


def test_captured_and_replayed_beside_another_graph():
    """Two graphs with workspaces of their own, replayed at the same time on two streams."""
    x, w = _randn(200, 504, seed=1, dtype=torch.bfloat16), _randn(640, 504, seed=2, dtype=torch.bfloat16, scale=504 ** -0.5)
    dh = _randn(200, 320, seed=3, dtype=torch.bfloat16)
    ops.init()

    def step():
        h, z = ops.gated(x, w, preact="packed")
        return h, z, ops.gated_backward(dh, ops.pack8(x), w, z)

    want = step()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out, torch.cuda.Stream()))
    for _ in range(3):
        for g, out, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, (h, z, d), _ in graphs:
        assert torch.equal(h, want[0]) and torch.equal(z.codes.view(torch.uint8), want[1].codes.view(torch.uint8))
        for k in d:
            assert torch.equal(d[k], want[2][k])
    ops.check_status()


def test_a_block_trained_through_to_the_upload():
    """x -> gated -> linear8 -> loss and back, activations kept in 8 bits, and the weights' gradients through the quantizer: each
    gradient against fp64 autograd on the values that the calls were given."""
    M, K, F, V, dt = 64, 96, 160, 50, torch.bfloat16
    x, wg = _randn(M, K, seed=1, dtype=dt), _randn(2 * F, K, seed=2, dtype=dt, scale=K ** -0.5)
    wd = ops.pack8(_randn(V, F, seed=3, dtype=torch.float32, scale=F ** -0.5), tiles=True)
    tokens = torch.randint(0, V, (M,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).int()
    h, z = ops.gated(x, wg, preact="packed")
    h8, x8 = ops.pack8(h), ops.pack8(x)
    logits = ops.linear8(h8, wd)
    s = ops.token_logprobs(logits, tokens)
    dlogits = ops.token_logprobs_backward(logits, tokens, s["lse"], d_logprob=torch.full((M,), -1.0 / M, device="cuda"))
    down = ops.linear_backward(dlogits, h8, wd)
    up = ops.gated_backward(down["dx"], x8, wg, z)

    leaves = [t.double().requires_grad_() for t in (values(h8), values(wd))]
    loss = torch.nn.functional.cross_entropy(leaves[0] @ leaves[1].T, tokens.long())
    dh, dwd = torch.autograd.grad(loss, leaves)
    # roundings of the logits (2^-8 of up to 8, in exp), of dlogits and of the results
    assert float((down["dx"].double() - dh).norm() / dh.norm()) < 0.04
    assert float((down["dw"].double() - dwd).norm() / dwd.norm()) < 0.04
    zv = values(z).requires_grad_()
    out = torch.nn.functional.silu(zv[:, :F]) * zv[:, F:]
    dz, = torch.autograd.grad(out, zv, down["dx"].double())
    for got, want in ((up["dx"], dz @ wg.double()), (up["dw"], dz.T @ values(x8)), (up["db"], dz.sum(0))):
        assert float((got.double() - want).norm() / want.norm()) < 0.01            # two roundings of 2^-9 at most, root mean square
    g = torch.cat([up["dw"].float().flatten(), down["dw"].float().flatten()])
    ctx = laq.Laq(model=laq.MODEL_EXTERNAL, M=1, p=g.numel(), alpha=0.1, b=8, D=1, xi=[0.0], tbar=10, trace_capacity=1)
    ctx.set_gradients(g.reshape(1, -1).cpu().numpy())
    tr = ctx.step(1, trace=True)
    assert float(tr["R"][0, 0]) == float(g.abs().max())
    ctx.close()
    ops.check_status()
