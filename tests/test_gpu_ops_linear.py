"""linear and its gradient against fp64, and a run of the operators together with the quantizer.

Bounds (t = the operands' type, h_t = finfo(t).eps / 2 a rounding to it, u = 2^-24):
  products of two 16-bit numbers are exact in fp32; the tensor core adds them 16 at a time to an fp32 accumulator, each
  step off by at most an ulp (2^-23) of the sum of magnitudes so far, and a split adds a few more: a product is off by at
  most (K / 16 + 16) 2^-23 sum |x w| =: A;
  the activations are 1.13-Lipschitz at most and their own arithmetic (ex2 and rcp to 2^-22 relative, arguments to
  a few u) is off by 16 u |z| (1 + |z|); then one rounding h_t |y|;
  dZ is rounded once, h_t |dz|, where the activation is not none or relu: h_t sum |dz w| more in dX, and so in dW;
  slopes are off by 32 u (1 + z^2) at most (|z| cut at 20: beyond it they are 0 or 1).
"""
import math

import numpy as np
import pytest
import torch

from paper_1909_07588_b200 import laq, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ["none", "relu", "gelu", "silu"]
GELU = math.sqrt(2 / math.pi)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(*shape, seed, dtype, scale=1.0):
    return (torch.randn(*shape, generator=_gen(seed), device="cuda") * scale).to(dtype)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(GELU * (z + 0.044715 * z ** 3)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if act == "gelu":
        th = torch.tanh(GELU * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * GELU * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _within(got, want, bound, what):
    excess = ((got.double() - want).abs() - bound).max()
    assert bool(got.isfinite().all()) and float(excess) <= 0, "%s: off by %g more than it may" % (what, float(excess))


def _product_bound(a, b, K):
    """of a @ b with K terms"""
    return (K / 16 + 16) * 2.0 ** -23 * (a.abs() @ b.abs())


def _check_forward(x, w, bias, act, residual, preact=True, **kw):
    K = x.shape[1]
    half = torch.finfo(x.dtype).eps / 2
    xd, wd = x.double(), w.double()
    z = xd @ wd.T + (0 if bias is None else bias.double())
    y = _act(z, act) + (0 if residual is None else residual.double())
    zb = _product_bound(xd, wd.T, K) + 4 * U * (z.abs() + (0 if bias is None else bias.double().abs()))
    yb = 1.13 * zb + 16 * U * z.abs() * (1 + z.abs()) + 2 * U * y.abs()
    tiny = torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps
    got = ops.linear(x, w, bias, activation=act, residual=residual, preact=preact, **kw)
    if preact:
        got, gz = got
        _within(gz, z, zb + half * (z.abs() + zb) + tiny, "z")
    _within(got, y, yb + half * (y.abs() + yb) + tiny, "y")
    return got


SHAPES = [(1, 1, 1), (1, 16, 8), (3, 5, 7), (1, 257, 129), (2, 4096, 64), (7, 100, 1000), (16, 200, 784), (33, 131, 72), (64, 64, 64),
          (100, 200, 784), (129, 129, 129), (130, 520, 1032), (257, 96, 200), (500, 10, 784), (512, 512, 512), (777, 1000, 333),
          (1500, 300, 40), (1024, 768, 2048), (40, 2048, 4096), (5000, 24, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", SHAPES)
def test_forward(M, N, K, dtype):
    dt = DTYPES[dtype]
    x, w = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt, scale=K ** -0.5)
    b, r = _randn(N, seed=3, dtype=dt), _randn(M, N, seed=4, dtype=dt)
    for act in ACTS:
        _check_forward(x, w, b, act, r)
    _check_forward(x, w, None, "none", None, preact=False)
    _check_forward(x, w, b, "gelu", None, preact=False)
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(1, 1, 1), (2, 3, 5), (1, 300, 120), (20, 40, 64), (100, 200, 784), (129, 129, 129), (300, 64, 1000),
                                     (1000, 200, 784), (600, 520, 136), (2048, 512, 1024), (4100, 16, 24), (64, 2048, 1024)])
def test_gradient(M, N, K, dtype):
    dt = DTYPES[dtype]
    half, tiny = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    x, w = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt, scale=K ** -0.5)
    dy, z = _randn(M, N, seed=3, dtype=dt), _randn(M, N, seed=4, dtype=dt, scale=2.0)
    xd, wd, zd = x.double(), w.double(), z.double()
    for act in ACTS:
        dz = dy.double() * _slope(zd, act)
        smooth = act in ("gelu", "silu")
        dzb = (32 * U * dy.double().abs() * (1 + zd * zd) if smooth else 0 * dz)
        round_dz = (half * (dz.abs() + dzb) + tiny if smooth else 0 * dz) + dzb
        bx = _product_bound(dz, wd, N) + 1.01 * (round_dz @ wd.abs())
        bw = _product_bound(dz.T, xd, M) + 1.01 * (round_dz.T @ xd.abs())
        got = ops.linear_backward(dy, x, w, z=None if act == "none" else z, activation=act)
        assert set(got) == {"dx", "dw", "db"}
        _within(got["dx"], dz @ wd, bx + half * ((dz @ wd).abs() + bx) + tiny, "dx " + act)
        _within(got["dw"], dz.T @ xd, bw + half * ((dz.T @ xd).abs() + bw) + tiny, "dw " + act)
        # a run's rows, then the runs: at most M additions
        _within(got["db"], dz.sum(0), (M * U + 2 * U) * dz.abs().sum(0) + dzb.sum(0) + 1e-30, "db " + act)
        if not smooth:
            g32 = ops.linear_backward(dy, x, w, z=None if act == "none" else z, activation=act, dw_dtype=torch.float32, dx=False, db=False)
            assert set(g32) == {"dw"} and g32["dw"].dtype == torch.float32
            _within(g32["dw"], dz.T @ xd, bw + U * (dz.T @ xd).abs() + 1e-30, "fp32 dw " + act)
    ops.check_status()


def test_far_preactivations():
    """Activations and slopes where exp overflows or z^3 does."""
    for dt in DTYPES.values():
        far = [0.0, -0.0, 5.0, -5.0, 19.5, -19.5, 21.0, -21.0, 100.0, -100.0, 6e4, -6e4] + ([1e30, -1e30] if dt == torch.bfloat16 else [])
        z = torch.tensor(far, device="cuda", dtype=dt).repeat(16, 1)
        n = z.shape[1]
        x, w = torch.zeros(16, 16, device="cuda", dtype=dt), torch.zeros(n, 16, device="cuda", dtype=dt)
        x[:, 0] = 1
        w[:, 0] = z[0]
        for act in ("relu", "gelu", "silu"):
            y = ops.linear(x, w, activation=act).double()
            zd = z.double()
            assert torch.allclose(y, _act(zd, act), rtol=torch.finfo(dt).eps, atol=1e-6), act
            got = ops.linear_backward(torch.ones_like(z), x, w, z=z, activation=act, dx=False, dw=False)["db"].double() / 16
            assert torch.allclose(got, _slope(zd[0].clamp(-1e3, 1e3), act), rtol=1e-5, atol=1e-6), act


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(1, 40, 56), (70, 40, 56), (300, 136, 264)])
def test_strides_and_odd_addresses(M, N, K, dtype):
    """Operands and results inside wider tensors; what lies beside them stays as it was."""
    dt = DTYPES[dtype]

    def inside(rows, cols, left, pad, seed):
        t = _randn(rows + 2, cols + left + pad, seed=seed, dtype=dt)
        return t, t[1:1 + rows, left:left + cols]

    for left, pad in ((0, 0), (8, 8), (1, 2), (3, 4)):
        _, x = inside(M, K, left, pad, 1)
        _, w = inside(N, K, left, pad, 2)
        _, r = inside(M, N, left, pad, 3)
        big, y = inside(M, N, left, pad, 4)
        b = _randn(N + 1, seed=5, dtype=dt)[left % 2:N + left % 2]
        before = big.clone()
        _check_forward(x, w, b, "gelu", r, preact=False, out=y)
        mark = torch.ones_like(big, dtype=torch.bool)
        mark[1:1 + M, left:left + N] = False
        assert torch.equal(big[mark], before[mark])
        # in place over the residual
        rr = r.clone()
        _check_forward(x, w, b, "silu", r.clone(), preact=False)
        y2 = ops.linear(x, w, b, activation="silu", residual=rr, out=rr)
        assert y2 is rr and torch.equal(rr, ops.linear(x, w, b, activation="silu", residual=r))
        _, dy = inside(M, N, left, pad, 6)
        _, z = inside(M, N, left, pad, 7)
        got = ops.linear_backward(dy, x, w, z=z, activation="relu", dw_dtype=torch.float32)
        want = ops.linear_backward(dy.contiguous(), x.contiguous(), w.contiguous(), z=z.contiguous(), activation="relu", dw_dtype=torch.float32)
        for k in want:
            assert torch.equal(got[k], want[k]), k
    ops.check_status()


def test_no_rows_and_single_rows():
    x, w = torch.empty(0, 24, device="cuda").bfloat16(), _randn(8, 24, seed=1, dtype=torch.bfloat16)
    assert ops.linear(x, w).shape == (0, 8)
    got = ops.linear_backward(torch.empty(0, 8, device="cuda").bfloat16(), x, w)
    assert got["dx"].shape == (0, 24) and not bool(got["dw"].any()) and not bool(got["db"].any())


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(act):
    """The loss sum(y) in fp16 differences of z: the slope that linear_backward uses against the forward call's own values,
    taken at points h apart (h = 2^-4): off by h^2 / 6 of a third derivative below 2, and by y's rounding over h."""
    h = 2.0 ** -4
    z = torch.arange(-64, 65, device="cuda").half() * h
    n = z.numel()
    x = torch.zeros(8, 16, device="cuda").half()
    x[:, 0] = 1
    value = lambda v: ops.linear(x, torch.nn.functional.pad(v[:, None], (0, 15)), activation=act)[0].double()
    d = (value(z + h) - value(z - h)) / (2 * h)
    got = ops.linear_backward(torch.ones(8, n, device="cuda").half(), x, torch.zeros(n, 16, device="cuda").half(), z=z.repeat(8, 1),
                              activation=act, dx=False, dw=False)["db"].double() / 8
    assert float((got - d).abs().max()) <= h * h * 2 / 6 + 2.0 ** -11 * 5 / h


def test_workspaces_streams_and_graphs():
    M, N, K = 257, 133, 205                       # odd rows: every operand is copied to the workspace
    dt = torch.bfloat16
    x, w, b = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt), _randn(N, seed=3, dtype=dt)
    dy = _randn(M, N, seed=4, dtype=dt)
    ops.init()
    ws = [torch.empty(1 << 20, dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]

    def chain(workspace=None, stream=None):
        y, z = ops.linear(x, w, b, activation="gelu", preact=True, workspace=workspace, stream=stream)
        g = ops.linear_backward(dy, x, w, z=z, activation="gelu", workspace=workspace, stream=stream)
        return [y, z, g["dx"], g["dw"], g["db"]]

    torch.cuda.synchronize()
    graphs, outs = [], []
    for s, k in zip(streams, ws):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(chain(workspace=k))
        graphs.append(g)
    for seed in (5, 6):
        x.copy_(_randn(M, K, seed=seed, dtype=dt))
        want = chain()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):         # two captured graphs at the same time, each with a workspace of its own
            with torch.cuda.stream(s):
                g.replay()
                g.replay()
        other = chain(stream=streams[0])
        torch.cuda.synchronize()
        for got in outs + [other]:
            assert all(torch.equal(p, q) for p, q in zip(got, want))
    with pytest.raises(laq.LaqError) as e:
        ops.linear(x, w, b, workspace=torch.empty(1000, dtype=torch.uint8, device="cuda"))
    assert e.value.status == laq.LAQ_EWORKSPACE
    ops.check_status()


FEW = [(1, 1), (3, 2), (5, 7), (4, 8), (17, 9), (130, 64), (10, 784), (200, 785), (131, 1000), (300, 2056), (1026, 4099), (4096, 512),
       (9472, 520), (9473, 512), (9477, 1024), (19001, 263)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N, K", FEW)
def test_forward_of_few_rows(N, K, dtype):
    dt = DTYPES[dtype]
    for M in (1, 2, 3, 4, 5):
        x, w = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt, scale=K ** -0.5)
        b, r = _randn(N, seed=3, dtype=dt), _randn(M, N, seed=4, dtype=dt)
        for act, bias, res in (("none", None, None), ("gelu", b, r), ("silu", b, None)):
            _check_forward(x, w, bias, act, res)
        # columns of wider matrices: rows that start at any element, and rows that start at vectors
        for at in (1, 8):
            wide = _randn(N, K + 24, seed=5, dtype=dt, scale=K ** -0.5)
            xs = _randn(M, K + 24, seed=6, dtype=dt)
            _check_forward(xs[:, at:at + K], wide[:, at:at + K], b, "relu", r)
    ops.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("K", [8, 264, 1000, 4097])
def test_few_rows_with_infinities(K, dtype):
    """An infinity gives infinities, or what is not a number where it meets a zero, in its own row and nowhere else."""
    dt = DTYPES[dtype]
    w = _randn(37, K, seed=2, dtype=dt).abs() + 0.5
    for M in (1, 2, 3, 4):
        for at in (0, K // 2, K - 1):
            x = _randn(M, K, seed=1, dtype=dt)
            x[0, at] = -math.inf
            w[5, at] = 0.0
            y = ops.linear(x, w)
            assert bool(y[0, 5].isnan()) and bool((y[0, :5] == -math.inf).all()) and bool((y[0, 6:] == -math.inf).all())
            assert bool(y[1:].isfinite().all())
            w[5, at] = 1.0


@pytest.mark.parametrize("M, N, K", [(64, 200, 784), (257, 133, 205), (2048, 1024, 512), (16, 1024, 2048)])
def test_calls_without_a_pause(M, N, K):
    # the kernels of a call, and those of the calls behind it, wait for what they read and for the memory that they reuse
    w, z, b = (_randn(*s, seed=70 + i, dtype=torch.bfloat16) for i, s in enumerate([(N, K), (M, N), (N,)]))
    xs = [_randn(M, K, seed=80 + i, dtype=torch.bfloat16) for i in range(3)]
    dys = [_randn(M, N, seed=90 + i, dtype=torch.bfloat16) for i in range(3)]

    def run(i):
        g = ops.linear_backward(dys[i], xs[i], w, z=z, activation="gelu")
        return ops.linear(xs[i], w, b, activation="gelu"), g["dx"], g["dw"], g["db"]

    want = []
    for i in range(3):
        torch.cuda.synchronize()
        want.append(run(i))
        torch.cuda.synchronize()
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for it in range(60):
        for got, one in zip(run(it % 3), want[it % 3]):
            wrong += (got != one).sum()
    assert int(wrong) == 0
    ops.check_status()


def test_first_calls_of_a_process_may_be_captured():
    """Nothing that a first call sets up (shared-memory limits, occupancy, the driver's entry point) disturbs a capture."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_1909_07588_b200 import ops
ops.init()
x = torch.randn(300, 264, device="cuda").bfloat16(); w = torch.randn(3000, 264, device="cuda").bfloat16()
tok = torch.randint(0, 3000, (300, 9), device="cuda").int(); val = torch.randn(300, 9, device="cuda"); one = torch.ones(300, device="cuda")
y = torch.randint(0, 3000, (300,), device="cuda").int()
def chain():
    s = ops.linear(x, w)
    a = ops.token_logprobs(s, y, top_k=3)
    b = ops.distill(s, tok, val, d_loss=one)
    g = ops.linear_backward(b["dlogits"], x, w, dw_dtype=torch.float32)
    return [s, a["logprob"], ops.token_logprobs_backward(s, y, a["lse"], d_logprob=one), b["loss"], g["dx"], g["dw"], g["db"]]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = chain()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(got, chain()))
ops.check_status()
print("captured")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]


def test_refusals():
    dt = torch.bfloat16
    x, w = _randn(4, 24, seed=1, dtype=dt), _randn(8, 24, seed=2, dtype=dt)
    y = _randn(4, 8, seed=3, dtype=dt)
    wrong = [
        lambda: ops.linear(x.float(), w.float()), lambda: ops.linear(x, w.half()), lambda: ops.linear(x, w[:, :23]),
        lambda: ops.linear(x, w, y[0].float()), lambda: ops.linear(x, w, y[0, :7]), lambda: ops.linear(x, w, activation="tanh"),
        lambda: ops.linear(x, w, residual=y[:3]), lambda: ops.linear(x, w, residual=y.half()), lambda: ops.linear(x, w.t()),
        lambda: ops.linear(x.t(), w), lambda: ops.linear(x[0], w), lambda: ops.linear(x[:, :0], w[:, :0]), lambda: ops.linear(x, w[:0]),
        lambda: ops.linear(x, w.cpu()), lambda: ops.linear(x, w, out=y.float()),
        lambda: ops.linear_backward(y, x, w, activation="gelu"), lambda: ops.linear_backward(y[:3], x, w),
        lambda: ops.linear_backward(y, x, w, dw_dtype=torch.float16),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)
    for act in ("gelu", "silu"):                  # 16 bits of dZ would not justify 32 of dW
        with pytest.raises(laq.LaqError) as e:
            ops.linear_backward(y, x, w, z=y, activation=act, dw_dtype=torch.float32)
        assert e.value.status == laq.LAQ_EINVAL and "fp32" in str(e.value)


@pytest.mark.parametrize("M, N, K", [(16, 256, 4096), (300, 300, 512), (2048, 1024, 1024)])
def test_starved_product_runs_out_and_is_reported(M, N, K):
    """One block's loader issues no copies: its waits run out, the call returns, the next check says so, and the same call
    without that works.  (A split tile, single blocks, pairs.)"""
    dt = torch.bfloat16
    x, w = _randn(M, K, seed=1, dtype=dt), _randn(N, K, seed=2, dtype=dt)
    want = ops.linear(x, w)
    ops.check_status()
    ops.linear(x, w, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    ops.check_status()
    assert torch.equal(ops.linear(x, w), want)
    ops.check_status()


# --- a run of them together --------------------------------------------------------------------------------------------

class _Model:
    """A classifier over V classes: h = x + gelu(x W1^T + b1), logits = h W2^T; parameters in fp32, layers in bf16."""

    def __init__(self, D, V, seed):
        rng = np.random.default_rng(seed)
        self.D, self.V = D, V
        self.theta = (rng.standard_normal(D * D + D + V * D) * 0.2).astype(np.float32)

    def parts(self, theta):
        D, V = self.D, self.V
        t = torch.from_numpy(theta).cuda() if isinstance(theta, np.ndarray) else theta
        return t[:D * D].view(D, D), t[D * D:D * D + D], t[D * D + D:].view(V, D)

    def gradient(self, theta, x, loss):
        """Through the operators; loss(logits) gives (value, logits' gradient)."""
        W1, b1, W2 = (p.bfloat16().contiguous() for p in self.parts(theta))
        h, z = ops.linear(x, W1, b1, activation="gelu", residual=x, preact=True)
        logits = ops.linear(h, W2)
        value, dlogits = loss(logits)
        g2 = ops.linear_backward(dlogits, h, W2, dw_dtype=torch.float32, db=False)
        g1 = ops.linear_backward(g2["dx"], x, W1, z=z, activation="gelu", dx=False)
        return value, torch.cat([g1["dw"].float().reshape(-1), g1["db"], g2["dw"].reshape(-1)])

    def plain(self, theta, x, loss):
        W1, b1, W2 = self.parts(theta)
        W1, b1, W2 = (p.bfloat16().double().requires_grad_() for p in (W1, b1, W2))
        xd = x.double()
        h = xd + torch.nn.functional.gelu(xd @ W1.T + b1, approximate="tanh")
        value = loss(h @ W2.T)
        value.backward()
        return value.detach(), torch.cat([p.grad.reshape(-1) for p in (W1, b1, W2)])


@pytest.mark.parametrize("kind", ["logprobs", "distill"])
def test_local_gradients_of_a_larger_model(kind):
    """Two workers' gradients through layer, loss and their gradients, handed to the library as external gradients; with
    quantizer and trigger off an iteration is gradient descent on their sum.

    Roundings to bf16 (2^-9 each, relative to the rounded value): h, logits, dlogits, dx, z, dz and dW1, seven in a row at
    most on the way to any parameter; their first-order effects are relative to the vectors' norms, so 7 2^-9 (about 1.4 %)
    times the growth through the layers.  The layers are near an identity plus a small part: a factor of two covers it."""
    D, V, T, M = 48, 1000, 96, 2
    model = _Model(D, V, 1)
    theta = model.theta
    total, plain_total = 0, 0
    grads = []
    for m in range(M):
        x = _randn(T, D, seed=10 + m, dtype=torch.bfloat16)
        y = torch.randint(0, V, (T,), generator=_gen(20 + m), device="cuda").int()
        if kind == "logprobs":
            w = torch.rand(T, generator=_gen(30 + m), device="cuda") + 0.5           # policy-gradient weights

            def loss(logits):
                st = ops.token_logprobs(logits, y)
                value = -(w * st["logprob"]).mean() - 0.1 * st["entropy"].mean()
                return value, ops.token_logprobs_backward(logits, y, st["lse"], st["entropy"], -w / T, torch.full_like(w, -0.1 / T))

            def plain(s):
                logp = torch.log_softmax(s, dim=1)
                return -(w.double() * logp.gather(1, y.long()[:, None])[:, 0]).mean() + 0.1 * (logp.exp() * logp).sum(1).mean()
        else:
            tok = torch.randint(0, V, (T, 8), generator=_gen(40 + m), device="cuda").int()
            val = torch.randn(T, 8, generator=_gen(50 + m), device="cuda")

            def loss(logits):
                res = ops.distill(logits, tok, val, temperature=2.0, d_loss=torch.full((T,), 1.0 / T, device="cuda"), out=logits)
                return res["loss"].mean(), res["dlogits"]

            def plain(s):
                q = torch.softmax(val.double() / 2, dim=1)
                logp = torch.log_softmax(s / 2, dim=1).gather(1, tok.long())
                return 4 * (q * (q.log() - logp)).sum(1).mean()
        value, g = model.gradient(theta, x, loss)
        pv, pg = model.plain(theta, x, plain)
        assert abs(float(value) - float(pv)) <= 2 * 2 * 2.0 ** -9 * abs(float(pv))
        assert float((g.double() - pg).norm()) <= 2 * 7 * 2.0 ** -9 * float(pg.norm())
        grads.append(g)
        total, plain_total = total + float(value), plain_total + float(pv)
    ops.check_status()
    ctx = laq.Laq(model=laq.MODEL_EXTERNAL, M=M, p=theta.size, alpha=0.25, b=8, D=1, xi=[0.0], tbar=10, theta0=theta,
                  flags=laq.FLAG_QUANT_OFF | laq.FLAG_TRIGGER_OFF)
    ctx.set_gradients(torch.stack(grads))
    ctx.step(1)
    got = ctx.get_state(big=False)["theta"]
    agg = (grads[0] + grads[1]).cpu().numpy()
    np.testing.assert_array_equal(got, theta - np.float32(0.25) * agg)
    # quantized to 8 bits an upload is within half a grid step of the gradient: R / 255, and the fp32 operations that take
    # it there: d, d + R, s and the quotient move t by at most 4 u of 255, that is 8 R u of d, and s q and the difference to R
    # round by 2 R u each: 12 R u together
    q = laq.Laq(model=laq.MODEL_EXTERNAL, M=M, p=theta.size, alpha=0.25, b=8, D=1, xi=[0.0], tbar=10, theta0=theta)
    q.set_gradients(torch.stack(grads))
    q.step(1)
    state = q.get_state()
    for m in range(M):
        R = float(grads[m].abs().max())
        assert float(np.abs(state["qprev"][m] - grads[m].cpu().numpy()).max()) <= R / 255 + 12 * R * U
    ctx.close()
    q.close()
