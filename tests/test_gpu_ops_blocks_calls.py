"""How calls on 8-bit matrices and of the gated block stand beside each other and beside the rest of a program, and how far they reach."""
import math

import pytest
import torch

from paper_1909_07588_b200 import laq, ops
from tests.test_gpu_ops_blocks import _check8, _pair, values
from tests.test_gpu_ops_calls import _run
from tests.test_gpu_ops_gated import _check as _check_gated
from tests.test_gpu_ops_linear import _act, _product_bound, _randn, _slope, _within

pytestmark = pytest.mark.gpu
BF = torch.bfloat16

SETUP = """
import torch
from paper_1909_07588_b200 import laq, ops
bf = torch.bfloat16

def made(dt=bf, M=300, F=136, K=264, odd=0):
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return dict(x=rnd(M, K + odd).to(dt)[:, odd:], w=rnd(2 * F, K).to(dt), v=rnd(F, K), b=rnd(2 * F).to(dt), dh=rnd(M, F).to(dt), z=rnd(M, 2 * F).to(dt), dt=dt)

def flat(v):
    return [u for t in (v.values() if isinstance(v, dict) else v) for u in ([t.codes.view(torch.uint8), t.scales] if isinstance(t, ops.Packed8) else [t])]

def restored(t, s):
    p, q = ops.pack8(t["x"], stream=s), ops.pack8(t["v"], tiles=True, stream=s)
    return [p, q, ops.unpack8(p, dtype=t["dt"], stream=s)]

def eight(t, s):
    p, q = ops.pack8(t["x"], stream=s), ops.pack8(t["v"], tiles=True, stream=s)
    y, z = ops.linear8(p, q, t["b"][:t["v"].shape[0]], activation="gelu", residual=t["dh"], preact=True, dtype=t["dt"], stream=s)
    d = ops.linear_backward(t["dh"], p, q, z=ops.pack8(z, stream=s), activation="gelu", stream=s)
    return [y, z] + list(d.values())

calls = [
    restored,
    eight,
    lambda t, s: ops.gated(t["x"], t["w"], t["b"], preact=True, stream=s),
    lambda t, s: ops.gated(t["x"], t["w"], preact="packed", stream=s),
    lambda t, s: ops.gated_backward(t["dh"], t["x"], t["w"], t["z"], stream=s),
    lambda t, s: ops.gated_backward(t["dh"], ops.pack8(t["x"], stream=s), t["w"], ops.pack8(t["z"], stream=s), stream=s),
]
"""


def test_inputs_may_be_let_go_of_when_a_call_on_another_stream_has_returned():
    assert "done" in _run(SETUP + """
side = torch.cuda.Stream()
for call in calls:
    want = flat(call(made(), None))
    torch.cuda.synchronize()
    t = made()
    shapes = [(v.shape, v.dtype) for v in t.values() if isinstance(v, torch.Tensor)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    got = call(t, side)
    t = None
    for _ in range(3):
        again = [torch.zeros(s, dtype=d, device="cuda") for s, d in shapes]
    torch.cuda.synchronize()
    for a, b in zip(flat(got), want):
        assert torch.equal(a, b)
ops.check_status()
print("done")
""")


def test_first_calls_of_a_thread():
    assert "done" in _run(SETUP + """
import concurrent.futures as cf
for call in calls:
    t = made()
    torch.cuda.synchronize()
    with cf.ThreadPoolExecutor(1) as pool:
        got = flat(pool.submit(call, t, None).result(timeout=60))
        torch.cuda.synchronize()
    for a, b in zip(got, flat(call(t, None))):
        assert torch.equal(a, b)
ops.check_status()
print("done")
""")


@pytest.mark.parametrize("which", range(6))
def test_first_calls_of_a_process_under_capture(which):
    assert "done" in _run(SETUP + """
t = made()
ops.init()
torch.cuda.synchronize()
call = calls[%d]
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = flat(call(t, None))
g.replay()
torch.cuda.synchronize()
for a, b in zip(got, flat(call(t, None))):
    assert torch.equal(a, b)
ops.check_status()
print("done")
""" % which)


def test_only_the_first_call_takes_device_memory_for_code():
    assert "done" in _run(SETUP + """
for call in calls:
    call(made(M=8, F=8, K=8), None)
torch.cuda.synchronize()

def used():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved()

for dt in (torch.float32, bf, torch.float16):
    torch.randn(3, 4, device="cuda").to(dt)
start = used()
for dt in (bf, torch.float16):
    for M, F, K in ((1, 40, 4000), (2, 40, 40), (3, 40, 4000), (4, 40, 40), (16, 512, 2048), (300, 300, 264), (2048, 2048, 512), (3000, 2304, 640), (70000, 16, 24)):
        for odd in (0, 1):
            for call in calls:
                call(made(dt, M, F, K, odd), None)
                assert used() == start, (dt, M, F, K, odd)
    assert used() == start
ops.check_status()
print("done")
""")


def test_two_threads_at_once():
    """The same calls from two threads on streams of their own, over and over."""
    assert "done" in _run(SETUP + """
import concurrent.futures as cf
t = made(M=700, F=520, K=392)
want = [[u.clone() for u in flat(c(t, None))] for c in calls]
torch.cuda.synchronize()
def work(_):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.default_stream())
    for i in range(20):
        for call, expected in zip(calls, want):
            got = flat(call(t, s))
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, expected))
    return "fine"
with cf.ThreadPoolExecutor(2) as pool:
    assert list(pool.map(work, range(2), timeout=200)) == ["fine", "fine"]
ops.check_status()
print("done")
""", timeout=300)


# --- tiles whose results leave by copies of their own -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, torch.float16])
@pytest.mark.parametrize("M, N, K", [(2304, 2304, 640), (3000, 1400, 1100), (2100, 2312, 72), (4097, 1288, 2000)])
def test_wide_tiles(M, N, K, dtype):
    x, w = _pair(M, N, K)
    b, r = _randn(N, seed=3, dtype=dtype), _randn(M, N, seed=4, dtype=dtype)
    for act in ("none", "gelu"):
        for bias, residual in ((None, None), (b, None), (None, r), (b, r)):
            y = _check8(x, w, bias, act, residual, dtype, preact=False)
    # between other rows, which stay as they are, over the residual, and at addresses that allow no copies
    big = _randn(M + 2, N + 16, seed=5, dtype=dtype)
    before, inside = big.clone(), big[1:1 + M, 8:8 + N]
    assert ops.linear8(x, w, b, activation="gelu", residual=r, dtype=dtype, out=inside) is inside and torch.equal(inside, y)
    mark = torch.ones_like(big, dtype=torch.bool)
    mark[1:1 + M, 8:8 + N] = False
    assert torch.equal(big[mark], before[mark])
    over = r.clone()
    assert torch.equal(ops.linear8(x, w, b, activation="gelu", residual=over, dtype=dtype, out=over), y)
    odd = _randn(M, N + 3, seed=6, dtype=dtype)[:, 1:1 + N]
    assert torch.equal(ops.linear8(x, w, b, activation="gelu", residual=r, dtype=dtype, out=odd), y)
    ops.check_status()


@pytest.mark.parametrize("residual", [False, True])
def test_bounded_wait_of_wide_tiles(residual):
    x, w = _pair(3000, 2304, 2048)
    r = _randn(3000, 2304, seed=4, dtype=BF) if residual else None
    before = ops.linear8(x, w, residual=r)
    ops.check_status()
    ops.linear8(x, w, residual=r, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    assert torch.equal(ops.linear8(x, w, residual=r), before)
    ops.check_status()


# --- three to 32 rows -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, torch.float16])
@pytest.mark.parametrize("N, K", [(1, 1), (15, 16), (17, 129), (40, 1000), (257, 4096), (33, 900), (130, 385), (20_000, 136), (9_700, 1100)])
def test_some_rows(N, K, dtype):
    """Rows of codes that end within a block and within 16 codes, with NaN behind them, more columns than the SMs hold at once, and
    neighbours of the result that stay as they are."""
    for M in (3, 4, 8, 9, 16, 17, 32):
        x, w = _pair(M, N, K)

        def among(p, rows):
            pitch = -(-K // 16) * 16 + 32
            codes = torch.full((p.codes.shape[0] + 2 * rows, pitch), 0x7f, dtype=torch.uint8, device="cuda")
            codes[rows:rows + p.codes.shape[0], 16:16 + K] = p.codes.view(torch.uint8)
            scales = torch.full((p.scales.shape[0] + 2, p.scales.shape[1] + 3), math.nan, device="cuda")
            scales[1:-1, 1:-2] = p.scales
            return ops.Packed8(codes.view(torch.float8_e4m3fn)[rows:rows + p.codes.shape[0], 16:16 + K], scales[1:-1, 1:-2])
        b, r = _randn(N, seed=3, dtype=dtype), _randn(M, N, seed=4, dtype=dtype)
        y = _check8(x, w, b, "silu", r, dtype)
        x, w = among(x, 2), among(w, 1)
        assert torch.equal(ops.linear8(x, w, b, activation="silu", residual=r, dtype=dtype), y)
        big = _randn(M + 2, N + 5, seed=5, dtype=dtype)
        before, inside = big.clone(), big[1:1 + M, 3:3 + N]
        inside.copy_(r)
        assert torch.equal(ops.linear8(x, w, b, activation="silu", residual=inside, dtype=dtype, out=inside), y)
        mark = torch.ones_like(big, dtype=torch.bool)
        mark[1:1 + M, 3:3 + N] = False
        assert torch.equal(big[mark], before[mark])
    ops.check_status()


@pytest.mark.parametrize("dtype", [BF, torch.float16])
@pytest.mark.parametrize("F, K", [(1, 8), (15, 16), (33, 130), (40, 1000), (130, 4096), (7, 900), (10_000, 72), (4_900, 1100), (4100, 4104)])
def test_some_rows_of_a_block(F, K, dtype):
    """The same of gates and ups: rows of numbers that end within a block and within eight of them, with NaN behind them."""
    for M in (3, 4, 5, 8, 9, 16, 17, 32):
        x, w, b = _randn(M, K, seed=1, dtype=dtype), _randn(2 * F, K, seed=2, dtype=dtype, scale=K ** -0.5), _randn(2 * F, seed=3, dtype=dtype)

        def among(p):
            big = torch.full((p.shape[0] + 4, -(-K // 8) * 8 + 16), math.nan, dtype=dtype, device="cuda")
            big[2:-2, 8:8 + K] = p
            return big[2:-2, 8:8 + K]
        x, w = among(x), among(w)
        big = _randn(M + 2, F + 5, seed=5, dtype=dtype)
        before, inside = big.clone(), big[1:1 + M, 3:3 + F]
        h, z = _check_gated(x, w, b, "silu", out=inside)
        assert torch.equal(h, inside)
        mark = torch.ones_like(big, dtype=torch.bool)
        mark[1:1 + M, 3:3 + F] = False
        assert torch.equal(big[mark], before[mark])
        h8, z8 = ops.gated(x, w, b, preact="packed")
        want = ops.pack8(z)
        assert torch.equal(h8, h) and torch.equal(z8.scales, want.scales) and torch.equal(z8.codes.view(torch.uint8), want.codes.view(torch.uint8))
    ops.check_status()


# --- refusals of the binding -----------------------------------------------------------------------------------------------

def test_binding_refuses():
    bf = lambda *s: torch.zeros(*s, device="cuda", dtype=BF)
    f32 = torch.zeros(4, 200, device="cuda")
    x, w = ops.pack8(f32), ops.pack8(torch.zeros(300, 200, device="cuda"), tiles=True)
    rows = ops.pack8(torch.zeros(300, 200, device="cuda"))
    wrong = ops.Packed8(x.codes, x.scales[:, :1])
    with pytest.raises(ValueError, match="scales must have shape"):
        ops.unpack8(wrong)
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        ops.unpack8(ops.Packed8(x.codes.view(torch.uint8), x.scales))
    with pytest.raises(ValueError, match="float32"):
        ops.unpack8(ops.Packed8(x.codes, x.scales.double()))
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        ops.pack8(torch.zeros(4, 8, device="cuda", dtype=torch.float64))
    with pytest.raises(ValueError, match="no columns"):
        ops.pack8(torch.zeros(4, 0, device="cuda"))
    with pytest.raises(ValueError, match="two dimensions"):
        ops.pack8(torch.zeros(4, device="cuda"))
    with pytest.raises(ValueError, match="unit stride"):
        ops.pack8(torch.zeros(8, 4, device="cuda").t())
    with pytest.raises(ValueError, match="not those of tiles"):
        ops.pack8(torch.zeros(300, 200, device="cuda"), tiles=True, out=rows)
    with pytest.raises(ValueError, match="scale for each row"):
        ops.linear8(w, w)
    with pytest.raises(ValueError, match="scale for each tile"):
        ops.linear8(x, rows)
    with pytest.raises(ValueError, match="outputs, 200"):
        ops.linear8(x, ops.pack8(torch.zeros(300, 199, device="cuda"), tiles=True))
    with pytest.raises(ValueError, match="dtype must be"):
        ops.linear8(x, w, dtype=torch.float32)
    with pytest.raises(ValueError, match="activation"):
        ops.linear8(x, w, activation="tanh")
    with pytest.raises(ValueError, match="gates"):
        ops.gated(bf(4, 200), bf(301, 200))
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        ops.gated(f32, torch.zeros(300, 200, device="cuda"))
    with pytest.raises(ValueError, match="preact"):
        ops.gated(bf(4, 200), bf(300, 200), preact="8bit")
    with pytest.raises(laq.LaqError, match="65536"):
        ops.gated(bf(4, 65544), bf(4, 65544))
    with pytest.raises(ValueError, match="z must have shape"):
        ops.gated_backward(bf(4, 150), bf(4, 200), bf(300, 200), bf(4, 150))
    with pytest.raises(ValueError, match="dy must be"):
        ops.linear_backward(torch.zeros(4, 300, device="cuda"), x, w)
    with pytest.raises(ValueError, match="must be torch.float16|must be torch.bfloat16"):
        ops.gated_backward(bf(4, 150), bf(4, 200), bf(300, 200), torch.zeros(4, 300, device="cuda", dtype=torch.float16))
    with pytest.raises(laq.LaqError, match="overlap"):
        ops.gated(bf(0, 8), bf(8, 8))                            # no rows: nothing is looked at
        a = bf(8, 8)
        ops.gated(a, bf(16, 8), out=a)
    with pytest.raises(laq.LaqError, match="workspace"):
        ops.gated(bf(300, 201), bf(300, 201), workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    host = torch.zeros(4, 200).to(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="CUDA tensor"):
        ops.unpack8(ops.Packed8(host, x.scales))
    with pytest.raises(ValueError, match="CUDA tensor"):
        ops.unpack8(ops.Packed8(x.codes, x.scales.cpu()))


# --- offsets that pass 32 bits ------------------------------------------------------------------------------------------

def _far(M, K, seed):
    """[M, K] of zeros but for the last rows."""
    x = torch.zeros(M, K, device="cuda", dtype=BF)
    x[-5:] = _randn(5, K, seed=seed, dtype=BF)
    return x


def test_packed_matrices_of_more_than_32_bits():
    x = _far(70_000, 32_768, 1)                                  # 2.3e9 numbers
    for tiles in (False, True):
        p = ops.pack8(x, tiles=tiles)
        small = ops.pack8(x[-5:])
        back = ops.unpack8(p)
        if not tiles:
            assert torch.equal(p.codes[-5:].view(torch.uint8), small.codes.view(torch.uint8)) and torch.equal(p.scales[-5:], small.scales)
            assert torch.equal(back[-5:], ops.unpack8(small))
        else:
            assert float((back[-5:].float() - x[-5:].float()).abs().max()) <= 2.0 ** -4 * float(x.abs().max())
        assert not bool(back[:-5].any())
        del p, back


def test_products_of_more_than_32_bits():
    M, N, K = 140_000, 16_384, 128                               # 2.3e9 results
    x = _far(M, K, 1)
    w = ops.pack8(_randn(N, K, seed=2, dtype=torch.float32), tiles=True)
    p = ops.pack8(x)
    y = ops.linear8(p, w)
    want = ops.linear8(ops.Packed8(p.codes[-64:], p.scales[-64:]), w)
    assert torch.equal(y[-64:], want) and not bool(y[:-5].any())
    del y, p
    F = 8_192
    wg = _randn(2 * F, 64, seed=3, dtype=BF)
    x = _far(M, 64, 4)
    h, z = ops.gated(x, wg, preact=True)
    hs, zs = ops.gated(x[-64:], wg, preact=True)
    assert torch.equal(z[-64:], zs) and torch.equal(h[-64:], hs) and not bool(z[:-5].any())
    h8, z8 = ops.gated(x, wg, preact="packed")
    assert torch.equal(h8, h) and torch.equal(ops.unpack8(ops.Packed8(z8.codes[-64:], z8.scales[-64:])), ops.unpack8(ops.pack8(zs)))
    dh = _far(M, F, 5)
    for kept in (z, z8):
        d = ops.gated_backward(dh, x, wg, kept)                  # sums over 140000 rows, 135000 of them of zeros
        part = z[-64:] if kept is z else ops.Packed8(z8.codes[-64:], z8.scales[-64:])
        few = ops.gated_backward(dh[-64:], x[-64:], wg, part)
        assert not bool(d["dx"][:-5].any())
        # The two calls cut their sums differently (64 rows are split over a cluster): each is off by A of its 16-bit dz's sum and by one
        # rounding, 2^-8, so that they differ by twice that at most.
        g, u = (zs if kept is z else values(part)).double().chunk(2, dim=1)
        dz = torch.cat([dh[-64:].double() * u * _slope(g, "silu"), dh[-64:].double() * _act(g, "silu")], dim=1)
        for name, a, b, n in (("dx", dz, wg.double(), 2 * F), ("dw", dz.T, x[-64:].double(), M)):
            bound = 1.01 * _product_bound(a, b, n)
            got = d[name][-64:] if name == "dx" else d[name]
            _within(got, few[name].double(), 2 * bound + 2.02 * 2.0 ** -8 * (few[name].double().abs() + bound), name)
        assert torch.allclose(d["db"], few["db"], rtol=1e-5, atol=1e-5)
    ops.check_status()
