"""Matrices in 8 bits against their definition in fp64, bit for bit, and the layer on them with its gradient.

Bounds (t = the layer's type, h_t = finfo(t).eps / 2 a rounding to it, u = 2^-24):
  a code is the nearest of the e4m3 numbers to x / s, a scale the least power of two: both are compared exactly;
  products of two codes are exact in fp32; the tensor core adds up a block of 128 (an ulp, 2^-23, of the sum of magnitudes for
  every 16 terms at most), and each block's sum, times the product of two powers of two, joins by one fused multiply-add (u of the
  sums so far): the product is off by at most (K / 16 + 16) 2^-23 sum |x w| =: A, as a 16-bit layer's is;
  the rest is as in a 16-bit layer (tests/test_gpu_ops_linear.py).
"""
import math

import pytest
import torch

from paper_1909_07588_b200 import laq, ops
from tests.test_gpu_ops_linear import ACTS, DTYPES, U, _act, _product_bound, _randn, _slope, _within

pytestmark = pytest.mark.gpu
ALL = dict(DTYPES, f32=torch.float32)


def reference(x, tiles):
    """(values, scales) of x [rows, cols] in fp64, from the definition; NaN where x is not finite."""
    rows, cols = x.shape
    high = 128 if tiles else 1
    down, across = -(-rows // high), -(-cols // 128)
    b = torch.zeros(down * high, across * 128, dtype=torch.float64, device=x.device)
    b[:rows, :cols] = x.double()
    b = b.view(down, high, across, 128).transpose(1, 2)
    finite = b.isfinite()
    top = torch.where(finite, b.abs(), 0.0).amax(dim=(2, 3))
    power = torch.full_like(top, -126.0)
    for k in range(-125, 122):                     # the least k with top <= 448 2^k
        power = torch.where(top > 448.0 * 2.0 ** (k - 1), float(k), power)
    scale = torch.ldexp(torch.ones_like(top).cpu(), power.cpu()).to(x.device)
    v = torch.where(finite, b, 0.0) / scale[:, :, None, None]
    _, e = torch.frexp(v)                          # |v| in [2^(e-1), 2^e)
    step = torch.ldexp(torch.ones_like(v).cpu(), (e.clamp(min=-5) - 4).cpu()).to(x.device)
    v = torch.round(v / step) * step * scale[:, :, None, None]
    v = torch.where(finite, v, math.nan)
    return v.transpose(1, 2).reshape(down * high, across * 128)[:rows, :cols], scale


def values(p):
    """What a Packed8 stands for, in fp64."""
    rows, cols = p.codes.shape
    s = p.scales.double().repeat_interleave(128, dim=1)[:, :cols]
    if p.scales.shape[0] != rows:
        s = s.repeat_interleave(128, dim=0)[:rows]
    return p.codes.double() * s


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=1e300), torch.nan_to_num(b.double(), nan=1e300))


SHAPES = [(1, 1), (1, 128), (3, 129), (128, 128), (129, 127), (64, 200), (5, 1000), (17, 2048), (300, 4097), (1000, 72), (4099, 8), (257, 640)]


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("dtype", sorted(ALL))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_pack_and_unpack(rows, cols, dtype, tiles):
    dt = ALL[dtype]
    x = _randn(rows, cols, seed=rows + cols, dtype=torch.float32)
    x *= torch.exp2(torch.randint(-12, 8, (rows, cols), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").float())
    x = x.to(dt)
    want, scale = reference(x, tiles)
    p = ops.pack8(x, tiles=tiles)
    assert p.shape == (rows, cols) and p.scales.shape == scale.shape and torch.equal(p.scales.double(), scale)
    assert torch.equal(values(p), want)
    for to in (torch.float32, torch.bfloat16):
        assert torch.equal(ops.unpack8(p, dtype=to).double(), want)            # exact
    assert torch.equal(ops.unpack8(p, dtype=torch.float16), want.to(torch.float16))
    assert ops.unpack8(p).dtype is torch.bfloat16


@pytest.mark.parametrize("dtype", sorted(ALL))
def test_values_at_the_borders(dtype):
    """Ties, the largest and least of codes, blocks of zeros, values that are no numbers, magnitudes at the type's ends."""
    dt = ALL[dtype]
    big = torch.finfo(dt).max
    blocks = [[448.0, 432.0, 1.0, 1.0625, 1.1875, -1.1875, 2.0 ** -6, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, -(2.0 ** -10), 0.0, -0.0],
              [450.0, 464.0, 1.0], [0.0, -0.0], [math.nan, 1.0, math.inf, -math.inf, 0.25], [math.inf, -math.inf], [math.nan],
              [big, -big, 1.0], [big / 2], [torch.finfo(dt).smallest_normal, torch.finfo(dt).smallest_normal / 4],
              [torch.finfo(dt).tiny * torch.finfo(dt).eps], [7.0 / 8 * 512, 7.0 / 8], [449.0], [896.0, 895.0]]
    x = torch.zeros(len(blocks), 256, dtype=dt)
    for i, b in enumerate(blocks):
        x[i, 100:100 + len(b)] = torch.tensor(b, dtype=torch.float64).to(dt)
    x = x.cuda()
    want, scale = reference(x, False)
    p = ops.pack8(x)
    assert torch.equal(p.scales.double(), scale) and same(values(p), want)
    assert bool((p.codes.view(torch.uint8)[0, 112] == 0x80).all())                # the sign of zero
    # finite values stay finite in every type, at its largest if need be
    for to in ALL.values():
        got, finite = ops.unpack8(p, dtype=to), want.isfinite()
        assert torch.equal(got.isfinite(), finite)
        limit = torch.finfo(to).max
        assert torch.equal(got[finite], want[finite].clamp(-limit, limit).to(to))


@pytest.mark.parametrize("tiles", [False, True])
def test_strides_and_odd_addresses(tiles):
    for left, pad in ((0, 0), (8, 8), (1, 2), (3, 4), (16, 0)):
        for rows, cols in ((1, 40), (70, 300), (130, 130)):
            big = _randn(rows + 2, cols + left + pad, seed=left + cols, dtype=torch.bfloat16)
            x = big[1:1 + rows, left:left + cols]
            want, scale = reference(x, tiles)
            codes = torch.full((rows + 2, cols + left + pad), 7, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            scales = torch.full((scale.shape[0] + 1, scale.shape[1] + left + 1), 7.0, device="cuda")
            out = ops.Packed8(codes[1:1 + rows, left:left + cols], scales[:scale.shape[0], left:left + scale.shape[1]])
            assert ops.pack8(x, tiles=tiles, out=out) is out
            assert torch.equal(values(out), want) and torch.equal(out.scales.double(), scale)
            beside = codes.view(torch.uint8).clone()
            beside[1:1 + rows, left:left + cols] = 7
            assert bool((beside == 7).all()) and bool((scales[scale.shape[0]:] == 7).all())
            wide = torch.full_like(big, 5.0)
            ops.unpack8(out, out=wide[1:1 + rows, left:left + cols])
            assert torch.equal(wide[1:1 + rows, left:left + cols].double(), want)
            wide[1:1 + rows, left:left + cols] = 5.0
            assert bool((wide == 5.0).all())


def test_no_rows():
    x = torch.empty(0, 300, device="cuda")
    p = ops.pack8(x)
    assert p.shape == (0, 300) and p.scales.shape == (0, 3) and ops.unpack8(p).shape == (0, 300)
    w = ops.pack8(_randn(8, 300, seed=1, dtype=torch.float32), tiles=True)
    assert ops.linear8(p, w).shape == (0, 8)
    dy = torch.empty(0, 8, device="cuda").bfloat16()
    got = ops.linear_backward(dy, p, w)
    assert got["dx"].shape == (0, 300) and not bool(got["dw"].any()) and not bool(got["db"].any())


def _check8(x, w, bias, act, residual, dtype, preact=True, **kw):
    K = x.shape[1]
    half = torch.finfo(dtype).eps / 2
    xd, wd = values(x), values(w)
    z = xd @ wd.T + (0 if bias is None else bias.double())
    y = _act(z, act) + (0 if residual is None else residual.double())
    zb = _product_bound(xd, wd.T, K) + 4 * U * (z.abs() + (0 if bias is None else bias.double().abs()))
    yb = 1.13 * zb + 16 * U * z.abs() * (1 + z.abs()) + 2 * U * y.abs()
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    got = ops.linear8(x, w, bias, activation=act, residual=residual, preact=preact, dtype=dtype, **kw)
    if preact:
        got, gz = got
        _within(gz, z, zb + half * (z.abs() + zb) + tiny, "z")
    _within(got, y, yb + half * (y.abs() + yb) + tiny, "y")
    return got


PRODUCTS = [(1, 1, 1), (1, 16, 8), (3, 5, 7), (1, 257, 129), (2, 4096, 128), (4, 100, 1000), (7, 100, 1000), (16, 200, 784), (33, 131, 72),
            (64, 64, 64), (100, 200, 784), (129, 129, 129), (130, 520, 1032), (257, 96, 200), (500, 10, 784), (512, 512, 512),
            (777, 1000, 333), (1500, 300, 40), (1024, 768, 2048), (40, 2048, 4096), (5000, 24, 16), (3000, 1400, 1100)]


def _pair(M, N, K, seed=1):
    x = _randn(M, K, seed=seed, dtype=torch.float32)
    x *= torch.exp2(torch.randint(-6, 6, (M, -(-K // 128)), generator=torch.Generator(device="cuda").manual_seed(seed + 2), device="cuda").float()
                    ).repeat_interleave(128, dim=1)[:, :K]
    w = _randn(N, K, seed=seed + 1, dtype=torch.float32, scale=K ** -0.5)
    w *= torch.exp2(torch.arange(-(-N // 128), device="cuda").float() % 5 - 2).repeat_interleave(128)[:N, None]
    return ops.pack8(x), ops.pack8(w, tiles=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", PRODUCTS)
def test_product(M, N, K, dtype):
    dt = DTYPES[dtype]
    x, w = _pair(M, N, K)
    b, r = _randn(N, seed=3, dtype=dt), _randn(M, N, seed=4, dtype=dt)
    for act in ACTS:
        _check8(x, w, b, act, r, dt)
    _check8(x, w, None, "none", None, dt, preact=False)
    ops.check_status()


@pytest.mark.parametrize("M, N, K", [(1, 40, 56), (3, 40, 300), (70, 40, 56), (300, 136, 264)])
def test_product_of_strided_codes(M, N, K):
    x, w = _pair(M, N, K)
    plain = ops.linear8(x, w)
    for left, pad in ((16, 16), (1, 2), (8, 0), (5, 11)):
        def inside(p):
            codes = torch.zeros(p.codes.shape[0] + 2, K + left + pad, dtype=torch.uint8, device="cuda")
            scales = torch.full((p.scales.shape[0], p.scales.shape[1] + left), math.nan, device="cuda")
            codes[1:-1, left:left + K] = p.codes.view(torch.uint8)
            scales[:, left:] = p.scales
            return ops.Packed8(codes.view(torch.float8_e4m3fn)[1:-1, left:left + K], scales[:, left:])
        got = ops.linear8(inside(x), inside(w))
        assert torch.equal(got, plain) or M <= 4            # few rows: sums of other lengths
        _check8(inside(x), inside(w), None, "none", None, torch.bfloat16, preact=False)
    r = _randn(M, N, seed=9, dtype=torch.bfloat16)
    want = ops.linear8(x, w, residual=r)
    assert ops.linear8(x, w, residual=r, out=r) is r and torch.equal(r, want)


def test_codes_that_are_no_numbers():
    """A NaN of X spoils its row and no other, one of W its column."""
    for M in (3, 40, 300):
        x, w = _pair(M, 70, 300)
        clean = ops.linear8(x, w)
        x.codes.view(torch.uint8)[1, 5] = 0x7f
        w.codes.view(torch.uint8)[7, 290] = 0xff
        y = ops.linear8(x, w)
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[1] = True
        bad[:, 7] = True
        assert torch.equal(y.isnan(), bad) and torch.equal(y[~bad], clean[~bad])


def test_far_scales():
    """Scales at both ends of what pack8 gives, where their product is a normal number."""
    for M in (2, 50):
        x, w = _pair(M, 96, 256)
        y = ops.linear8(x, w, dtype=torch.bfloat16)
        x2, w2 = ops.Packed8(x.codes, x.scales * 2.0 ** 110), ops.Packed8(w.codes, w.scales * 2.0 ** -110)
        assert torch.equal(ops.linear8(x2, w2), y)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M, N, K", [(1, 1, 1), (2, 3, 5), (1, 300, 120), (20, 40, 64), (100, 200, 784), (129, 129, 129), (600, 520, 136),
                                     (2048, 512, 1024), (64, 2048, 1024)])
def test_gradient_from_packed_operands(M, N, K, dtype):
    """Exactly the gradient of the restored operands: those are numbers of the layer's type."""
    dt = DTYPES[dtype]
    x, w = ops.pack8(_randn(M, K, seed=1, dtype=dt)), ops.pack8(_randn(N, K, seed=2, dtype=dt), tiles=True)
    dy, z = _randn(M, N, seed=3, dtype=dt), ops.pack8(_randn(M, N, seed=4, dtype=dt, scale=2.0))
    xr, wr, zr = (ops.unpack8(p, dtype=dt) for p in (x, w, z))
    for act in ACTS:
        need = act != "none"
        want = ops.linear_backward(dy, xr, wr, z=zr if need else None, activation=act)
        for some in ((x, wr, zr), (xr, w, zr), (xr, wr, z), (x, w, z)):
            if some[2] is z and not need:
                continue
            got = ops.linear_backward(dy, some[0], some[1], z=some[2] if need else None, activation=act)
            for k in want:
                assert torch.equal(got[k], want[k]), (act, k)
    got = ops.linear_backward(dy, x, w, z=z, activation="relu", dw_dtype=torch.float32, dx=False, db=False)
    dz = dy.double() * _slope(values(z), "relu")
    assert set(got) == {"dw"}
    _within(got["dw"], dz.T @ values(x), _product_bound(dz.T, values(x), M) + U * (dz.T @ values(x)).abs() + 1e-30, "fp32 dw")
    ops.check_status()


def test_gradient_from_tiles_and_odd_addresses():
    """z and x with a scale a tile; codes at odd addresses."""
    M, N, K = 200, 131, 260
    dt = torch.bfloat16
    dy, w = _randn(M, N, seed=3, dtype=dt), _randn(N, K, seed=2, dtype=dt)
    x, z = ops.pack8(_randn(M, K, seed=1, dtype=dt), tiles=True), ops.pack8(_randn(M, N, seed=4, dtype=dt), tiles=True)
    want = ops.linear_backward(dy, ops.unpack8(x), w, z=ops.unpack8(z), activation="silu")
    odd = lambda p: ops.Packed8(torch.nn.functional.pad(p.codes.view(torch.uint8), (3, 2)).view(torch.float8_e4m3fn)[:, 3:-2], p.scales)
    for a, b in ((x, z), (odd(x), odd(z))):
        got = ops.linear_backward(dy, a, w, z=b, activation="silu")
        for k in want:
            assert torch.equal(got[k], want[k]), k


def test_bounded_wait_of_the_product():
    x, w = _pair(300, 256, 512)
    before = ops.linear8(x, w)
    ops.check_status()
    ops.linear8(x, w, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    assert torch.equal(ops.linear8(x, w), before)
    ops.check_status()


def test_captured_and_replayed_on_another_stream():
    x, w = _pair(200, 320, 500)
    dy = _randn(200, 320, seed=8, dtype=torch.bfloat16)
    raw = _randn(200, 500, seed=9, dtype=torch.float32)
    want = ops.pack8(raw), ops.linear8(x, w), ops.linear_backward(dy, x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    side = ops.linear8(x, w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(side, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p = ops.pack8(raw)
        y = ops.linear8(x, w)
        d = ops.linear_backward(dy, x, w)
    raw.mul_(2.0)                                  # powers of two: the codes stay, the scales double
    x.scales.mul_(2.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(p.codes.view(torch.uint8), want[0].codes.view(torch.uint8)) and torch.equal(p.scales, want[0].scales * 2)
    assert torch.equal(y, want[1] * 2) and torch.equal(d["dw"], want[2]["dw"] * 2) and torch.equal(d["dx"], want[2]["dx"])


def test_scales_that_are_no_powers_of_two():
    """Another program's scales: the product of two is rounded once (u), which the bound's 16 2^-23 holds; a value is rounded to fp32
    and then to the type asked for."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for M, N, K in ((3, 70, 300), (40, 520, 1000), (700, 1300, 650), (2304, 2304, 512)):
        x, w = _pair(M, N, K)
        x.scales.mul_(torch.rand(x.scales.shape, generator=gen, device="cuda") + 0.5)
        w.scales.mul_(torch.rand(w.scales.shape, generator=gen, device="cuda") + 0.5)
        _check8(x, w, None, "silu", None, torch.bfloat16, preact=False)
        for dt in ALL.values():
            v, half = values(x), torch.finfo(dt).eps / 2
            _within(ops.unpack8(x, dtype=dt), v, (half + 2 * U) * v.abs() + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps, "values")
    x, z, w = (ops.pack8(_randn(300, n, seed=n, dtype=torch.bfloat16)) for n in (200, 136, 72))
    z.scales.mul_(torch.rand(z.scales.shape, generator=gen, device="cuda") + 0.5)
    dy, wd = _randn(300, 136, seed=5, dtype=torch.bfloat16), _randn(136, 200, seed=6, dtype=torch.bfloat16)
    dz = dy.double() * _slope(values(z), "silu")             # z is read as it is, in fp32
    db = ops.linear_backward(dy, x, wd, z=z, activation="silu")["db"]
    _within(db, dz.sum(0), (302 * U) * dz.abs().sum(0) + 40 * U * (dy.double().abs() * (1 + values(z) ** 2)).sum(0), "db")
    ops.check_status()


def test_gated_gradient_from_tiles():
    """z with a scale a tile, as pack8(z, tiles=True) makes it."""
    for F in (136, 131):
        dh, x, w = _randn(300, F, seed=1, dtype=torch.bfloat16), _randn(300, 72, seed=2, dtype=torch.bfloat16), _randn(2 * F, 72, seed=3, dtype=torch.bfloat16)
        z = ops.pack8(_randn(300, 2 * F, seed=4, dtype=torch.bfloat16), tiles=True)
        xt = ops.pack8(x, tiles=True)
        want = ops.gated_backward(dh, ops.unpack8(xt), w, ops.unpack8(z))
        got = ops.gated_backward(dh, xt, w, z)
        for k in want:
            assert torch.equal(got[k], want[k]), (F, k)
