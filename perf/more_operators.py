"""Measured cases of the operators that train larger layers: the gated block, 8-bit activations, and the 8-bit product.

``gated``    both projections of a gated feed-forward block, activation and product in one call, and the block's gradient;
``packed``   activations kept in 8 bits between the forward and the backward pass: written and read back (``pack``), and a
             layer's gradient computed from them (``bwd``);
``linear8``  a layer's product on 8-bit operands with a scale for each block of 128.

8-bit values are e4m3 codes with one fp32 scale, a power of two, for 128 columns of a row (activations) or for a tile of 128
rows and 128 columns (weights).  ``run`` computes a case with elementary torch operations in fp32 (``own = False``) or with
this package's entry points (``own = True``).  ``exact`` computes the same outputs from the definitions in fp64.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128
LARGEST_OPERATIONS = 4 * 8192 * 4096 * 4096      # of one case's products together
LARGEST_VALUES = 8192 * 4096                     # of one tensor that is packed and read back


def listed():
    return [
        # one token through the block: both weights are read once
        dict(name="gated_token", op="gated", dir="fwd", M=1, F=11008, K=4096, dtype="bf16", act="silu", bias=False, preact="no"),
        # a long batch through the block, nothing kept (evaluation, or recomputed later)
        dict(name="gated_batch", op="gated", dir="fwd", M=8192, F=4096, K=4096, dtype="bf16", act="silu", bias=False, preact="no"),
        # a training step's forward pass, whose projections are kept in 8 bits for the gradient
        dict(name="gated_training", op="gated", dir="fwd", M=4096, F=5504, K=2048, dtype="bf16", act="silu", bias=False, preact="packed"),
        # odd sizes with biases, projections kept as they are
        dict(name="gated_ragged", op="gated", dir="fwd", M=517, F=1501, K=1000, dtype="f16", act="gelu", bias=True, preact="yes"),
        # the block's gradient from 16-bit activations
        dict(name="gated_gradient", op="gated", dir="bwd", M=8192, F=4096, K=2048, dtype="bf16", act="silu", x_packed=False, z_packed=False),
        # the same from 8-bit activations, odd sizes
        dict(name="gated_gradient_packed", op="gated", dir="bwd", M=3001, F=2050, K=1030, dtype="f16", act="gelu", x_packed=True, z_packed=True),
        # a layer's input written for the backward pass and read back
        dict(name="pack_batch", op="packed", dir="pack", M=8192, K=4096, dtype="bf16", tiles=False),
        # the hidden activations of a few samples of this repository's network: latency
        dict(name="pack_network", op="packed", dir="pack", M=64, K=200, dtype="f16", tiles=False),
        # a wide layer's gradient from 8-bit input and pre-activation
        dict(name="packed_gradient", op="packed", dir="bwd", M=8192, N=4096, K=1024, dtype="bf16", act="gelu", x_packed=True,
             w_packed=False, z_packed=True),
        # a layer in 8 bits over a long batch, with its residual
        dict(name="linear8_batch", op="linear8", M=8192, N=4096, K=4096, dtype="bf16", act="gelu", bias=True, residual=True, preact=False),
        # one token through it: the weight's bytes are read once
        dict(name="linear8_token", op="linear8", M=1, N=4096, K=4096, dtype="bf16", act="silu", bias=True, residual=True, preact=False),
        # a batch of odd sizes: blocks that end early, a pre-activation for training
        dict(name="linear8_ragged", op="linear8", M=300, N=1025, K=777, dtype="f16", act="silu", bias=True, residual=False, preact=True),
    ]


def _log_uniform(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["gated", "packed", "linear8"])
    dtype = rng.choice(["bf16", "f16"])
    M, N, K = _log_uniform(rng, 1, 16384), _log_uniform(rng, 8, 8192), _log_uniform(rng, 8, 8192)
    if rng.random() < 0.6:                         # layers are mostly multiples of 8 wide; the others come as they are
        N, K = N // 8 * 8, K // 8 * 8
    if op == "gated":
        if rng.random() < 0.5:
            M = max(1, min(M, LARGEST_OPERATIONS // (4 * N * K)))
            return dict(op=op, dir="fwd", M=M, F=N, K=K, dtype=dtype, act=rng.choice(["silu", "gelu", "relu", "none"]),
                        bias=rng.random() < 0.5, preact=rng.choice(["no", "yes", "packed"]))
        M = max(1, min(M, LARGEST_OPERATIONS // (8 * N * K)))
        return dict(op=op, dir="bwd", M=M, F=N, K=K, dtype=dtype, act=rng.choice(["silu", "gelu", "relu", "none"]),
                    x_packed=rng.random() < 0.5, z_packed=rng.random() < 0.5)
    if op == "linear8":
        M = max(1, min(M, LARGEST_OPERATIONS // (4 * N * K)))
        return dict(op=op, M=M, N=N, K=K, dtype=dtype, act=rng.choice(["none", "relu", "gelu", "silu"]),
                    bias=rng.random() < 0.5, residual=rng.random() < 0.5, preact=rng.random() < 0.5)
    if rng.random() < 0.5:
        M = max(1, min(M, LARGEST_VALUES // K))
        return dict(op=op, dir="pack", M=M, K=K, dtype=rng.choice(["f32", "bf16", "f16"]), tiles=rng.random() < 0.3)
    M = max(1, min(M, LARGEST_OPERATIONS // (4 * N * K)))
    return dict(op=op, dir="bwd", M=M, N=N, K=K, dtype=dtype, act=rng.choice(["none", "relu", "gelu", "silu"]),
                x_packed=rng.random() < 0.8, w_packed=rng.random() < 0.4, z_packed=rng.random() < 0.6)


# --- inputs ----------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _activations(g, rows, cols, dtype=torch.float32):
    """Values whose columns differ in size, as a layer's inputs do."""
    size = (torch.randn(cols, generator=g, device="cuda") * 0.5).exp()
    return (torch.randn(rows, cols, generator=g, device="cuda") * size).to(dtype)


def prepare(case, seed):
    g = _generator(seed)
    t = DTYPES[case["dtype"]]
    st = dict(case=case)
    if case["op"] == "gated":
        M, F, K = case["M"], case["F"], case["K"]
        st["x"] = _activations(g, M, K, t)
        st["w"] = _randn(g, 2 * F, K, scale=1.0 / math.sqrt(K), dtype=t)
        if case["dir"] == "fwd":
            st["bias"] = _randn(g, 2 * F, scale=0.5, dtype=t) if case["bias"] else None
            return st
        st["dh"] = _randn(g, M, F, dtype=t)
        st["z"] = _randn(g, M, 2 * F, dtype=t)
    elif case["op"] == "linear8":
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _activations(g, M, K)
        st["w"] = _randn(g, N, K, scale=1.0 / math.sqrt(K))
        st["bias"] = _randn(g, N, scale=0.5, dtype=t) if case["bias"] else None
        st["residual"] = _randn(g, M, N, dtype=t) if case["residual"] else None
        case = dict(case, x_packed=True, w_packed=True)
    elif case["dir"] == "pack":
        st["x"] = _activations(g, case["M"], case["K"], t)
        return st
    else:
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _activations(g, M, K, t)
        st["w"] = _randn(g, N, K, scale=1.0 / math.sqrt(K), dtype=t)
        st["dy"] = _randn(g, M, N, dtype=t)
        st["z"] = _randn(g, M, N, dtype=t) if case["act"] != "none" else None
    for name in ("x", "w", "z"):
        if case.get(name + "_packed") and st.get(name) is not None:
            st[name] = _codes(st[name].float(), name == "w")
    return st


# --- plain forms -----------------------------------------------------------------------------------------------------

def _blocks(x, tiles):
    """x [rows, cols], padded with zeros to whole blocks: [block rows, rows of a block, block columns, 128]."""
    rows, cols = x.shape
    high = BLOCK if tiles else 1
    down, across = -(-rows // high), -(-cols // BLOCK)
    whole = torch.zeros(down * high, across * BLOCK, dtype=x.dtype, device=x.device)
    whole[:rows, :cols] = x
    return whole.view(down, high, across, BLOCK)


def _codes(x, tiles):
    """(codes, scales) of fp32 values: the least power of two that brings a block's largest within 448."""
    rows, cols = x.shape
    b = _blocks(x, tiles)
    size = b.abs()
    largest = torch.where(size < math.inf, size, torch.zeros_like(size)).amax(dim=(1, 3))
    part, power = torch.frexp(largest)             # 448 = 0.875 2^9
    power = torch.where(part > 0.875, power - 8, power - 9).clamp(min=-126)
    power = torch.where(largest > 0, power, torch.full_like(power, -126))
    scales = torch.ldexp(torch.ones_like(largest), power)
    v = b / scales[:, None, :, None]
    v = torch.where(size < math.inf, v, torch.full_like(v, math.nan))
    codes = v.to(torch.float8_e4m3fn).view(b.shape[0] * b.shape[1], -1)[:rows, :cols]
    return codes.contiguous(), scales


def _values(packed, t):
    """What (codes, scales) stand for."""
    codes, scales = packed
    rows, cols = codes.shape
    b = _blocks(codes.to(t), scales.shape[0] != rows)
    v = b * scales.to(t)[:, None, :, None]
    return v.view(b.shape[0] * b.shape[1], -1)[:rows, :cols]


def _given(v, t):
    """An operand, 16-bit or packed, as numbers of type t."""
    return _values(v, t) if isinstance(v, tuple) else v.to(t)


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + (-z).exp())
    u = math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)
    return z / (1 + (-2 * u).exp())


def _act_slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        sg = 1 / (1 + (-z).exp())
        return sg * (1 + z * (1 - sg))
    c = math.sqrt(2 / math.pi)
    sg = 1 / (1 + (-2 * c * (z + 0.044715 * z * z * z)).exp())
    return sg + z * sg * (1 - sg) * 2 * c * (1 + 3 * 0.044715 * z * z)


def _layer_gradient(dz, st, t, dw_dtype):
    return dict(dx=(dz @ _given(st["w"], torch.float32)).to(t), dw=(dz.T @ _given(st["x"], torch.float32)).to(dw_dtype), db=dz.sum(dim=0))


def _weight_gradient_dtype(case):
    """fp32 where the layer's own gradient is exact in its type (no activation, ReLU), else the layer's type."""
    return torch.float32 if case["act"] in ("none", "relu") else DTYPES[case["dtype"]]


def _plain(st):
    case = st["case"]
    t, f32 = DTYPES[case["dtype"]], torch.float32
    if case["op"] == "packed" and case["dir"] == "pack":
        packed = _codes(st["x"].to(f32), case["tiles"])
        return dict(values=_values(packed, f32).to(t), scales=packed[1])
    if case["op"] == "packed":
        dz = st["dy"].to(f32)
        if case["act"] != "none":
            dz = dz * _act_slope(_given(st["z"], f32), case["act"])
        return _layer_gradient(dz, st, t, _weight_gradient_dtype(case))
    if case["op"] == "linear8":
        z = _values(st["x"], f32) @ _values(st["w"], f32).T
        if st["bias"] is not None:
            z = z + st["bias"].to(f32)
        y = _act(z, case["act"])
        if st["residual"] is not None:
            y = y + st["residual"].to(f32)
        return dict(y=y.to(t), z=z.to(t)) if case["preact"] else dict(y=y.to(t))
    F = case["F"]
    if case["dir"] == "bwd":
        z, dh = _given(st["z"], f32), st["dh"].to(f32)
        gate, up = z[:, :F], z[:, F:]
        dz = torch.cat([dh * up * _act_slope(gate, case["act"]), dh * _act(gate, case["act"])], dim=1)
        return _layer_gradient(dz, st, t, t)
    z = st["x"].to(f32) @ st["w"].to(f32).T
    if st["bias"] is not None:
        z = z + st["bias"].to(f32)
    out = dict(h=(_act(z[:, :F], case["act"]) * z[:, F:]).to(t))
    if case["preact"] == "yes":
        out["z"] = z.to(t)
    elif case["preact"] == "packed":
        out["z"] = _values(_codes(z.to(t).to(f32), False), f32).to(t)
    return out


# --- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _plain(state)


def _run_own(st):
    from paper_1909_07588_b200 import ops
    case = st["case"]
    t = DTYPES[case["dtype"]]
    packed = lambda v: ops.Packed8(*v) if isinstance(v, tuple) else v
    if case["op"] == "packed" and case["dir"] == "pack":
        p = ops.pack8(st["x"], tiles=case["tiles"])
        return dict(values=ops.unpack8(p, dtype=t), scales=p.scales)
    if case["op"] == "packed":
        return ops.linear_backward(st["dy"], packed(st["x"]), packed(st["w"]), z=packed(st["z"]), activation=case["act"],
                                   dw_dtype=_weight_gradient_dtype(case))
    if case["op"] == "linear8":
        y = ops.linear8(packed(st["x"]), packed(st["w"]), st["bias"], activation=case["act"], residual=st["residual"],
                        preact=case["preact"], dtype=t)
        return dict(y=y[0], z=y[1]) if case["preact"] else dict(y=y)
    if case["dir"] == "bwd":
        return ops.gated_backward(st["dh"], packed(st["x"]), st["w"], packed(st["z"]), activation=case["act"])
    if case["preact"] == "no":
        return dict(h=ops.gated(st["x"], st["w"], st["bias"], activation=case["act"]))
    h, z = ops.gated(st["x"], st["w"], st["bias"], activation=case["act"], preact=True if case["preact"] == "yes" else "packed")
    return dict(h=h, z=z if case["preact"] == "yes" else ops.unpack8(z, dtype=t))


def _bytes(rows, cols, size, packed, high=1):
    return rows * cols + 4 * -(-rows // high) * -(-cols // BLOCK) if packed else rows * cols * size


def work(case):
    e, M, K = SIZES[case["dtype"]], case["M"], case["K"]
    if case["op"] == "packed" and case["dir"] == "pack":
        # the input read, the packed form written and read, the values written
        return dict(bytes=2 * M * K * e + 2 * _bytes(M, K, e, True, BLOCK if case["tiles"] else 1), flops=4 * M * K)
    if case["op"] == "linear8":
        extra = M * case["N"] * (1 + int(case["residual"]) + int(case["preact"])) + case["N"] * int(case["bias"])
        return dict(bytes=_bytes(M, K, e, True) + _bytes(case["N"], K, e, True, BLOCK) + e * extra, flops=2 * M * case["N"] * K)
    if case["op"] == "packed":
        N = case["N"]
        w = 4 if case["act"] in ("none", "relu") else e
        read = e * M * N + (0 if case["act"] == "none" else _bytes(M, N, e, case["z_packed"])) + _bytes(M, K, e, case["x_packed"]) \
            + _bytes(N, K, e, case["w_packed"], BLOCK)
        return dict(bytes=read + e * M * K + w * N * K + 4 * N, flops=4 * M * N * K)
    F = case["F"]
    if case["dir"] == "bwd":
        read = e * M * F + _bytes(M, 2 * F, e, case["z_packed"]) + _bytes(M, K, e, case["x_packed"]) + e * 2 * F * K
        return dict(bytes=read + e * M * K + e * 2 * F * K + 4 * 2 * F, flops=8 * M * F * K)
    z = 0 if case["preact"] == "no" else _bytes(M, 2 * F, e, False)
    if case["preact"] == "packed":                 # written packed, read back, and the values written
        z += 2 * _bytes(M, 2 * F, e, True)
    return dict(bytes=e * (M * K + 2 * F * K + 2 * F * int(case["bias"]) + M * F) + z, flops=4 * M * F * K)


# --- the definitions in fp64 -------------------------------------------------------------------------------------------

def _exponent(v):
    """floor(log2 v) of positive normal fp64 numbers, from their bits."""
    return (v.view(torch.int64) >> 52) - 1023


def _power(k):
    """2^k in fp64."""
    return ((k + 1023) << 52).view(torch.float64)


def _exact_codes(x, tiles):
    """Values (fp64) of x rounded to 4 significant bits below its block's scale, and the scales: 448 bounds a code, 2^-9 is
    its least step."""
    rows, cols = x.shape
    high = BLOCK if tiles else 1
    down, across = (rows + high - 1) // high, (cols + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(x, (0, across * BLOCK - cols, 0, down * high - rows))
    x = x.reshape(down, high, across, BLOCK).transpose(1, 2)
    top = x.abs().flatten(2).max(dim=2).values
    below = (_exponent((top / 448.0).clamp(min=2.0 ** -200))).clamp(min=-126)      # 448 2^(below + 1) holds the largest
    scale = _power(torch.where(448.0 * _power(below) < top, below + 1, below))
    v = x / scale[:, :, None, None]
    step = _power(_exponent(v.abs().clamp(min=2.0 ** -6)) - 3)
    v = torch.round(v / step) * step * scale[:, :, None, None]
    return v.transpose(1, 2).reshape(down * high, across * BLOCK)[:rows, :cols], scale


def _exact_operand(v):
    if not isinstance(v, tuple):
        return v.double()
    codes, scales = v
    rows, cols = codes.shape
    s = scales.double().repeat_interleave(BLOCK, dim=1)[:, :cols]
    if scales.shape[0] != rows:
        s = s.repeat_interleave(BLOCK, dim=0)[:rows]
    return codes.double() * s


def _exact_act(z, act):
    """The activation and its slope."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if act == "silu":
        sg = torch.sigmoid(z)
        return z * sg, sg + z * sg * (1.0 - sg)
    c = math.sqrt(2.0 / math.pi)
    th = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * z * (1.0 - th * th) * c * (1.0 + 0.134145 * z * z)


def exact(case, seed):
    st = prepare(case, seed)
    t = DTYPES[case["dtype"]]
    if case["op"] == "packed" and case["dir"] == "pack":
        values, scales = _exact_codes(st["x"].double(), case["tiles"])
        return dict(values=values, scales=scales)
    x, w = _exact_operand(st["x"]), _exact_operand(st["w"])
    if case["op"] == "linear8":
        z = x @ w.T
        if st["bias"] is not None:
            z = z + st["bias"].double()
        y = _exact_act(z, case["act"])[0]
        if st["residual"] is not None:
            y = y + st["residual"].double()
        return dict(y=y, z=z) if case["preact"] else dict(y=y)
    if case["op"] == "packed":
        dz = st["dy"].double()
        if case["act"] != "none":
            dz = dz * _exact_act(_exact_operand(st["z"]), case["act"])[1]
        return dict(dx=dz @ w, dw=dz.T @ x, db=dz.sum(dim=0))
    if case["dir"] == "bwd":
        gate, up = _exact_operand(st["z"]).chunk(2, dim=1)
        value, slope = _exact_act(gate, case["act"])
        dh = st["dh"].double()
        dz = torch.cat([dh * up * slope, dh * value], dim=1)
        return dict(dx=dz @ w, dw=dz.T @ x, db=dz.sum(dim=0))
    z = x @ w.T
    if st["bias"] is not None:
        z = z + st["bias"].double()
    gate, up = z.chunk(2, dim=1)
    out = dict(h=_exact_act(gate, case["act"])[0] * up)
    if case["preact"] == "yes":
        out["z"] = z
    elif case["preact"] == "packed":               # 8-bit values of what is rounded to the layer's type first
        out["z"] = _exact_codes(z.to(t).double(), False)[0]
    return out
