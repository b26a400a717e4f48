"""Measured cases of the model-side operators: what a worker computes before its gradient is quantized.

Three operators stand between a worker's samples and the local gradient that the library quantizes and uploads:

``linear``    a layer's product with bias, activation and residual in its epilogue, and its gradient;
``logprobs``  log probabilities of given tokens, with the entropy and the top alternatives, and its gradient;
``distill``   the divergence from a teacher's top logits, and its gradient (alone, or in the same call as the loss).

``run`` computes a case with elementary torch operations in fp32 (``own = False``) or with this package's entry
points (``own = True``).  ``exact`` computes the same outputs from the definitions in fp64.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
LARGEST_ROWS = 1 << 29            # tokens x vocabulary of the largest case
LARGEST_LINEAR = 2 * 8192 * 4096 * 4096     # operations of the largest product (all products of a gradient together)


def listed():
    return [
        # one decoding step of one sequence: latency of a single long row, with alternatives to show
        dict(name="logprobs_decode", op="logprobs", dir="fwd", T=1, V=131072, dtype="bf16", top_k=8, temperature=1.0, masked=0.0),
        # scoring a long prompt or a batch of sampled answers: every token's log probability and 20 alternatives
        dict(name="logprobs_prompt", op="logprobs", dir="fwd", T=4096, V=131072, dtype="bf16", top_k=20, temperature=1.0, masked=0.0),
        # constrained decoding over an odd vocabulary: four of five entries masked with -inf, padded rows, fp32 logits
        dict(name="logprobs_masked", op="logprobs", dir="fwd", T=517, V=50001, dtype="f32", top_k=5, temperature=0.7, masked=0.8),
        # policy-gradient step: gradients of log probability and entropy, odd vocabulary (rows start at odd addresses)
        dict(name="logprobs_gradient", op="logprobs", dir="bwd", T=4096, V=100003, dtype="bf16", top_k=0, temperature=1.0, masked=0.0),
        # distillation step: loss and logit gradient in one call, mean over the batch known beforehand
        dict(name="distill_step", op="distill", dir="step", T=8192, V=65536, dtype="bf16", K=64, temperature=2.0, ragged=False),
        # the same on a small batch with an odd vocabulary, fp16, rows with fewer teacher entries or none
        dict(name="distill_ragged", op="distill", dir="step", T=513, V=32003, dtype="f16", K=100, temperature=1.0, ragged=True),
        # validation loss on a few rows
        dict(name="distill_eval", op="distill", dir="fwd", T=64, V=32000, dtype="f32", K=16, temperature=1.0, ragged=False),
        # gradient with row weights that are only known after the loss
        dict(name="distill_gradient", op="distill", dir="bwd", T=2048, V=131072, dtype="bf16", K=32, temperature=1.5, ragged=True),
        # one token through a layer: the weights are read once
        dict(name="linear_token", op="linear", dir="fwd", M=1, N=4096, K=4096, dtype="bf16", act="silu", residual=True, preact=False),
        # a layer over a long batch, with its residual
        dict(name="linear_batch", op="linear", dir="fwd", M=8192, N=4096, K=4096, dtype="bf16", act="gelu", residual=True, preact=False),
        # the 784-200 layer of this repository's network workload: 6000 samples of one worker, gradient in fp32
        dict(name="linear_network_gradient", op="linear", dir="bwd", M=6000, N=200, K=784, dtype="bf16", act="relu", residual=False, preact=False),
        # training a wide layer: gradients of input, weight and bias
        dict(name="linear_gradient", op="linear", dir="bwd", M=8192, N=4096, K=1024, dtype="bf16", act="gelu", residual=False, preact=False),
    ]


def _log_uniform(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["logprobs", "distill", "linear"])
    if op == "linear":
        direction = rng.choice(["fwd", "bwd"])
        M, N, K = _log_uniform(rng, 1, 16384), _log_uniform(rng, 8, 8192), _log_uniform(rng, 8, 8192)
        if rng.random() < 0.6:                     # layers are mostly multiples of 8 wide; the others come as they are
            N, K = N // 8 * 8, K // 8 * 8
        passes = 1 if direction == "fwd" else 2
        M = max(1, min(M, LARGEST_LINEAR // (2 * N * K * passes)))
        return dict(op=op, dir=direction, M=M, N=N, K=K, dtype=rng.choice(["bf16", "f16"]),
                    act=rng.choice(["none", "relu", "gelu", "silu"]), residual=rng.random() < 0.5, preact=rng.random() < 0.5)
    dtype = rng.choice(["f32", "bf16", "f16"])
    V = _log_uniform(rng, 10, 262144)
    T = _log_uniform(rng, 1, 16384)
    T = max(1, min(T, LARGEST_ROWS * 2 // SIZES[dtype] // V))
    temperature = rng.choice([1.0, 0.7, 2.0])
    if op == "logprobs":
        return dict(op=op, dir=rng.choice(["fwd", "bwd"]), T=T, V=V, dtype=dtype, top_k=rng.choice([0, 1, 5, 20, 32]),
                    temperature=temperature, masked=rng.choice([0.0, 0.0, 0.5, 0.99]))
    return dict(op=op, dir=rng.choice(["step", "fwd", "bwd"]), T=T, V=V, dtype=dtype, K=_log_uniform(rng, 1, 128),
                temperature=temperature, ragged=rng.random() < 0.5)


# --- inputs ----------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _logits(case, g):
    """Rows like a trained model's: a broad body and one peak in each row; a share of the entries masked with -inf."""
    T, V = case["T"], case["V"]
    x = torch.randn(T, V, generator=g, device="cuda") * 2.5
    rows = torch.arange(T, device="cuda")
    peak = torch.randint(0, V, (T,), generator=g, device="cuda")
    x[rows, peak] += 12.0
    if case.get("masked", 0.0) > 0.0:
        drop = torch.rand(T, V, generator=g, device="cuda") < case["masked"]
        drop[rows, peak] = False
        x.masked_fill_(drop, -math.inf)
    return x.to(DTYPES[case["dtype"]])


def prepare(case, seed):
    g = _generator(seed)
    st = dict(case=case)
    if case["op"] == "linear":
        M, N, K, t = case["M"], case["N"], case["K"], DTYPES[case["dtype"]]
        st["x"] = _randn(g, M, K, dtype=t)
        st["w"] = _randn(g, N, K, scale=1.0 / math.sqrt(K), dtype=t)
        if case["dir"] == "fwd":
            st["bias"] = _randn(g, N, scale=0.5, dtype=t)
            st["residual"] = _randn(g, M, N, dtype=t) if case["residual"] else None
        else:
            st["dy"] = _randn(g, M, N, dtype=t)
            st["z"] = _randn(g, M, N, dtype=t) if case["act"] != "none" else None
        return st
    T, V = case["T"], case["V"]
    st["logits"] = _logits(case, g)
    if case["op"] == "logprobs":
        top = st["logits"].argmax(dim=1)
        other = torch.randint(0, V, (T,), generator=g, device="cuda")
        keep = torch.rand(T, generator=g, device="cuda") < 0.5
        other = torch.where(st["logits"].gather(1, other[:, None])[:, 0] == -math.inf, top, other)
        tokens = torch.where(keep, top, other)
        if case["masked"] > 0.0 and T > 1:                     # padded positions
            tokens = torch.where(torch.rand(T, generator=g, device="cuda") < 0.1, torch.full_like(tokens, -1), tokens)
        st["tokens"] = tokens.to(torch.int32)
        if case["dir"] == "bwd":
            out = _logprobs(st["logits"], st["tokens"], 0, case["temperature"], torch.float64)
            st["lse"], st["entropy"] = out["lse"].float(), out["entropy"].float()
            st["d_logprob"] = _randn(g, T)
            st["d_entropy"] = _randn(g, T, scale=0.1)
        return st
    K = case["K"]
    st["teacher_tokens"] = torch.randint(0, V, (T, K), generator=g, device="cuda").to(torch.int32)
    st["teacher_logits"] = _randn(g, T, K, scale=2.0).sort(dim=1, descending=True).values.contiguous()
    if case["ragged"]:                                         # rows with fewer entries, some with none
        held = torch.randint(0, K + 1, (T, 1), generator=g, device="cuda")
        absent = torch.arange(K, device="cuda")[None, :] >= held
        st["teacher_tokens"].masked_fill_(absent, -1)
    st["d_loss"] = torch.full((T,), 1.0 / T, device="cuda") if case["dir"] == "step" else _randn(g, T)
    if case["dir"] == "bwd":
        st["lse"] = _distill(st, torch.float64, gradient=False)["lse"].float()
    return st


# --- plain forms -----------------------------------------------------------------------------------------------------

def _order_keys(x):
    """int64 keys that order a row by value, then by lowest index; the index comes back from the low half."""
    bits = (x.float() + 0.0).view(torch.int32).to(torch.int64)     # + 0.0: the two zeros are one value
    bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    last = x.shape[1] - 1
    return bits * (1 << 32) + (last - torch.arange(last + 1, device=x.device))


def _row_statistics(s):
    """lse and entropy of rows of scaled logits; rows of -inf alone have lse = -inf and entropy 0."""
    m = s.max(dim=1, keepdim=True).values
    shift = torch.where(m == -math.inf, torch.zeros_like(m), m)
    d = s - shift
    e = d.exp()
    total = e.sum(dim=1)
    moment = torch.where(e > 0, e * d, torch.zeros_like(e)).sum(dim=1)
    none = total == 0
    lse = shift[:, 0] + total.log()
    return lse, torch.where(none, torch.zeros_like(lse), total.log() - moment / torch.where(none, torch.ones_like(total), total))


def _logprobs(x, tokens, top_k, temperature, t):
    s = x.to(t) / temperature
    lse, entropy = _row_statistics(s)
    live = tokens >= 0
    given = s.gather(1, tokens.clamp(min=0).to(torch.int64)[:, None])[:, 0]
    logprob = torch.where(given == -math.inf, given, given - lse)
    zero = torch.zeros_like(lse)
    out = dict(logprob=torch.where(live, logprob, zero), entropy=torch.where(live, entropy, zero), lse=torch.where(live, lse, zero))
    if top_k:
        V = x.shape[1]
        n = min(top_k, V)
        best = _order_keys(x).topk(n, dim=1).values
        at = V - 1 - (best & 0xffffffff)
        value = s.gather(1, at)
        there = (value > -math.inf) & live[:, None]
        top_tokens = torch.full((x.shape[0], top_k), -1, dtype=torch.int32, device=x.device)
        top_logprobs = torch.full((x.shape[0], top_k), -math.inf, dtype=t, device=x.device)
        top_tokens[:, :n] = torch.where(there, at, torch.full_like(at, -1)).to(torch.int32)
        top_logprobs[:, :n] = torch.where(there, value - lse[:, None], torch.full_like(value, -math.inf))
        out.update(top_tokens=top_tokens, top_logprobs=top_logprobs)
    return out


def _logprobs_gradient(st, t):
    tau = st["case"]["temperature"]
    lse, entropy = st["lse"].to(t)[:, None], st["entropy"].to(t)[:, None]
    live = (st["tokens"] >= 0)[:, None]
    g, h = st["d_logprob"].to(t)[:, None], st["d_entropy"].to(t)[:, None]
    logp = st["logits"].to(t) / tau - lse
    p = logp.exp()
    d = -g * p - h * torch.where(p > 0, p * (logp + entropy), torch.zeros_like(p))
    d.scatter_add_(1, st["tokens"].clamp(min=0).to(torch.int64)[:, None], g)
    return torch.where(live, d / tau, torch.zeros_like(d))


def _distill(st, t, gradient):
    tau = st["case"]["temperature"]
    s = st["logits"].to(t) / tau
    at = st["teacher_tokens"].to(torch.int64)
    there = at >= 0
    row = there.any(dim=1)
    lse = _row_statistics(s)[0] if "lse" not in st else st["lse"].to(t)
    lse = torch.where(row, lse, torch.zeros_like(lse))
    at = at.clamp(min=0)
    tl = torch.where(there, st["teacher_logits"].to(t) / tau, torch.full((), -math.inf, dtype=t, device=s.device))
    tl = torch.where(row[:, None], tl, torch.zeros_like(tl))
    top = tl.max(dim=1, keepdim=True).values
    e = (tl - top).exp()
    total = e.sum(dim=1, keepdim=True)
    q = torch.where(row[:, None], e / total, torch.zeros_like(e))
    logq = tl - top - total.log()
    each = torch.where(q > 0, q * (logq - (s.gather(1, at) - lse[:, None])), torch.zeros_like(q))
    out = dict(loss=tau * tau * each.sum(dim=1), lse=lse)
    if gradient:
        p = (s - lse[:, None]).exp()
        p.scatter_add_(1, at, -q)
        scale = (st["d_loss"].to(t) * tau)[:, None]
        out["dlogits"] = torch.where(row[:, None], p * scale, torch.zeros_like(p))
    return out


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
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        sg = 1 / (1 + (-z).exp())
        return sg * (1 + z * (1 - sg))
    c = math.sqrt(2 / math.pi)
    sg = 1 / (1 + (-2 * c * (z + 0.044715 * z * z * z)).exp())
    return sg + z * sg * (1 - sg) * 2 * c * (1 + 3 * 0.044715 * z * z)


def _weight_gradient_dtype(case):
    """fp32 where the layer's own gradient is exact in its type (no activation, ReLU), else the layer's type."""
    return torch.float32 if case["act"] in ("none", "relu") else DTYPES[case["dtype"]]


def _linear(st, t, out_dtype, dw_dtype):
    case = st["case"]
    if case["dir"] == "fwd":
        z = st["x"].to(t) @ st["w"].to(t).T + st["bias"].to(t)
        y = _act(z, case["act"])
        if st["residual"] is not None:
            y = y + st["residual"].to(t)
        return dict(y=y.to(out_dtype), z=z.to(out_dtype)) if case["preact"] else dict(y=y.to(out_dtype))
    dz = st["dy"].to(t)
    if case["act"] != "none":
        dz = dz * _act_slope(st["z"].to(t), case["act"])
    return dict(dx=(dz @ st["w"].to(t)).to(out_dtype), dw=(dz.T @ st["x"].to(t)).to(dw_dtype),
                db=dz.sum(dim=0))


# --- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _run_own(state)
    if case["op"] == "linear":
        return _linear(state, torch.float32, DTYPES[case["dtype"]], _weight_gradient_dtype(case))
    if case["op"] == "logprobs":
        if case["dir"] == "fwd":
            return _logprobs(state["logits"], state["tokens"], case["top_k"], case["temperature"], torch.float32)
        return dict(dlogits=_logprobs_gradient(state, torch.float32).to(state["logits"].dtype))
    out = _distill(state, torch.float32, gradient=case["dir"] != "fwd")
    if case["dir"] == "fwd":
        return out
    out["dlogits"] = out["dlogits"].to(state["logits"].dtype)
    return out if case["dir"] == "step" else dict(dlogits=out["dlogits"])


def _run_own(state):
    from paper_1909_07588_b200 import ops
    case = state["case"]
    if case["op"] == "linear":
        if case["dir"] == "fwd":
            y = ops.linear(state["x"], state["w"], state["bias"], activation=case["act"], residual=state["residual"],
                           preact=case["preact"])
            return dict(y=y[0], z=y[1]) if case["preact"] else dict(y=y)
        return ops.linear_backward(state["dy"], state["x"], state["w"], z=state["z"], activation=case["act"],
                                   dw_dtype=_weight_gradient_dtype(case))
    if case["op"] == "logprobs":
        if case["dir"] == "fwd":
            return ops.token_logprobs(state["logits"], state["tokens"], top_k=case["top_k"], temperature=case["temperature"])
        return dict(dlogits=ops.token_logprobs_backward(state["logits"], state["tokens"], state["lse"], state["entropy"],
                                                        d_logprob=state["d_logprob"], d_entropy=state["d_entropy"],
                                                        temperature=case["temperature"]))
    if case["dir"] == "bwd":
        return dict(dlogits=ops.distill_backward(state["logits"], state["teacher_tokens"], state["teacher_logits"],
                                                 state["lse"], state["d_loss"], temperature=case["temperature"]))
    return ops.distill(state["logits"], state["teacher_tokens"], state["teacher_logits"], temperature=case["temperature"],
                       d_loss=state["d_loss"] if case["dir"] == "step" else None)


def work(case):
    if case["op"] == "linear":
        M, N, K, e = case["M"], case["N"], case["K"], SIZES[case["dtype"]]
        if case["dir"] == "fwd":
            extra = M * N * (1 + int(case["residual"]) + int(case["preact"]))
            return dict(bytes=e * (M * K + N * K + N + extra), flops=2 * M * N * K)
        w = 4 if case["act"] in ("none", "relu") else e
        read = e * (M * N * (1 if case["act"] == "none" else 2) + M * K + N * K)
        return dict(bytes=read + e * M * K + w * N * K + 4 * N, flops=4 * M * N * K)
    T, V, e = case["T"], case["V"], SIZES[case["dtype"]]
    if case["op"] == "logprobs":
        if case["dir"] == "fwd":
            return dict(bytes=T * (V * e + 4 + 12 + 8 * case["top_k"]), flops=6 * T * V)
        return dict(bytes=T * (2 * V * e + 4 + 16), flops=6 * T * V)
    rows = T * (8 * case["K"] + 12)
    if case["dir"] == "fwd":
        return dict(bytes=T * V * e + rows, flops=4 * T * V)
    return dict(bytes=2 * T * V * e + rows, flops=(8 if case["dir"] == "step" else 5) * T * V)


# --- the definitions in fp64 -------------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, st)
    step = max(1, (1 << 26) // case["V"])
    rows = [_exact_rows(case, st, slice(a, a + step)) for a in range(0, case["T"], step)]
    out = {k: torch.cat([p[k] for p in rows]) for k in rows[0]}
    if case["dir"] == "bwd":
        return dict(dlogits=out["dlogits"])
    return out


def _exact_rows(case, st, r):
    s = st["logits"][r].double().div(case["temperature"])
    lse = torch.logsumexp(s, dim=1)
    logp = s - lse[:, None]
    logp = torch.where(s == -math.inf, s, logp)
    p = torch.exp(logp)
    if case["op"] == "logprobs":
        y = st["tokens"][r].long()
        live = y >= 0
        y = torch.where(live, y, torch.zeros_like(y))
        if case["dir"] == "bwd":
            # the statistics are inputs of the gradient, in the 32 bits they are handed over in
            logp = s - st["lse"][r].double()[:, None]
            p = torch.exp(logp)
            g, h = st["d_logprob"][r].double(), st["d_entropy"][r].double()
            centred = torch.nan_to_num(logp, neginf=0.0) + st["entropy"][r].double()[:, None]
            d = torch.zeros_like(p)
            d[torch.arange(d.shape[0], device=d.device), y] = g
            d = d - g[:, None] * p - h[:, None] * p * centred
            return dict(dlogits=torch.where(live[:, None], d, 0.0) / case["temperature"])
        entropy = torch.special.entr(p).sum(dim=1)
        out = dict(logprob=torch.where(live, logp.gather(1, y[:, None])[:, 0], 0.0),
                   entropy=torch.where(live, entropy, 0.0), lse=torch.where(live, lse, 0.0))
        if case["top_k"]:
            k, n = case["top_k"], min(case["top_k"], case["V"])
            at = torch.argsort(st["logits"][r], dim=1, descending=True, stable=True)[:, :n]
            value = logp.gather(1, at)
            gone = (value == -math.inf) | ~live[:, None]
            tokens = torch.full((s.shape[0], k), -1, dtype=torch.int32, device=s.device)
            values = torch.full((s.shape[0], k), -math.inf, dtype=torch.float64, device=s.device)
            tokens[:, :n] = torch.where(gone, -1, at).int()
            values[:, :n] = torch.where(gone, -math.inf, value)
            out.update(top_tokens=tokens, top_logprobs=values)
        return out
    at = st["teacher_tokens"][r].long()
    there = at >= 0
    row = there.any(dim=1)
    t = torch.where(there, st["teacher_logits"][r].double().div(case["temperature"]), -math.inf)
    logq = torch.where(row[:, None], t - torch.logsumexp(t, dim=1)[:, None], -math.inf)
    q = torch.exp(logq)
    at = torch.where(there, at, torch.zeros_like(at))
    tau = case["temperature"]
    if case["dir"] == "bwd":
        lse = st["lse"][r].double()
        p = torch.exp(s - lse[:, None])
    loss = tau ** 2 * torch.where(q > 0, q * (logq - logp.gather(1, at)), 0.0).sum(dim=1)
    out = dict(loss=loss, lse=torch.where(row, lse, 0.0))
    if case["dir"] != "fwd":
        target = torch.zeros_like(p).index_put_((torch.arange(p.shape[0], device=p.device)[:, None].expand_as(at), at), q, accumulate=True)
        out["dlogits"] = torch.where(row[:, None], (p - target) * (tau * st["d_loss"][r].double())[:, None], 0.0)
    return out


def _exact_linear(case, st):
    x, w = st["x"].double(), st["w"].double()
    if case["dir"] == "fwd":
        z = torch.addmm(st["bias"].double(), x, w.T)
    else:
        z = None if st["z"] is None else st["z"].double()
    act = case["act"]
    c = math.sqrt(2.0 / math.pi)
    if case["dir"] == "fwd":
        if act == "none":
            y = z
        elif act == "relu":
            y = z.clamp(min=0.0)
        elif act == "silu":
            y = z * torch.sigmoid(z)
        else:
            y = 0.5 * z * (1.0 + torch.tanh(c * (z + 0.044715 * z ** 3)))
        if st["residual"] is not None:
            y = y + st["residual"].double()
        return dict(y=y, z=z) if case["preact"] else dict(y=y)
    dz = st["dy"].double()
    if act == "relu":
        dz = torch.where(z > 0, dz, 0.0)
    elif act == "silu":
        sg = torch.sigmoid(z)
        dz = dz * (sg + z * sg * (1.0 - sg))
    elif act == "gelu":
        th = torch.tanh(c * (z + 0.044715 * z ** 3))
        dz = dz * (0.5 * (1.0 + th) + 0.5 * z * (1.0 - th * th) * c * (1.0 + 0.134145 * z * z))
    return dict(dx=dz @ w, dw=dz.T @ x, db=dz.sum(dim=0))
