"""Every pointer of an operator's C call is looked at before the call touches the device: here (no GPU needed) that a
misaligned one is refused by its name, whichever it is.  tests/test_gpu_ops_buffers.py does the same with host memory."""
import ctypes as C

import pytest

from paper_1909_07588_b200 import build, laq


@pytest.fixture(scope="module")
def lib():
    build.build()
    return laq.load_library()


T, V, K = 4, 16, 3
A = 1 << 20         # addresses that lie far apart: nothing is ever read from them here
ROWS = {
    "laq_token_logprobs": dict(
        order=["logits", 0, T, V, V, 1.0, "tokens", 2, "logprob", "entropy", "lse", "top_tokens", "top_logprobs"]),
    "laq_token_logprobs_backward": dict(
        order=["logits", 0, T, V, V, 1.0, "tokens", "lse", "entropy", "grad_logprob", "grad_entropy", "grad_logits", V]),
    "laq_distill": dict(
        order=["logits", 0, T, V, V, 1.0, "teacher_tokens", "teacher_logits", K, K, "loss", "lse", "grad_loss", "grad_logits", V]),
    "laq_distill_backward": dict(
        order=["logits", 0, T, V, V, 1.0, "teacher_tokens", "teacher_logits", K, K, "lse", "grad_loss", "grad_logits", V]),
}


def row_call(lib, name, place, dtype=0):
    """(status, text) of the call with the pointers that `place` gives for the names of its arguments."""
    args = [place(a) if isinstance(a, str) else a for a in ROWS[name]["order"]]
    args[1] = dtype
    err = C.create_string_buffer(256)
    rc = getattr(lib, name)(*args, None, err, 256)
    return rc, err.value.decode()


def pointers(name):
    return [a for a in ROWS[name]["order"] if isinstance(a, str)]


LINEAR = {
    0: ["x", "w", "bias", "residual", "y", "z", "status"],
    1: ["dy", "z", "x", "w", "dx", "dw", "db", "status"],
}
COLS = dict(x=64, w=64, dx=64, dw=64)       # the others have rows of 48


def linear_call(lib, backward, place, workspace=None, M=32):
    c = laq.laq_linear_call()
    c.dtype, c.activation, c.M, c.N, c.K, c.dw_dtype = 1, 1, M, 48, 64, 0
    for name in LINEAR[backward]:
        setattr(c, name, place(name))
        if hasattr(c, "ld_" + name):
            setattr(c, "ld_" + name, COLS.get(name, 48))
    need = lib.laq_linear_workspace_bytes(C.byref(c), backward)
    err = C.create_string_buffer(256)
    f = lib.laq_linear_backward if backward else lib.laq_linear_forward
    rc = f(C.byref(c), (workspace if need else None), need, None, err, 256)
    return rc, err.value.decode()


@pytest.mark.parametrize("name", sorted(ROWS))
def test_row_calls_name_the_misaligned_buffer(lib, name):
    at = {n: A * (i + 1) for i, n in enumerate(pointers(name))}
    for bad in pointers(name):
        rc, text = row_call(lib, name, lambda n: at[n] + (2 if n == bad else 0))
        assert rc == laq.LAQ_EINVAL and "aligned" in text and bad in text


@pytest.mark.parametrize("backward", [0, 1])
def test_linear_names_the_misaligned_buffer(lib, backward):
    at = {n: A * (i + 1) for i, n in enumerate(LINEAR[backward])}
    for bad in LINEAR[backward]:
        rc, text = linear_call(lib, backward, lambda n: at[n] + (1 if n == bad else 0), workspace=64 * A)
        assert rc == laq.LAQ_EINVAL and "aligned" in text and bad in text


def test_buffers_that_a_call_does_not_use_do_not_matter(lib):
    """Alternatives' places without alternatives; what only the other product of a gradient reads."""
    err = C.create_string_buffer(256)
    rc = lib.laq_token_logprobs(A, 0, T, V, V, 1.0, None, 0, None, 2 * A, 3 * A, 5, 7, None, err, 256)
    assert "aligned" not in err.value.decode()
    at = {n: A * (i + 1) for i, n in enumerate(LINEAR[1])}
    for gone, unused in (("dw", "x"), ("dx", "w")):
        _, text = linear_call(lib, 1, lambda n: None if n == gone else 5 if n == unused else at[n], workspace=64 * A)
        assert "aligned" not in text


def test_without_a_device_every_call_says_so(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    for name in ROWS:
        rc, text = row_call(lib, name, lambda n: A * (pointers(name).index(n) + 1))
        assert rc == laq.LAQ_EINVAL and "no current CUDA device" in text
    for backward in (0, 1):
        rc, text = linear_call(lib, backward, lambda n: A * (LINEAR[backward].index(n) + 1), workspace=64 * A)
        assert rc == laq.LAQ_EINVAL and "no current CUDA device" in text


def _bytes(p, rows, cols, ld, size):
    return {p + (r * ld + c) * size + b for r in range(rows) for c in range(cols) for b in range(size)}


def test_linear_refuses_outputs_that_share_memory(lib):
    """Exactly those: y against x over many geometries, byte sets deciding (w and the status lie elsewhere)."""
    import random
    rng = random.Random(3)
    err = C.create_string_buffer(256)
    seen = [0, 0]
    for _ in range(4000):
        M, N, K = rng.randint(1, 5), rng.randint(1, 6), rng.randint(1, 6)
        c = laq.laq_linear_call()
        c.dtype, c.M, c.N, c.K = 1, M, N, K
        c.ld_x = K + rng.randint(0, 9)
        c.ld_y = rng.choice([c.ld_x, N + rng.randint(0, 9)])
        c.ld_y = max(c.ld_y, N)
        c.x = A
        c.y = A + 2 * rng.randint(-40, 40)
        c.w, c.ld_w, c.status = 4 * A, K, 8 * A
        shared = bool(_bytes(c.x, M, K, c.ld_x, 2) & _bytes(c.y, M, N, c.ld_y, 2))
        need = lib.laq_linear_workspace_bytes(C.byref(c), 0)
        rc = lib.laq_linear_forward(C.byref(c), 16 * A if need else None, need, None, err, 256)
        assert rc == laq.LAQ_EINVAL and ("y and x overlap" if shared else "device") in err.value.decode()
        seen[shared] += 1
    assert min(seen) > 500


@pytest.mark.parametrize("backward", [0, 1])
def test_linear_refuses_every_pair_with_an_output(lib, backward):
    at = {n: A * (i + 1) for i, n in enumerate(LINEAR[backward])}
    outputs = ["dx", "dw", "db", "status"] if backward else ["y", "z", "status"]
    for o in outputs:
        for other in LINEAR[backward]:
            if other == o:
                continue
            rc, text = linear_call(lib, backward, lambda n: at[other] if n == o else at[n], workspace=64 * A)
            if (o, other) == ("y", "residual"):
                assert "device" in text                 # the residual may be y itself
            else:
                assert rc == laq.LAQ_EINVAL and "overlap" in text and o in text and other in text
    if backward:
        rc, text = linear_call(lib, 1, lambda n: at[n], workspace=at["x"])
        assert "workspace" in text and "overlap" in text
        return
    # y over a residual that is x as well would race with the product
    rc, text = linear_call(lib, 0, lambda n: at["x"] if n in ("y", "residual") else at[n], workspace=64 * A)
    assert "y and x overlap" in text or "x and y overlap" in text
    rc, text = linear_call(lib, 0, lambda n: at["residual"] + 2 if n == "y" else at[n], workspace=64 * A)
    assert "y and residual overlap" in text


def test_strides_that_reach_beyond_any_memory_are_refused(lib):
    err = C.create_string_buffer(256)
    for ld in (1 << 60, 1 << 62, (1 << 63) - 1):
        rc = lib.laq_token_logprobs(A, 0, T, V, ld, 1.0, None, 0, None, 2 * A, 3 * A, None, None, None, err, 256)
        assert rc == laq.LAQ_EINVAL and "beyond" in err.value.decode()


@pytest.mark.parametrize("name", ["laq_token_logprobs_backward", "laq_distill", "laq_distill_backward"])
def test_row_gradients_refuse_exactly_what_overlaps(lib, name):
    """The gradient's place against the logits: the logits themselves, rows between their rows (column halves of one matrix,
    every other row) and separate memory are taken, any other common byte is refused."""
    import random
    rng = random.Random(4)
    seen = [0, 0, 0]
    for _ in range(3000):
        rows, cols = rng.randint(1, 5), rng.randint(1, 6)
        ld = cols + rng.randint(0, 14)
        ld_d = rng.choice([ld, cols + rng.randint(0, 14)])
        dtype = rng.choice([0, 1])
        size = 4 if dtype == 0 else 2
        x, dx = A, A + size * rng.randint(-40, 40) * rng.randint(0, 1)
        args = list(ROWS[name]["order"])
        grad_at = args.index("grad_logits")
        args[2], args[3], args[4], args[grad_at + 1] = rows, cols, ld, ld_d
        args = [(x if a == "logits" else dx if a == "grad_logits" else A * (i + 2)) if isinstance(a, str) else a for i, a in enumerate(args)]
        args[1] = dtype
        err = C.create_string_buffer(256)
        rc = getattr(lib, name)(*args, None, err, 256)
        itself = x == dx and (rows == 1 or ld == ld_d)
        shared = bool(_bytes(x, rows, cols, ld, size) & _bytes(dx, rows, cols, ld_d, size))
        refused = shared and not itself
        assert rc == laq.LAQ_EINVAL and ("overlap" if refused else "device") in err.value.decode()
        seen[2 if itself else int(shared)] += 1
    assert min(seen) > 100


@pytest.mark.parametrize("name", sorted(ROWS))
def test_row_calls_refuse_every_pair_with_an_output(lib, name):
    at = {n: A * (i + 1) for i, n in enumerate(pointers(name))}
    outputs = {"laq_token_logprobs": ["logprob", "entropy", "lse", "top_tokens", "top_logprobs"], "laq_distill": ["loss", "lse", "grad_logits"]}
    for o in outputs.get(name, ["grad_logits"]):
        for other in pointers(name):
            if other == o:
                continue
            rc, text = row_call(lib, name, lambda n: at[other] if n == o else at[n])
            if (o, other) == ("grad_logits", "logits"):
                assert "device" in text
            else:
                assert rc == laq.LAQ_EINVAL and "overlap" in text and o in text and other in text
