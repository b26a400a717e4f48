"""Pointers that a C call cannot use are refused by name before anything is launched; the same call with device memory runs."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_1909_07588_b200 import laq, ops
from tests.test_ops_buffers import K, LINEAR, ROWS, T, V, linear_call, pointers, row_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    return laq.load_library()


def _places(names):
    """Zeroed device memory for every name, and host memory."""
    return ({n: torch.zeros(1 << 14, dtype=torch.uint8, device="cuda") for n in names}, np.zeros(1 << 14, dtype=np.uint8))


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("name", sorted(ROWS))
def test_row_calls_refuse_host_memory(lib, name, dtype):
    dev, host = _places(pointers(name))
    pinned = torch.zeros(1 << 14, dtype=torch.uint8).pin_memory()
    assert row_call(lib, name, lambda n: dev[n].data_ptr(), dtype) == (laq.LAQ_OK, "")
    for bad in pointers(name):
        for wrong in (host.ctypes.data, pinned.data_ptr(), 1 << 12):
            rc, text = row_call(lib, name, lambda n: wrong if n == bad else dev[n].data_ptr(), dtype)
            assert rc == laq.LAQ_EINVAL and text.startswith(bad) and "device memory" in text, (bad, text)
    torch.cuda.synchronize()


@pytest.mark.parametrize("M", [2, 32])
@pytest.mark.parametrize("backward", [0, 1])
def test_linear_refuses_host_memory(lib, backward, M):
    dev, host = _places(LINEAR[backward])
    ws = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    assert linear_call(lib, backward, lambda n: dev[n].data_ptr(), ws.data_ptr(), M) == (laq.LAQ_OK, "")
    for bad in LINEAR[backward]:
        rc, text = linear_call(lib, backward, lambda n: host.ctypes.data // 16 * 16 if n == bad else dev[n].data_ptr(), ws.data_ptr(), M)
        assert rc == laq.LAQ_EINVAL and text.startswith(bad) and "device memory" in text, (bad, text)
    if backward:
        rc, text = linear_call(lib, 1, lambda n: dev[n].data_ptr(), (host.ctypes.data + 255) // 256 * 256, M)
        assert rc == laq.LAQ_EINVAL and "workspace" in text
    torch.cuda.synchronize()


def test_gradient_of_no_rows_refuses_host_memory(lib):
    host = np.zeros(1 << 14, dtype=np.uint8)
    c = laq.laq_linear_call()
    c.dtype, c.M, c.N, c.K, c.dw_dtype, c.ld_dw = 1, 0, 8, 8, 1, 8
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.status, c.dw = status.data_ptr(), host.ctypes.data
    err = C.create_string_buffer(256)
    assert lib.laq_linear_backward(C.byref(c), None, 0, None, err, 256) == laq.LAQ_EINVAL and b"dw is not device memory" in err.value


def test_memory_of_a_private_pool_is_taken(lib):
    """Memory of a private pool of the framework's allocator, too."""
    x = torch.randn(4, 100, device="cuda")
    pool = torch.cuda.MemPool()
    with torch.cuda.use_mem_pool(pool):
        y = x.clone()
    assert torch.equal(ops.token_logprobs(x)["lse"], ops.token_logprobs(y)["lse"])


def test_linear_over_its_own_input_is_refused():
    x, w = torch.randn(40, 64, device="cuda").bfloat16(), torch.randn(64, 64, device="cuda").bfloat16()
    b = torch.randn(64, device="cuda").bfloat16()
    before, want = x.clone(), ops.linear(x, w, b, residual=x)
    for call in (lambda: ops.linear(x, w, out=x), lambda: ops.linear(x, w, b, residual=x, out=x), lambda: ops.linear(x[:39], w, out=x[1:]),
                 lambda: ops.linear(x, w, out=w[:40]), lambda: ops.linear(x[:1], w, bias=b, out=b[None])):
        with pytest.raises(laq.LaqError, match="overlap") as e:
            call()
        assert e.value.status == laq.LAQ_EINVAL
    assert torch.equal(x, before)
    # rows that lie between the input's rows are not its own
    wide = torch.cat([x, torch.zeros_like(x)], dim=1)
    y = ops.linear(wide[:, :64], w, b, residual=wide[:, :64], out=wide[:, 64:])
    assert torch.equal(y, want) and torch.equal(wide[:, :64], x)
    ops.check_status()


@pytest.mark.parametrize("V", [100, 3000, 40001])
def test_row_gradients_into_the_other_half_of_a_wide_buffer(V):
    """Columns beside the logits' in the same rows, and the rows between them, are separate places."""
    rows = 9
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(rows, V, generator=g, device="cuda").bfloat16()
    tokens = torch.randint(0, V, (rows,), generator=g, device="cuda").int()
    one = torch.ones(rows, device="cuda")
    tok, val = tokens[:, None].contiguous(), torch.zeros(rows, 1, device="cuda")
    st = ops.token_logprobs(x, tokens)
    want = [ops.token_logprobs_backward(x, tokens, st["lse"], st["entropy"], one, one), ops.distill(x, tok, val, d_loss=one)["dlogits"],
            ops.distill_backward(x, tok, val, st["lse"], one)]
    calls = [lambda s, o: ops.token_logprobs_backward(s, tokens, st["lse"], st["entropy"], one, one, out=o),
             lambda s, o: ops.distill(s, tok, val, d_loss=one, out=o)["dlogits"],
             lambda s, o: ops.distill_backward(s, tok, val, st["lse"], one, out=o)]
    for call, w in zip(calls, want):
        for columns in (True, False):
            wide = torch.zeros(rows, 2 * V, dtype=x.dtype, device="cuda") if columns else torch.zeros(2 * rows, V, dtype=x.dtype, device="cuda")
            src, dst = (wide[:, :V], wide[:, V:]) if columns else (wide[::2], wide[1::2])
            src.copy_(x)
            got = call(src, dst)
            # rows that start elsewhere within 16 bytes take their elements in another order: a step of the type at most
            assert float((got.float() - w.float()).abs().max()) <= 2.0 ** -7 * float(w.float().abs().max())
            assert torch.equal(src, x)
