"""Argument checks of the operators that need no GPU: the C calls refuse before they touch the device, the binding before
it allocates."""
import ctypes as C

import pytest
import torch

from paper_1909_07588_b200 import build, laq, ops


@pytest.fixture(scope="module")
def lib():
    build.build()
    return laq.load_library()


def _logprobs(lib, dtype=1, rows=4, vocab=100, stride=100, temperature=1.0, logits=4096, tokens=4096, top_k=0, out=4096, top=4096):
    err = C.create_string_buffer(256)
    rc = lib.laq_token_logprobs(logits, dtype, rows, vocab, stride, temperature, tokens, top_k, out, out, out, top, top, None, err, 256)
    return rc, err.value.decode()


@pytest.mark.parametrize("bad, text", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 28), "rows"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 31) - 1, stride=1 << 31), "vocab"), (dict(stride=99), "stride"),
    (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
    (dict(temperature=float("inf")), "temperature"), (dict(logits=None), "null"), (dict(logits=4097), "aligned"),
])
def test_token_logprobs_refuses(lib, bad, text):
    rc, message = _logprobs(lib, **bad)
    assert rc == laq.LAQ_EINVAL and text in message


def test_no_rows_launch_nothing_and_need_no_device(lib):
    assert _logprobs(lib, rows=0, logits=None)[0] == laq.LAQ_OK
    err = C.create_string_buffer(256)
    assert lib.laq_distill(None, 0, 0, 10, 10, 1.0, None, None, 4, 4, None, None, None, None, 0, None, err, 256) == laq.LAQ_OK
    assert lib.laq_distill_backward(None, 0, 0, 10, 10, 1.0, None, None, 4, 4, None, None, None, 0, None, err, 256) == laq.LAQ_OK
    assert lib.laq_token_logprobs_backward(None, 0, 0, 10, 10, 1.0, None, None, None, None, None, None, 0, None, err, 256) == laq.LAQ_OK


def test_error_buffer_is_optional(lib):
    assert lib.laq_token_logprobs(None, 9, 1, 1, 1, 1.0, None, 0, None, None, None, None, None, None, None, 0) == laq.LAQ_EINVAL


def _call(**kw):
    c = laq.laq_linear_call()
    c.dtype, c.activation, c.M, c.N, c.K = 1, 0, 64, 32, 48
    c.x = c.w = c.y = c.dy = c.z = 4096
    c.ld_x = c.ld_w = 48
    c.ld_y = c.ld_dy = c.ld_z = 32
    c.status = 4096
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("bad, text", [
    (dict(dtype=0), "dtype"), (dict(M=-1), "M must"), (dict(N=0), "M must"), (dict(K=0), "M must"), (dict(K=1 << 31), "M must"),
    (dict(activation=4), "activation"), (dict(activation=-1), "activation"), (dict(status=None), "status"),
    (dict(flags=2), "flags"),
])
def test_linear_refuses(lib, bad, text):
    err = C.create_string_buffer(256)
    for f in (lib.laq_linear_forward, lib.laq_linear_backward):
        assert f(C.byref(_call(**bad)), None, 0, None, err, 256) == laq.LAQ_EINVAL
        assert text in err.value.decode()
        assert f(None, None, 0, None, err, 256) == laq.LAQ_EINVAL


def test_linear_workspace(lib):
    size = lambda back=0, **kw: lib.laq_linear_workspace_bytes(C.byref(_call(**kw)), back)
    assert size() == 0                                        # 16-byte rows: used as they are
    assert size(x=4098) == 64 * 48 * 2                        # an odd address: a copy of x
    assert size(K=47, ld_x=47, ld_w=47) == 64 * 48 * 2 + 32 * 48 * 2
    assert size(N=0) == 0
    assert size(1, dx=4096, ld_dx=48) == 0                    # no activation: dY serves as dZ
    assert size(1, dx=4096, ld_dx=48, activation=1) == 64 * 32 * 2
    assert size(1, db=4096) == 2 * 32 * 4                     # partial sums of two runs of 32 rows
    err = C.create_string_buffer(256)
    c = _call(x=4098)
    assert lib.laq_linear_forward(C.byref(c), None, 0, None, err, 256) == laq.LAQ_EWORKSPACE
    assert lib.laq_linear_forward(C.byref(c), 4096 + 8, 1 << 20, None, err, 256) == laq.LAQ_EWORKSPACE
    assert lib.laq_linear_forward(C.byref(c), 4096, 100, None, err, 256) == laq.LAQ_EWORKSPACE


def test_struct_layout_matches_header(tmp_path):
    """The header's laq_linear_call, compiled as plain C, against the ctypes mirror."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f[0] for f in laq.laq_linear_call._fields_]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "laq.h"', "int main(void){",
             'printf("size %zu\\n", sizeof(laq_linear_call));']
    lines += ['printf("%s %%zu\\n", offsetof(laq_linear_call, %s));' % (n, n) for n in names] + ["return 0;}"]
    (tmp_path / "l.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = dict(l.split() for l in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(out["size"]) == C.sizeof(laq.laq_linear_call)
    for n in names:
        assert int(out[n]) == getattr(laq.laq_linear_call, n).offset, n


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        ops.token_logprobs(x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA tensor"):
        ops.distill(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="CUDA tensor"):
        ops.linear(x.bfloat16(), x.bfloat16())
