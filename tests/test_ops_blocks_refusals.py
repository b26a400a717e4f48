"""Argument checks of the calls on 8-bit matrices and of the gated block that need no GPU: by name, before anything is launched."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_1909_07588_b200 import build, laq, ops

A = 1 << 20         # addresses that lie far apart: nothing is ever read from them here
M, F, K, N = 32, 24, 200, 48
EINVAL, OK = laq.LAQ_EINVAL, laq.LAQ_OK


@pytest.fixture(scope="module")
def lib():
    build.build()
    return laq.load_library()


def _blocks(codes, scales, cols, high=1):
    q = laq.laq_blocks()
    q.codes, q.ld_codes, q.scales, q.ld_scales, q.block_rows = codes, cols, scales, -(-cols // 128), high
    return q


def _err():
    return C.create_string_buffer(256)


def _pack(lib, x=A, dtype=1, rows=M, cols=K, ld=K, q=None):
    err = _err()
    rc = lib.laq_pack_blocks(x, dtype, rows, cols, ld, _blocks(2 * A, 3 * A, K) if q is None else q, None, err, 256)
    return rc, err.value.decode()


def _unpack(lib, x=A, dtype=1, rows=M, cols=K, ld=K, q=None):
    err = _err()
    rc = lib.laq_unpack_blocks(_blocks(2 * A, 3 * A, K) if q is None else q, rows, cols, x, dtype, ld, None, err, 256)
    return rc, err.value.decode()


def _changed(**kw):
    q = _blocks(2 * A, 3 * A, K)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


@pytest.mark.parametrize("bad, text", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"),
    (dict(cols=1 << 31), "cols"), (dict(ld=K - 1), "stride"), (dict(x=None), "null"), (dict(x=A + 1), "aligned"),
    (dict(q=_changed(codes=None)), "null"), (dict(q=_changed(scales=None)), "null"), (dict(q=_changed(block_rows=2)), "block_rows"),
    (dict(q=_changed(block_rows=0)), "block_rows"), (dict(q=_changed(ld_codes=K - 1)), "stride"), (dict(q=_changed(ld_scales=1)), "scales"),
    (dict(q=_changed(scales=3 * A + 2)), "scales"), (dict(q=_changed(ld_codes=1 << 62)), "beyond"),
])
def test_pack_and_unpack_refuse(lib, bad, text):
    for call in (_pack, _unpack):
        rc, message = call(lib, **bad)
        assert rc == EINVAL and text in message, message


def test_pack_and_unpack_refuse_shared_memory(lib):
    assert "overlap" in _pack(lib, x=2 * A)[1] and "overlap" in _unpack(lib, x=2 * A)[1]
    assert "overlap" in _pack(lib, q=_changed(scales=2 * A + 64))[1]
    assert "overlap" in _pack(lib, x=3 * A)[1] and "overlap" in _unpack(lib, x=3 * A)[1]
    for call in (_pack, _unpack):
        assert "overlap" not in call(lib)[1]
        assert call(lib, rows=0, x=None)[0] == OK                      # no rows: nothing is looked at
    assert lib.laq_pack_blocks(None, 9, 1, 1, 1, None, None, None, 0) == EINVAL      # the error text is optional


LAYER = {0: ["x", "x scales", "w", "w scales", "bias", "residual", "y", "z", "status"],
         1: ["dy", "x", "x scales", "w", "w scales", "z", "z scales", "dx", "dw", "db", "status"]}


def layer_call(lib, backward, place, workspace=None, rows=M, **kw):
    c = laq.laq_linear_call()
    c.dtype, c.activation, c.M, c.N, c.K, c.dw_dtype = 1, 1, rows, N, K, 0
    for name in LAYER[backward]:
        if hasattr(c, name) and name not in ("x", "w") and not (backward and name == "z"):
            setattr(c, name, place(name))
            if hasattr(c, "ld_" + name):
                setattr(c, "ld_" + name, K if name in ("dx", "dw") else N)
    for k, v in kw.items():
        if hasattr(c, k):
            setattr(c, k, v)
    xq, wq = _blocks(place("x"), place("x scales"), K), _blocks(place("w"), place("w scales"), K, 128)
    xq.block_rows, wq.block_rows = kw.get("x_high", 1), kw.get("w_high", 128)
    need = lib.laq_linear_blocks_workspace_bytes(C.byref(c), xq, wq, backward)
    err = _err()
    if backward:
        rc = lib.laq_linear_blocks_backward(C.byref(c), xq, wq, _blocks(place("z"), place("z scales"), N), workspace if need else None, need, None, err, 256)
    else:
        rc = lib.laq_linear_blocks_forward(C.byref(c), xq, wq, workspace if need else None, need, None, err, 256)
    return rc, err.value.decode()


GATED = {0: ["x", "w", "bias", "h", "z", "z scales", "status"],
         1: ["dh", "x", "x scales", "w", "z", "z scales", "dx", "dw", "db", "status"]}


def gated_call(lib, backward, place, workspace=None, packed=True, **kw):
    c = laq.laq_gated_call()
    c.dtype, c.activation, c.M, c.F, c.K = 1, 3, M, F, K
    wide = dict(x=K, w=K, dx=K, dw=K, z=2 * F)
    for name in GATED[backward]:
        if hasattr(c, name) and not (packed and (name == "z" or (backward and name == "x"))):
            setattr(c, name, place(name))
            if hasattr(c, "ld_" + name):
                setattr(c, "ld_" + name, wide.get(name, F))
    if packed:
        c.z_blocks = C.pointer(_blocks(place("z"), place("z scales"), 2 * F))
        if backward:
            c.x_blocks = C.pointer(_blocks(place("x"), place("x scales"), K))
    for k, v in kw.items():
        setattr(c, k, v)
    need = lib.laq_gated_workspace_bytes(C.byref(c), backward)
    err = _err()
    rc = (lib.laq_gated_backward if backward else lib.laq_gated_forward)(C.byref(c), workspace if need else None, need, None, err, 256)
    return rc, err.value.decode()


CALLS = [(layer_call, LAYER, 0), (layer_call, LAYER, 1), (gated_call, GATED, 0), (gated_call, GATED, 1)]
SIZES = {"x": 1, "w": 1, "z": 1, "x scales": 4, "w scales": 4, "z scales": 4, "db": 4, "status": 4}
IDS = ["linear8", "packed gradient", "gated", "gated gradient"]


def _size(call, names, backward, name):
    if call is gated_call and name == "w" or call is gated_call and name == "x" and not backward or call is layer_call and name == "z" and not backward:
        return 2
    return SIZES.get(name, 2)


@pytest.mark.parametrize("call, names, backward", CALLS, ids=IDS)
def test_every_pointer_is_checked_by_name(lib, call, names, backward):
    at = {n: A * (i + 1) for i, n in enumerate(names[backward])}
    for bad in names[backward]:
        if _size(call, names, backward, bad) > 1:
            rc, text = call(lib, backward, lambda n: at[n] + (1 if n == bad else 0), workspace=64 * A)
            assert rc == EINVAL and "aligned" in text and bad.split()[0] in text and ("scales" in text) == ("scales" in bad), (bad, text)
    outputs = {0: ["y", "z", "status", "h", "z scales"], 1: ["dx", "dw", "db", "status"]}[backward]
    for o in [n for n in outputs if n in names[backward]]:
        for other in names[backward]:
            if other == o or call is layer_call and not backward and (o, other) == ("y", "residual"):
                continue
            rc, text = call(lib, backward, lambda n: at[other] if n == o else at[n], workspace=64 * A)
            assert rc == EINVAL and "overlap" in text, (o, other, text)
    if backward:
        rc, text = call(lib, 1, lambda n: at[n], workspace=at["x"])
        assert "workspace" in text and "overlap" in text
    if not torch.cuda.is_available():
        assert "no current CUDA device" in call(lib, backward, lambda n: at[n], workspace=64 * A)[1]


@pytest.mark.parametrize("call, names, backward", CALLS, ids=IDS)
def test_sizes_and_settings(lib, call, names, backward):
    at = {n: A * (i + 1) for i, n in enumerate(names[backward])}
    place = lambda n: at[n]
    bads = [(dict(dtype=0), "dtype"), (dict(M=-1), "M must"), (dict(K=0), "K"), (dict(activation=4), "activation"), (dict(activation=-1), "activation"),
            (dict(status=None), "status"), (dict(flags=2), "flags")]
    bads += [(dict(F=0), "F must"), (dict(F=1 << 30), "F must"), (dict(K=65537), "K must")] if call is gated_call else [(dict(N=0), "M must")]
    for bad, text in bads:
        rc, message = call(lib, backward, place, workspace=64 * A, **bad)
        assert rc == EINVAL and text in message, (bad, message)
    if call is layer_call and not backward:
        assert "scale for each row" in layer_call(lib, 0, place, 64 * A, x_high=128)[1]
        assert "tile" in layer_call(lib, 0, place, 64 * A, w_high=1)[1]


def test_gated_refuses_both_forms_of_an_operand(lib):
    at = {n: A * (i + 1) for i, n in enumerate(GATED[1] + ["h", "bias"])}
    for backward in (0, 1):
        rc, text = gated_call(lib, backward, lambda n: at[n], workspace=64 * A, z=50 * A)
        assert rc == EINVAL and "z and z_blocks" in text
    rc, text = gated_call(lib, 1, lambda n: at[n], workspace=64 * A, x=50 * A)
    assert rc == EINVAL and "x and x_blocks" in text


def test_workspaces(lib):
    def need(backward, packed=False, **kw):
        c = laq.laq_gated_call()
        c.dtype, c.activation, c.M, c.F, c.K = 1, 3, 64, 24, 48
        c.x = c.w = c.dh = c.z = 4096
        c.ld_x = c.ld_w = 48
        c.ld_z = 48
        for k, v in kw.items():
            setattr(c, k, v)
        return lib.laq_gated_workspace_bytes(C.byref(c), backward), c
    assert need(0)[0] == 0 and need(0, x=4098)[0] == 64 * 48 * 2 and need(0, F=0)[0] == 0 and need(0, K=65537)[0] == 0
    assert need(1)[0] == 0 and need(1, dx=4096)[0] == 64 * 48 * 2
    assert need(1, db=4096)[0] == 512              # partial sums of two runs of 32 rows, 384 bytes, in units of 256
    size, c = need(1, dw=4096, ld_dw=48)
    c.status = 4096
    err = _err()
    for ws, n in ((None, 0), (4096 + 8, 1 << 20), (4096, size - 1)):
        assert lib.laq_gated_backward(C.byref(c), ws, n, None, err, 256) == laq.LAQ_EWORKSPACE
    q = _blocks(2 * A, 3 * A, 200)
    l = laq.laq_linear_call()
    l.dtype, l.M, l.N, l.K = 1, 32, 48, 200
    assert lib.laq_linear_blocks_workspace_bytes(C.byref(l), q, _blocks(5 * A, 6 * A, 208, 128), 0) == 32 * 208 + (-32 * 208) % 256      # x's pitch of 200 bytes
    assert lib.laq_linear_blocks_workspace_bytes(C.byref(l), None, None, 0) == 0
    l.dw = 4096
    assert lib.laq_linear_blocks_workspace_bytes(C.byref(l), q, None, 1) == 32 * 200 * 2            # x restored
    assert lib.laq_gated_workspace_bytes(None, 0) == 0 and lib.laq_linear_blocks_workspace_bytes(None, None, None, 0) == 0


def test_null_calls(lib):
    err = _err()
    assert lib.laq_gated_forward(None, None, 0, None, err, 256) == EINVAL and lib.laq_gated_backward(None, None, 0, None, err, 256) == EINVAL
    assert lib.laq_linear_blocks_forward(None, None, None, None, 0, None, err, 256) == EINVAL
    assert lib.laq_linear_blocks_backward(None, None, None, None, None, 0, None, err, 256) == EINVAL


@pytest.mark.parametrize("name", ["laq_blocks", "laq_gated_call"])
def test_struct_layout_matches_header(tmp_path, name):
    root, mirror = os.path.dirname(os.path.dirname(os.path.abspath(__file__))), getattr(laq, name)
    names = [f[0] for f in mirror._fields_]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "laq.h"', "int main(void){", 'printf("size %%zu\\n", sizeof(%s));' % name]
    lines += ['printf("%s %%zu\\n", offsetof(%s, %s));' % (n, name, n) for n in names] + ["return 0;}"]
    (tmp_path / "l.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = dict(l.split() for l in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(out["size"]) == C.sizeof(mirror)
    for n in names:
        assert int(out[n]) == getattr(mirror, n).offset, n


def test_binding_refuses():
    x = torch.zeros(4, 8)
    codes, scales = torch.zeros(4, 200).to(torch.float8_e4m3fn), torch.zeros(4, 2)
    for call in (lambda: ops.pack8(x), lambda: ops.unpack8(ops.Packed8(codes, scales)), lambda: ops.gated(x, x), lambda: ops.gated_backward(x, x, x, x),
                 lambda: ops.linear8(ops.Packed8(codes, scales), ops.Packed8(codes, scales)),
                 lambda: ops.linear_backward(x, ops.Packed8(codes, scales), x)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="Packed8"):
        ops.unpack8(codes)
    with pytest.raises(ValueError, match="Packed8"):
        ops.linear8(codes, codes)
