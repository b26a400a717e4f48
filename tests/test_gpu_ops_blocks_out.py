"""What is given as `out` of the calls on 8-bit matrices is looked at like every other argument."""
import pytest
import torch

from paper_1909_07588_b200 import laq, ops

pytestmark = pytest.mark.gpu


def test_out_of_pack8():
    x = torch.randn(40, 200, device="cuda")
    p = ops.pack8(x)
    for out in (p.codes, x, p.scales, [p.codes, p.scales], tuple(p), (), "out"):
        for stream in (None, torch.cuda.Stream()):
            with pytest.raises(ValueError, match="out must be a Packed8"):
                ops.pack8(x, out=out, stream=stream)
    for out in (ops.Packed8(x, p.scales), ops.Packed8(p.codes[:39], p.scales[:39]), ops.Packed8(p.codes, p.scales.cpu()), ops.Packed8(None, None)):
        with pytest.raises(ValueError, match="out"):
            ops.pack8(x, out=out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = ops.Packed8(torch.zeros_like(p.codes.view(torch.uint8)).view(torch.float8_e4m3fn), torch.zeros_like(p.scales))
    s.wait_stream(torch.cuda.current_stream())
    assert ops.pack8(x, out=q, stream=s) is q
    s.synchronize()
    assert torch.equal(q.codes.view(torch.uint8), p.codes.view(torch.uint8)) and torch.equal(q.scales, p.scales)


def test_out_of_unpack8():
    x = torch.randn(40, 200, device="cuda")
    p = ops.pack8(x)
    for out in ([], "out", p, x.cpu()):
        with pytest.raises(ValueError, match="out must be a CUDA tensor"):
            ops.unpack8(p, out=out)
    for out, text in ((x.double(), "dtype must be"), (x[:39], "out must have shape"), (x.t().contiguous().t(), "unit stride")):
        with pytest.raises(ValueError, match=text):
            ops.unpack8(p, out=out)
    memory = torch.zeros(40, 400, dtype=torch.uint8, device="cuda")          # codes in the left half of each row
    q = ops.Packed8(memory.view(torch.float8_e4m3fn)[:, :200], p.scales)
    with pytest.raises(laq.LaqError, match="overlap"):
        ops.unpack8(q, out=memory.view(torch.bfloat16))
