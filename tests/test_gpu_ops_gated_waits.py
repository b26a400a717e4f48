"""A wait that runs out in the kernel of the gated block's long sums ends the call with a status, with and without projections, on pairs of SMs and
lone ones, and leaves the next calls as they were; the same calls captured, on two streams, and from two threads."""
import concurrent.futures as cf

import pytest
import torch

from paper_1909_07588_b200 import laq, ops
from tests.test_gpu_ops_linear import _randn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
# M, F, K, preact: tiles of pairs of SMs with and without Z, and of lone ones
CALLS = [(3000, 1500, 3001, False), (4097, 5504, 2048, True), (4097, 5504, 2048, "packed"), (2304, 4352, 136, "packed"), (1024, 768, 2048, False), (2500, 1100, 1100, True)]


def _flat(out):
    h, z = out if isinstance(out, tuple) and not isinstance(out, ops.Packed8) else (out, None)
    return [h] + ([z.codes.view(torch.uint8), z.scales] if isinstance(z, ops.Packed8) else [] if z is None else [z])


def _inputs(M, F, K):
    return _randn(M, K, seed=1, dtype=BF), _randn(2 * F, K, seed=2, dtype=BF, scale=K ** -0.5), _randn(2 * F, seed=3, dtype=BF)


@pytest.mark.parametrize("M, F, K, preact", CALLS)
def test_bounded_wait(M, F, K, preact):
    x, w, b = _inputs(M, F, K)
    before = _flat(ops.gated(x, w, b, preact=preact))
    ops.check_status()
    ops.gated(x, w, b, preact=preact, flags=ops.LINEAR_STARVE)
    with pytest.raises(laq.LaqError) as e:
        ops.check_status()
    assert e.value.status == laq.LAQ_ETIMEOUT
    for got, want in zip(_flat(ops.gated(x, w, b, preact=preact)), before):
        assert torch.equal(got, want)
    ops.check_status()


def test_captured_beside_one_another_and_from_threads():
    calls = [(_inputs(M, F, K), preact) for M, F, K, preact in CALLS]
    want = [_flat(ops.gated(*t, preact=p)) for t, p in calls]
    graphs = []
    for t, p in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = ops.gated(*t, preact=p)
        graphs.append((g, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(4):
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for (_, out, _), expected in zip(graphs, want):
        assert all(torch.equal(a, b) for a, b in zip(_flat(out), expected))

    def work(_):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.default_stream())
        for _ in range(5):
            for (t, p), expected in zip(calls, want):
                got = _flat(ops.gated(*t, preact=p, stream=s))
                s.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, expected))
        return "fine"
    with cf.ThreadPoolExecutor(2) as pool:
        assert list(pool.map(work, range(2), timeout=200)) == ["fine", "fine"]
    ops.check_status()
