"""How calls of the operators stand beside each other and beside the rest of a program."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code, timeout=300):
    """In a process of its own: what is tested is what a process does first, or what it has left behind."""
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=timeout)
    assert out.returncode == 0, out.stderr[-3000:]
    return out.stdout


def test_an_error_of_an_earlier_call_is_not_taken_for_an_operators():
    """A library call that fails (a synchronisation on a stream under capture, refused on the host) leaves an error behind in
    its thread; an operator that follows runs, says so, and gives the results that it gives without."""
    assert "done" in _run("""
import torch
from paper_1909_07588_b200 import laq, ops
bf = torch.bfloat16
x, w = torch.randn(64, 96, device="cuda").to(bf), torch.randn(40, 96, device="cuda").to(bf)
logits = torch.randn(6, 5000, device="cuda")
tok = torch.randint(0, 5000, (6,), device="cuda").int()
dy = torch.randn(64, 40, device="cuda").to(bf)
one = torch.ones(6, device="cuda")
long = torch.randn(2, 140000, device="cuda")         # distilled in two passes
calls = [
    lambda: [ops.token_logprobs(logits, tok, top_k=3)["logprob"]],
    lambda: [ops.distill(logits, tok[:, None].contiguous(), one[:, None].contiguous(), d_loss=one)["dlogits"]],
    lambda: [ops.distill(long, tok[:2, None].contiguous(), one[:2, None].contiguous(), d_loss=one[:2])["dlogits"]],
    lambda: [ops.linear(x[:1], w)],
    lambda: [ops.linear(x, w)],
    lambda: [ops.linear(x[:, :95], w[:, 1:])],
    lambda: list(ops.linear_backward(dy, x, w, z=dy, activation="gelu").values()),
]
want = [c() for c in calls]
side = torch.cuda.Stream()
with torch.cuda.stream(side):
    ctx = laq.Laq(model=laq.MODEL_EXTERNAL, M=1, p=64, alpha=0.25, b=8, D=1, xi=[0.0], tbar=10)
    ctx.sync()
torch.cuda.synchronize()
failed = 0
for call, expected in zip(calls, want):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        try:
            ctx.sync()
        except laq.LaqError:
            failed += 1
        try:
            graph.capture_end()
        except RuntimeError:
            pass
    got = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, expected))
assert failed == len(calls)
ops.check_status()
print("done")
""")


def test_only_the_first_call_takes_device_memory_for_code():
    """After one small call of a row operator and one of a layer, no form of any call takes device memory other than what the
    framework's allocator takes for the outputs."""
    assert "done" in _run("""
import torch
from paper_1909_07588_b200 import ops
bf = torch.bfloat16

def rows(dt, T, V):
    x = torch.randn(T, V, device="cuda").to(dt)
    tok = torch.zeros(T, dtype=torch.int32, device="cuda")
    one = torch.ones(T, device="cuda")
    s = ops.token_logprobs(x, tok, top_k=3)
    ops.token_logprobs_backward(x, tok, s["lse"], s["entropy"], one, one)
    r = ops.distill(x, tok[:, None].contiguous(), one[:, None].contiguous(), d_loss=one)
    ops.distill(x, tok[:, None].contiguous(), one[:, None].contiguous())
    ops.distill_backward(x, tok[:, None].contiguous(), one[:, None].contiguous(), r["lse"], one)

def layer(dt, M, N, K, odd=0):
    x, w = torch.randn(M, K + odd, device="cuda").to(dt)[:, odd:], torch.randn(N, K, device="cuda").to(dt)
    dy = torch.randn(M, N, device="cuda").to(dt)
    ops.linear(x, w, activation="gelu")
    ops.linear_backward(dy, x, w, z=dy, activation="gelu")
    ops.linear_backward(dy, x, w, dw_dtype=torch.float32)

rows(torch.float32, 1, 8)
layer(bf, 8, 8, 8)
torch.cuda.synchronize()

def used():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved()

for dt in (torch.float32, bf, torch.float16):       # what the framework itself needs for the inputs
    torch.randn(3, 4, device="cuda").to(dt)
start = used()
for dt in (torch.float32, bf, torch.float16):
    for T, V in ((3, 500), (2, 5000), (2400, 1500), (1200, 2100), (2, 30000), (2, 140000), (1, 270000)):
        rows(dt, T, V)
        assert used() == start, (dt, T, V)
for dt in (bf, torch.float16):
    for M, N, K in ((1, 40, 4000), (1, 40, 40), (2, 40, 4000), (3, 40, 40), (4, 40, 40), (16, 512, 2048), (300, 300, 264), (2048, 2048, 512),
                    (70000, 16, 24), (66000, 512, 512)):
        for odd in (0, 1):
            layer(dt, M, N, K, odd)
            assert used() == start, (dt, M, N, K, odd)
ops.check_status()
print("done")
""")


def test_first_calls_of_a_thread():
    """Each operator as the first thing that a thread does with the device, and its results."""
    assert "done" in _run("""
import concurrent.futures as cf
import torch
from paper_1909_07588_b200 import ops
bf = torch.bfloat16
x, w, dy = torch.randn(300, 512, device="cuda").to(bf), torch.randn(40, 512, device="cuda").to(bf), torch.randn(300, 40, device="cuda").to(bf)
logits = torch.randn(6, 5000, device="cuda")
tok = torch.randint(0, 5000, (6,), device="cuda").int()
one = torch.ones(6, device="cuda")
out = torch.empty(300, 40, device="cuda", dtype=bf)
calls = [
    lambda: list(ops.token_logprobs(logits, tok, top_k=3).values()),
    lambda: [ops.token_logprobs_backward(logits, tok, one, d_logprob=one)],
    lambda: list(ops.distill(logits, tok[:, None], one[:, None]).values()),
    lambda: list(ops.distill(logits, tok[:, None], one[:, None], d_loss=one).values()),
    lambda: [ops.distill_backward(logits, tok[:, None], one[:, None], one, one)],
    lambda: [ops.linear(x[:1], w)],
    lambda: [ops.linear(x, w, out=out)],
    lambda: [ops.linear(x[:, 1:], w[:, 1:])],
    lambda: list(ops.linear_backward(dy, x, w, z=dy, activation="gelu").values()),
]
want = [[t.clone() for t in c()] for c in calls]
torch.cuda.synchronize()
for call, expected in zip(calls, want):
    with cf.ThreadPoolExecutor(1) as pool:
        got = pool.submit(call).result(timeout=60)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, expected))
ops.check_status()
print("done")
""")


def test_a_wait_that_ran_out_is_told_to_every_caller():
    """The starved call's thread and another that called before it: each check tells the failure once."""
    assert "done" in _run("""
import threading, queue
import torch
from paper_1909_07588_b200 import laq, ops
bf = torch.bfloat16
x, w = torch.randn(300, 512, device="cuda").to(bf), torch.randn(300, 512, device="cuda").to(bf)
ops.linear(x, w)
orders, answers = queue.Queue(), queue.Queue()
def status():
    try:
        ops.check_status()
        return "ok"
    except laq.LaqError as e:
        return e.status
def other():
    while (f := orders.get()) is not None:
        try:
            answers.put(f())
        except Exception as e:
            answers.put(e)
t = threading.Thread(target=other, daemon=True)
t.start()
ask = lambda f: (orders.put(f), answers.get(timeout=60))[1]
def starve():
    ops.linear(x, w, flags=ops.LINEAR_STARVE)
    return status()
assert ask(lambda: (ops.linear(x, w), status())[1]) == "ok" and status() == "ok"
assert ask(starve) == laq.LAQ_ETIMEOUT
assert status() == laq.LAQ_ETIMEOUT and status() == "ok" and ask(status) == "ok"
orders.put(None)
t.join()
print("done")
""")


def test_inputs_may_be_let_go_of_when_a_call_on_another_stream_has_returned():
    """A call on a stream that is busy, its inputs dropped at once and their memory asked for again on the caller's stream:
    what is written there meanwhile must not reach the call."""
    assert "done" in _run("""
import torch
from paper_1909_07588_b200 import ops
bf = torch.bfloat16
side = torch.cuda.Stream()
g = torch.Generator(device="cuda")

def made():
    # fresh tensors of the caller's stream, the same values every time
    g.manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    n, V, K = 64, 30000, 8
    return dict(x=rnd(n, V).to(bf), tok=torch.randint(0, V, (n,), generator=g, device="cuda").int(), a=rnd(n), b=rnd(n), c=rnd(n),
                tt=torch.randint(0, V, (n, K), generator=g, device="cuda").int(), tv=rnd(n, K), h=rnd(n, 2048).to(bf), w=rnd(1024, 2048).to(bf),
                bias=rnd(1024).to(bf), r=rnd(n, 1024).to(bf), dy=rnd(n, 1024).to(bf))

calls = [
    lambda t, s: ops.token_logprobs(t["x"], t["tok"], top_k=4, stream=s),
    lambda t, s: dict(dx=ops.token_logprobs_backward(t["x"], t["tok"], t["a"], t["b"], t["c"], t["a"], stream=s)),
    lambda t, s: ops.distill(t["x"], t["tt"], t["tv"], d_loss=t["a"], stream=s),
    lambda t, s: dict(dx=ops.distill_backward(t["x"], t["tt"], t["tv"], t["a"], t["b"], stream=s)),
    lambda t, s: dict(y=ops.linear(t["h"], t["w"], t["bias"], activation="gelu", residual=t["r"], stream=s)),
    lambda t, s: ops.linear_backward(t["dy"], t["h"], t["w"], z=t["r"], activation="gelu", stream=s),
]
for call in calls:
    want = call(made(), None)
    torch.cuda.synchronize()
    t = made()
    shapes = [(v.shape, v.dtype) for v in t.values()]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)               # some 0.2 s
    got = call(t, side)
    t = None
    for _ in range(3):                               # the memory is there again if the allocator hands it out
        again = [torch.zeros(s, dtype=d, device="cuda") for s, d in shapes]
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k
ops.check_status()
print("done")
""")
