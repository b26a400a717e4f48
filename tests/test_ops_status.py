"""The status word of the product kernels' bounded waits, without a GPU: host tensors stand in for the words."""
import pytest
import torch

from paper_1909_07588_b200 import laq, ops


@pytest.fixture
def devices(monkeypatch):
    """Two devices, 1 the current one; only 1 has had a wait that ran out."""
    words = {0: torch.zeros(1, dtype=torch.int32), 1: torch.tensor([5], dtype=torch.int32)}
    monkeypatch.setattr(ops, "_status", words)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    return words


@pytest.mark.parametrize("device", [None, "cuda", torch.device("cuda"), 1, "cuda:1", torch.device("cuda", 1)])
def test_a_device_without_an_index_is_the_current_one(devices, device):
    with pytest.raises(laq.LaqError) as e:
        ops.check_status(device)
    assert e.value.status == laq.LAQ_ETIMEOUT
    ops.check_status(device)


@pytest.mark.parametrize("device", [0, "cuda:0", torch.device("cuda", 0)])
def test_another_device_is_looked_at_by_its_index(devices, device):
    ops.check_status(device)
    with pytest.raises(laq.LaqError):
        ops.check_status(1)


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), "meta"])
def test_devices_that_are_no_gpus_are_refused(devices, device):
    for call in (ops.check_status, ops.init):
        with pytest.raises(ValueError, match="not a CUDA device"):
            call(device)


def _in_thread(body):
    """body() in a thread of its own: what it returned or raised."""
    import threading
    out = []

    def run():
        try:
            out.append(body())
        except Exception as e:
            out.append(e)
    t = threading.Thread(target=run)
    t.start()
    t.join()
    return out[0]


@pytest.fixture
def one_device(monkeypatch):
    words = {0: torch.zeros(1, dtype=torch.int32)}
    monkeypatch.setattr(ops, "_status", words)
    monkeypatch.setattr(ops, "_failures", {}, raising=False)
    import threading
    monkeypatch.setattr(ops, "_local", threading.local())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    return words[0]


def test_a_failure_is_told_to_every_thread(one_device):
    """Two threads have called; one's check finds the failure and clears the word; the other's still tells it, once."""
    import queue
    import threading
    orders, answers = queue.Queue(), queue.Queue()

    def other():
        while True:
            f = orders.get()
            if f is None:
                return
            try:
                answers.put(f())
            except laq.LaqError as e:
                answers.put(e.status)
    t = threading.Thread(target=other)
    t.start()
    ask = lambda f: (orders.put(f), answers.get())[1]
    try:
        ask(lambda: ops._status_word(0) is not None)
        ops._status_word(0)
        one_device.fill_(4)
        with pytest.raises(laq.LaqError):
            ops.check_status()
        assert int(one_device) == 0
        ops.check_status()
        assert ask(ops.check_status) == laq.LAQ_ETIMEOUT
        assert ask(ops.check_status) is None
        # the other way round, and two failures between two checks
        one_device.fill_(8)
        assert ask(ops.check_status) == laq.LAQ_ETIMEOUT
        one_device.fill_(8)
        assert ask(ops.check_status) == laq.LAQ_ETIMEOUT
        with pytest.raises(laq.LaqError):
            ops.check_status()
        ops.check_status()
        # a thread whose first call comes later has nothing to do with it; one that only checks (it may replay a captured
        # graph) hears of all
        assert _in_thread(lambda: (ops._status_word(0), ops.check_status())[1]) is None
        assert isinstance(_in_thread(ops.check_status), laq.LaqError)
    finally:
        orders.put(None)
        t.join()


def test_checks_of_many_threads_each_tell_a_failure_once(one_device):
    import threading
    n, told, start = 16, [], threading.Barrier(16)

    def run():
        ops._status_word(0)
        start.wait()
        if threading.get_ident() == first[0]:
            one_device.fill_(1)
        start.wait()
        for _ in range(50):
            try:
                ops.check_status()
            except laq.LaqError:
                told.append(threading.get_ident())
    first = [None]
    threads = [threading.Thread(target=run) for _ in range(n)]
    for t in threads:
        t.start()
        first[0] = first[0] or t.ident
    for t in threads:
        t.join()
    assert len(told) == n and len(set(told)) == n
