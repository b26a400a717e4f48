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
