"""The torch classes' device scratch, which calls share a buffer, and their status words."""
import pytest
import torch

from paper_2606_21101_amd import dpi
from paper_2606_21101_amd.sequence import GatedRecurrence, SequenceEmbedding, _Workspaces


@pytest.fixture
def capturing(monkeypatch):
    """A switch in place of the device's answer, which needs a GPU."""
    now = {"is": False}
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now["is"])
    return now


def test_one_buffer_a_stream_that_grows(capturing):
    ws, cpu = _Workspaces(), torch.device("cpu")
    a = ws.get(7, 100, cpu)
    assert a.numel() >= 100 and ws.get(7, 60, cpu) is a and ws.get(8, 60, cpu) is not a
    assert ws.get(7, 200, cpu).numel() >= 200


def test_devices_share_no_buffer(capturing):
    """The default stream has the same handle on every device."""
    ws = _Workspaces()
    assert ws.get(0, 64, torch.device("cpu")).device.type == "cpu"
    assert ws.get(0, 64, torch.device("meta")).device.type == "meta"


def test_a_captured_call_shares_none(capturing):
    """What a graph writes to is not given to other calls, and not freed when one of them needs more."""
    ws, cpu = _Workspaces(), torch.device("cpu")
    eager = ws.get(7, 100, cpu)
    capturing["is"] = True
    first, second = ws.get(7, 100, cpu), ws.get(7, 100, cpu)
    assert first is not eager and first is not second and first.numel() >= 100
    capturing["is"] = False
    assert ws.get(7, 100, cpu) is eager


@pytest.mark.parametrize("status", [torch.zeros(1, dtype=torch.uint8), torch.zeros(1), torch.zeros(0, dtype=torch.int32)])
def test_a_status_that_is_no_word_is_refused(status):
    with pytest.raises(dpi.DpiError):
        SequenceEmbedding(torch.zeros((3, 4)), status=status)
    with pytest.raises(dpi.DpiError):
        GatedRecurrence(4, status=status)
