"""The order of the model operators' work and torch's, as the binding keeps it
(on stand-ins for torch's streams: no GPU is needed)."""
import contextlib
import types

import pytest

from paper_2601_17136_amd import kkm

torch = pytest.importorskip("torch")


class _Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


class _Tensor:
    def __init__(self, index, log):
        self.device = types.SimpleNamespace(index=index, type="cuda")
        self.log = log

    def record_stream(self, stream):
        self.log.append(("held for", stream.name))


@pytest.fixture
def two_devices(monkeypatch):
    """Device 0 is current; the tensors and the context (stream 7) are on device 1."""
    log, current = [], [0]

    @contextlib.contextmanager
    def device(index):
        index = index if isinstance(index, int) else index.index
        before, current[0] = current[0], index
        yield
        current[0] = before

    def name_of(d):
        if d is None:
            return current[0]
        return d if isinstance(d, int) else d.index

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: _Stream(f"current of {name_of(d)}", log))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d=None: _Stream(f"default of {name_of(d)}", log))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device=None: _Stream(f"stream {h} of {name_of(device)}", log))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    return log


@pytest.mark.parametrize("handle,place", [(7, "stream 7 of 1"), (0, "default of 1")])
def test_work_waits_for_the_stream_of_the_tensors_device(two_devices, monkeypatch, handle, place):
    log = two_devices
    monkeypatch.setattr(kkm, "kkm_get_stream", lambda ctx: handle)
    with kkm._ordered(None, _Tensor(1, log), _Tensor(1, log)):
        log.append("work")
    assert log == [(place, "waits for", "current of 1"), "work", ("current of 1", "waits for", place),
                   ("held for", place), ("held for", place)]


def test_no_order_is_needed_on_the_tensors_own_stream(two_devices, monkeypatch):
    log = two_devices
    monkeypatch.setattr(kkm, "kkm_get_stream", lambda ctx: 101)
    with kkm._ordered(None, _Tensor(1, log)):
        log.append("work")
    assert log == ["work"]


def test_addresses_and_absent_tensors_are_not_held(two_devices, monkeypatch):
    """Vectors may be given as raw addresses: their memory is the caller's to keep."""
    log = two_devices
    monkeypatch.setattr(kkm, "kkm_get_stream", lambda ctx: 7)
    with kkm._ordered(None, _Tensor(1, log), None, 0x7f0000000000, _Tensor(1, log)):
        log.append("work")
    assert log.count(("held for", "stream 7 of 1")) == 2 and "work" in log
