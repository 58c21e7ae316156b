"""probe_store waits for the current stream whichever way its own is named (no device: torch's
streams and the library's call are recorded)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2207_07736_amd import probe  # noqa: E402


class Stream:
    def __init__(self, address, log):
        self.cuda_stream, self.log = address, log

    def wait_stream(self, other):
        self.log.append((self.cuda_stream, "waits for", other.cuda_stream))


class Rows:
    is_cuda, device = True, "cuda:0"

    def data_ptr(self):
        return 256


@pytest.mark.parametrize("current", (0, 64, 128))
@pytest.mark.parametrize("own", ("none", "null", "raw", "stream"))
def test_the_store_follows_the_current_stream(monkeypatch, current, own):
    log = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(current, log))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0, log))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda address, device=None: Stream(address, log))

    class Library:
        @staticmethod
        def rlsim_probe_store(n, K, obs, action, reward, done, stream):
            log.append(("store", stream or 0))
            return 0

    monkeypatch.setattr(probe, "probe_lib", Library)
    stream, at = {"none": (None, 0), "null": (0, 0), "raw": (64, 64), "stream": (Stream(64, log), 64)}[own]
    rows = Rows()
    probe.probe_store(4, 2, rows, rows, rows, rows, stream=stream)
    assert log == ([] if at == current else [(at, "waits for", current)]) + [("store", at)]
