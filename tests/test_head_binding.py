"""The Python binding of the output head without a device: torch's streams and the library's
launches are recorded, tensors are the CPU's, and no kernel runs."""
import pytest

torch = pytest.importorskip("torch")

import paper_2207_07736_amd as p  # noqa: E402
from paper_2207_07736_amd import head as binding  # noqa: E402


class Stream:
    def __init__(self, name, address, log):
        self.name, self.cuda_stream, self.log = name, address, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


@pytest.fixture
def device(monkeypatch):
    """A log of launches and waits, streams to launch on, and the current one by name."""
    class Device:
        log, args, heads, current = [], [], [], "default"

    d = Device()
    d.streams = {name: Stream(name, at, d.log) for name, at in (("default", 0), ("own", 64), ("other", 128))}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: d.streams[d.current])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: d.streams["default"])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda at, device=None: next(s for s in d.streams.values() if s.cuda_stream == at))
    monkeypatch.setattr(binding, "rlsim_head_create", lambda *a: 1)
    monkeypatch.setattr(binding, "rlsim_head_destroy", lambda h: None)

    def launched(name):
        def f(h, args):
            d.log.append(name)
            d.args.append(args)
        return f

    monkeypatch.setattr(binding, "rlsim_head_distill", launched("distill"))
    monkeypatch.setattr(binding, "rlsim_head_sample", launched("sample"))

    def head(stream=None):
        h = p.Head(8, 16, stream=stream)
        h.device, h._ordinal = torch.device("cpu"), -1
        d.heads.append(h)
        return h

    d.head = head
    yield d
    for h in d.heads:                     # no handle is left for the real library to free
        h.h = None


def _teacher(rows=4):
    return torch.zeros(rows, 3), torch.zeros(rows, 3, dtype=torch.int32)


@pytest.mark.parametrize("own", ("default", "own"))
@pytest.mark.parametrize("current", ("default", "own", "other"))
@pytest.mark.parametrize("raw", (False, True))
def test_distill_loss_is_in_order_with_the_current_stream(device, own, current, raw):
    """Off the handle's stream, forward and backward launch between two waits: the handle's stream
    for the current one, then the current one for the handle's.  On it, they only launch."""
    stream = device.streams[own]
    head = device.head(None if own == "default" and not raw else stream.cuda_stream if raw else stream)
    device.current = current
    leaf = torch.zeros(4, 10, requires_grad=True)
    loss = head.distill_loss(leaf, *_teacher())
    want = ["distill"] if own == current else [(own, "waits for", current), "distill", (current, "waits for", own)]
    assert device.log == want
    device.log.clear()
    loss.mean().backward()
    assert device.log == want
    assert leaf.grad.shape == leaf.shape


def test_calls_without_a_graph_only_launch(device):
    """sample and distill are ordered by the caller: they take no part in torch's streams."""
    head = device.head(device.streams["own"])
    head.distill(torch.zeros(4, 10), *_teacher())
    head.sample(torch.zeros(4, 10), torch.zeros(4))
    assert device.log == ["distill", "sample"]


def test_a_gradient_written_in_place_is_seen_by_autograd(device):
    """What is written through an address raises the tensor's version, so that a graph which
    saved the tensor refuses to use the overwritten values; other tensors' versions stay."""
    head = device.head()
    leaf = torch.ones(4, 10, requires_grad=True)
    logits = leaf * 2.0
    other = (logits * logits).sum()                  # saves the logits
    out = head.distill(logits.detach(), *_teacher(), grad=logits.detach(), loss=False)
    assert out.data_ptr() == logits.data_ptr()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        other.backward()
    logits = leaf * 2.0
    other = (logits * logits).sum()
    teacher, index = _teacher()
    before = logits._version, teacher._version, index._version
    mine = torch.zeros(4, 10)
    head.distill(logits.detach(), teacher, index, grad=mine)
    head.distill(logits.detach(), teacher, index)
    head.sample(logits.detach(), torch.zeros(4))
    assert (logits._version, teacher._version, index._version) == before and mine._version == 1
    other.backward()


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
def test_no_rows(device, dtype):
    """An empty batch gives empty tensors, by no launch; its arguments are checked all the same."""
    head = device.head()
    logits, u = torch.zeros(0, 10, dtype=dtype), torch.zeros(0)
    teacher, index = _teacher(0)
    token = head.sample(logits, u, temperature=u, top_k=5)
    assert token.shape == (0,) and token.dtype == torch.int32
    token, logp = head.sample(logits, u, logp=True)
    assert token.shape == logp.shape == (0,) and logp.dtype == torch.float32
    loss, grad = head.distill(logits, teacher, index, rest=u, weight=u)
    assert loss.shape == (0,) and loss.dtype == torch.float32 and grad.shape == (0, 10) and grad.dtype == dtype
    out = torch.zeros(0, 10, dtype=dtype)
    assert head.distill(logits, teacher, index, grad=out, loss=False) is out
    assert head.distill(logits, teacher, index, grad=False).shape == (0,)
    leaf = logits.clone().requires_grad_()
    head.distill_loss(leaf, teacher, index).sum().backward()
    assert leaf.grad.shape == (0, 10)
    assert device.args == []
    for bad in (dict(u=torch.zeros(1)), dict(logits=logits.double()), dict(logits=torch.zeros(0)), dict(top_k=-1)):
        with pytest.raises(ValueError):
            head.sample(**{**dict(logits=logits, u=u), **bad})
    for bad in (dict(teacher=torch.zeros(1, 3)), dict(index=index.float()), dict(rest=torch.zeros(1)), dict(grad=torch.zeros(1, 10))):
        with pytest.raises(ValueError):
            head.distill(**{**dict(logits=logits, teacher=teacher, index=index), **bad})
