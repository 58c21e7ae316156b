"""The Python binding of the learner's operators without a device: torch's streams and the
library's launches are recorded, tensors are the CPU's, and no kernel runs."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2207_07736_amd as p  # noqa: E402
from paper_2207_07736_amd import learn as binding  # noqa: E402


class Stream:
    def __init__(self, name, address, log):
        self.name, self.cuda_stream, self.log = name, address, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


@pytest.fixture
def device(monkeypatch):
    """A log of launches and waits, streams to launch on, and the current one by name."""
    class Device:
        log, args, learners, current, capturing = [], [], [], "default", False

    d = Device()
    d.log, d.args, d.learners = [], [], []
    d.streams = {name: Stream(name, at, d.log) for name, at in (("default", 0), ("own", 64), ("other", 128))}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: d.streams[d.current])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: d.streams["default"])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: d.capturing)
    monkeypatch.setattr(binding, "rlsim_learner_create", lambda *a: 1)
    monkeypatch.setattr(binding, "rlsim_learner_destroy", lambda h: None)

    def launched(name):
        def f(h, *args):
            d.log.append(name)
            d.args.append(args)
        return f

    for name in ("scan", "scan_grad", "xent", "clip"):
        monkeypatch.setattr(binding, "rlsim_learner_" + name, launched(name))

    def learner(stream=None):
        made = p.Learner(8, 16, 32, stream=stream)
        made.device, made._ordinal = torch.device("cpu"), -1
        d.learners.append(made)
        return made

    d.learner = learner
    yield d
    for made in d.learners:               # no handle is left for the real library to free
        made.h = None


@pytest.mark.parametrize("own", ("default", "own"))
@pytest.mark.parametrize("current", ("default", "own", "other"))
def test_autograd_launches_in_order_with_the_current_stream(device, own, current):
    learner = device.learner(None if own == "default" else device.streams["own"])
    device.current = current
    x, gate = torch.zeros((5, 2, 3), requires_grad=True), torch.zeros((5, 2, 3), requires_grad=True)
    y, last = learner.recur(x, gate)
    (y.sum() + last.sum()).backward()
    hidden, matrix = torch.zeros((4, 3), requires_grad=True), torch.zeros((7, 3), requires_grad=True)
    learner.cross_entropy_loss(hidden, matrix, torch.zeros(4, dtype=torch.int64)).sum().backward()
    names = [entry for entry in device.log if isinstance(entry, str)]
    assert names == ["scan", "scan_grad", "xent", "xent"]
    if own == current:
        assert device.log == names
    else:
        for k, name in enumerate(names):
            assert device.log[3 * k:3 * k + 3] == [(own, "waits for", current), name, (current, "waits for", own)]


def test_plain_calls_wait_for_nothing(device):
    learner = device.learner(device.streams["own"])
    x = torch.zeros((5, 2, 3))
    y, last, marks = learner.scan(x, x, marks=True)
    learner.scan_grad(x, x, marks, y)
    learner.cross_entropy(x[0], x[0], torch.zeros(2, dtype=torch.uint8))
    learner.clip([x, None], 1.0)
    assert device.log == ["scan", "scan_grad", "xent", "clip"]


def test_autograd_is_not_captured(device):
    learner = device.learner()
    x = torch.zeros((5, 2, 3), requires_grad=True)
    y, _ = learner.recur(x, x)
    loss = learner.cross_entropy_loss(x[0], x[1], torch.zeros(2, dtype=torch.int64))
    device.capturing = True
    for call in (lambda: learner.recur(x, x), lambda: learner.cross_entropy_loss(x[0], x[1], torch.zeros(2, dtype=torch.int64)),
                 lambda: y.sum().backward(), lambda: loss.sum().backward()):
        with pytest.raises(RuntimeError, match="not captured"):
            call()
    assert device.log == ["scan", "xent"]
    learner.scan(x.detach(), x.detach())              # the plain calls are


@pytest.mark.parametrize("order", ("time", "batch", "wide"))
def test_rows_in_time_and_their_strides(device, order):
    learner = device.learner()
    T, n, d = 4, 3, 5
    x = (torch.zeros((T, n, d)) if order == "time" else torch.zeros((n, T, d)).transpose(0, 1) if order == "batch"
         else torch.zeros((T, n, d + 3))[:, :, 1:d + 1])
    state, done = torch.zeros((n, d)), torch.zeros((T, n), dtype=torch.bool)
    y, last, marks = learner.scan(x, x, state, done, marks=True, last=state)
    (a,) = device.args[-1]
    assert (a.T, a.n, a.channels, a.dtype) == (T, n, d, p.RLSIM_F32)
    assert (a.x, a.x_step, a.x_seq) == (x.data_ptr(), *x.stride()[:2]) == (a.gate, a.gate_step, a.gate_seq)
    assert (a.y, a.y_step, a.y_seq) == (y.data_ptr(), *y.stride()[:2]) and y.shape == x.shape and y.stride(2) == 1
    assert (y.stride(1) > y.stride(0)) == (order == "batch")
    assert last is state and a.last == a.state == state.data_ptr() and a.done == done.data_ptr()
    assert marks.shape == (1, n, d) and a.marks == marks.data_ptr()
    dx, dgate, dstate = learner.scan_grad(x, x, marks, None, done, state)
    a, g = device.args[-1]
    assert g.dy is None and g.dlast == state.data_ptr() and g.dx == dx.data_ptr() and g.dstate == dstate.data_ptr()
    assert (g.dx_step, g.dx_seq) == dx.stride()[:2] and (g.dgate_step, g.dgate_seq) == dgate.stride()[:2]


def test_writes_raise_versions(device):
    learner = device.learner()
    x, state, stats = torch.zeros((2, 3, 4)), torch.zeros((3, 4)), torch.zeros((2, 3))
    before = state._version
    learner.scan(x, x, state)
    assert state._version == before
    learner.scan(x, x, state, last=state)
    assert state._version == before + 1
    learner.cross_entropy(x[0, :2], x[1], torch.zeros(2, dtype=torch.int64), stats=stats)
    assert stats._version == 1
    a, b, out = torch.zeros(5), torch.zeros(5), torch.zeros(5)
    learner.clip([a], float("inf"))
    assert a._version == 0
    learner.clip([a, b], 1.0)
    assert a._version == b._version == 1
    learner.clip([a], 1.0, out=[out])
    assert a._version == 1 and out._version == 1


def test_the_table_of_tensors(device, monkeypatch):
    learner = device.learner()
    a, b = torch.zeros(7), torch.zeros((2, 3), dtype=torch.bfloat16)
    out = [torch.zeros(7, dtype=torch.float16), torch.zeros((2, 3))]
    rows = []

    def look(h, table, count, max_norm, norm):
        rows.append([binding.rlsim_tensor.from_address(table + i * ctypes.sizeof(binding.rlsim_tensor)) for i in range(count)])
        rows[-1] = [(r.data, r.out, r.elements, r.dtype, r.out_dtype) for r in rows[-1]]

    monkeypatch.setattr(binding, "rlsim_learner_clip", look)
    learner.clip([a, None, b], 2.0)
    learner.clip([a, None, b], 2.0, out=[out[0], None, out[1]])
    assert rows[0] == [(a.data_ptr(), None, 7, p.RLSIM_F32, p.RLSIM_F32), (b.data_ptr(), None, 6, p.RLSIM_BF16, p.RLSIM_BF16)]
    assert rows[1] == [(a.data_ptr(), out[0].data_ptr(), 7, p.RLSIM_F32, p.RLSIM_F16),
                       (b.data_ptr(), out[1].data_ptr(), 6, p.RLSIM_BF16, p.RLSIM_F32)]


def test_only_the_gradients_that_are_needed(device):
    learner = device.learner()
    for wants in ((True, False), (False, True)):
        hidden, matrix = torch.zeros((4, 3), requires_grad=wants[0]), torch.zeros((7, 3), requires_grad=wants[1])
        learner.cross_entropy_loss(hidden, matrix, torch.zeros(4, dtype=torch.int64)).sum().backward()
        (a,) = device.args[-1]
        assert (a.dhidden is not None, a.dmatrix is not None) == wants and a.loss is None and a.stats is not None


def test_refusals(device):
    learner = device.learner()
    x = torch.zeros((4, 3, 8))
    t = torch.zeros(3, dtype=torch.int64)
    bad = [
        (lambda: learner.scan(x[0], x[0]), "3-d"), (lambda: learner.scan(x, x.bfloat16()), "gate"),
        (lambda: learner.scan(x, x, torch.zeros((3, 8), dtype=torch.float64)), "state"),
        (lambda: learner.scan(x, x, done=torch.zeros((3, 4), dtype=torch.bool)), "done"),
        (lambda: learner.scan(x, x, last=torch.zeros((8, 3)).t()), "last"), (lambda: learner.scan(x.long(), x.long()), "float32"),
        (lambda: learner.scan_grad(x, x, None), "marks"), (lambda: learner.scan_grad(x, x, torch.zeros((1, 3, 8)), x[:3]), "dy"),
        (lambda: learner.scan_grad(x, x, torch.zeros((1, 3, 8)), dlast=torch.zeros(3)), "dlast"),
        (lambda: learner.cross_entropy(x[0], x[0], t, stats=torch.zeros(6)), "stats"),
        (lambda: learner.cross_entropy(x[0], x[0][:, :7], t), "matrix"),
        (lambda: learner.cross_entropy(x[0].expand(2, 3, 8)[0][:1].expand(3, 8), x[0], t), "rows apart"),
        (lambda: learner.clip([x.long()], 1.0), "float32"), (lambda: learner.clip([x[:, :, ::2]], 1.0), "side by side"),
        (lambda: learner.clip([x], 1.0, out=[x.long()]), "out"), (lambda: learner.clip([x], 0.0), "max_norm"),
    ]
    for call, match in bad:
        with pytest.raises(ValueError, match=match):
            call()
    assert not device.log
