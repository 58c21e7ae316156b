"""Distillation from a teacher's top logits on the GPU: losses and gradients lie within the
derived bounds of 64-bit ones at every size, mask and layout."""
import math

import numpy as np
import pytest

import head_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BITS = {torch.float32: 24, torch.bfloat16: 8, torch.float16: 11}
SIZES = (1, 2, 3, 5, 8, 13, 31, 33, 64, 65, 71, 127, 511, 512, 513, 1023, 1025, 2048, 2049, 4097, 8191, 8200, 16385,
         32769, 65537, 131080, 200003)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def head():
    import paper_2207_07736_amd as p
    h = p.Head(1 << 20, 1 << 20)
    yield h
    h.close()


def _same(got, want, tol, what):
    got, want, tol = np.asarray(got, np.float64), np.asarray(want, np.float64), np.asarray(tol, np.float64)
    with np.errstate(invalid="ignore"):
        ok = (np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (what, int((~ok).sum()), np.argwhere(~ok)[:3].tolist(), got[~ok][:3], want[~ok][:3])


def _check(head, s, t, index, tau=1.0, rest=None, weight=None, in_place=False):
    """Loss and gradient of one call against the plain rows."""
    dev = lambda v: None if v is None else torch.from_numpy(np.asarray(v, np.float32)).cuda()  # noqa: E731
    work = s.clone() if in_place else s
    loss, grad = head.distill(work, t, index, tau, dev(rest), dev(weight), grad=work if in_place else True)
    tau32 = float(np.float32(tau))
    sh, th, ih = s.float().cpu().numpy(), t.float().cpu().numpy(), index.cpu().numpy()
    lo, gr = loss.cpu().numpy(), grad.float().cpu().numpy()
    for r in range(s.shape[0]):
        slots = list(zip(ih[r].tolist(), th[r].tolist()))
        rr = None if rest is None else float(np.float32(rest[r]))
        w = 1.0 if weight is None else float(np.float32(weight[r]))
        want, g = ref.distill_row(sh[r], slots, tau32, rr, w)
        with np.errstate(all="ignore"):
            tl, tg = ref.distill_tolerance(sh[r], slots, tau32, rr, w, BITS[s.dtype])
        with np.errstate(over="ignore"):
            want = np.float32(want)                  # what the output can hold: beyond it, infinity
        _same(lo[r], want, tl if np.isfinite(tl) else 0.0, f"loss {r}")
        _same(gr[r], g, np.nan_to_num(tg, nan=0.0, posinf=0.0), f"gradient {r}")
    return loss, grad


def _case(rng, rows, V, k, dtype, index_dtype=torch.int32):
    s = (rng.standard_normal((rows, V)) * 3).astype(np.float32)
    t = (s + rng.standard_normal((rows, V))).astype(np.float32)
    top = np.argsort(-t, axis=1)[:, :k]
    rest = np.full(rows, -np.inf)
    if k < V:
        left = t.copy()
        np.put_along_axis(left, top, -np.inf, axis=1)
        rest = left.max(axis=1) + np.log(np.exp(left - left.max(axis=1, keepdims=True)).sum(axis=1))
    return (torch.from_numpy(s).cuda().to(DTYPES[dtype]),
            torch.from_numpy(np.take_along_axis(t, top, axis=1)).cuda().to(DTYPES[dtype]),
            torch.from_numpy(top).cuda().to(index_dtype), rest.astype(np.float32))


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_loss_and_gradient_at_every_size(head, V, dtype):
    rng = np.random.default_rng(V)
    rows = 8 if V < 5000 else 3
    for k, tau, with_rest in ((min(V, 2), 1.0, False), (min(V, 33), 2.0, True), (min(V, 150), 0.5, True)):
        s, t, index, rest = _case(rng, rows, V, k, dtype, torch.int64 if k == 2 else torch.int32)
        weight = rng.uniform(-2, 2, rows).astype(np.float32)
        _check(head, s, t, index, tau, rest if with_rest else None, weight)


@pytest.mark.parametrize("V", (4, 50, 600, 5000, 70001, 150000))
@pytest.mark.parametrize("with_rest", (False, True))
def test_masked_rows(head, V, with_rest):
    """Empty slots and rows, repeated entries, entries outside the row, masked student
    entries, NaN where nothing counts, weights of 0, and NaN that does count."""
    rng = np.random.default_rng(V)
    k = min(V, 20)
    for dtype in DTYPES:
        s, t, index, rest = _case(rng, 16, V, k, dtype)
        weight = rng.uniform(0.5, 2, 16).astype(np.float32)
        index[0] = -1
        t[0] = math.nan
        s[0] = math.nan
        rest[0] = -math.inf
        index[1, k // 2:] = -1
        t[1, k // 2:] = math.nan
        index[2, -1] = index[2, 0]
        t[2, -1] = 100.0
        index[3, 0] = V
        index[3, k // 2] = -7
        index[4, 0] = 2 ** 31 - 1
        weight[5] = 0.0
        s[5] = math.nan
        s[6, V // 2] = -math.inf
        t[6][index[6] == V // 2] = -math.inf
        s[7] = -math.inf
        t[8] = -math.inf
        rest[8] = -math.inf
        s[9, index[9].long()] = -math.inf
        t[10, 1:] = -math.inf
        s[11, 0] = math.nan
        t[12, 0] = math.nan
        s[13] = float(torch.finfo(s.dtype).min)
        s[14, 1:] = float(torch.finfo(s.dtype).min)
        rest[15] = -math.inf
        loss, grad = _check(head, s, t, index, 1.5, rest if with_rest else None, weight)
        assert loss[0] == 0 and not grad[0].any() and not grad[5].any()
        assert torch.isnan(loss[11]) and torch.isnan(loss[12])


@pytest.mark.parametrize("V", (64, 400, 3000, 40000, 200000))
def test_teachers_that_list_everything_or_nothing(head, V):
    """The rest alone; every entry listed with a rest left over; as many slots as a call takes."""
    rng = np.random.default_rng(V)
    s, t, index, rest = _case(rng, 3, V, min(V, 1024), "f32")
    _check(head, s, t, index, 1.0, rest)
    _check(head, s, t, index, 1.0)
    none = torch.full_like(index, -1)
    loss, grad = _check(head, s, t, none, 1.0, rest + 1.0 if V > 1024 else np.ones(3))
    assert loss.abs().max() < 1e-4 and grad.abs().max() < 1e-4
    if V <= 1024:
        loss, grad = head.distill(s, t, index, rest=torch.ones(3, device="cuda"))
        assert torch.isinf(loss).all() and torch.isfinite(grad).all()


def test_nearly_all_mass_listed(head):
    """The unlisted part is a millionth of the student's: as 1 - sum q it would vanish."""
    rng = np.random.default_rng(3)
    for V in (60, 3000, 100000):
        s, t, index, _ = _case(rng, 4, V, 6, "f32")
        s.scatter_add_(1, index.long(), torch.full(index.shape, 25.0 + math.log(V), device="cuda"))
        t += 25.0 + math.log(V)
        _check(head, s, t, index, 1.0, np.full(4, 9.0, np.float32))


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_place_equals_a_gradient_of_its_own(head, dtype):
    rng = np.random.default_rng(4)
    for V in (2, 64, 1001, 9000, 50001, 131072, 180001):
        s, t, index, rest = _case(rng, 5, V, min(V, 40), dtype)
        r = torch.from_numpy(rest).cuda() if V > 40 else None
        want = head.distill(s, t, index, 2.0, r)
        work = s.clone()
        got = head.distill(work, t, index, 2.0, r, grad=work)
        assert got[1].data_ptr() == work.data_ptr()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(head.distill(s, t, index, 2.0, r, loss=False), want[1])
        assert torch.equal(head.distill(s, t, index, 2.0, r, grad=False), want[0])


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_addresses_and_types(head, dtype):
    """Rows apart and at odd elements, for every tensor; a teacher of another type; what
    lies between the rows stays."""
    rng = np.random.default_rng(5)
    for V, k in ((2, 2), (63, 9), (1001, 20), (20011, 64), (140001, 5)):
        s, t, index, rest = _case(rng, 5, V, k, dtype)
        wide = torch.full((5, V + 7), 3.0, device="cuda", dtype=s.dtype)
        wide[:, 3:3 + V] = s
        out = torch.full((5, V + 9), 5.0, device="cuda", dtype=s.dtype)
        tw = torch.zeros((5, k + 3), device="cuda")
        tw[:, 1:1 + k] = t.float()
        iw = torch.zeros((5, k + 1), device="cuda", dtype=torch.int64)
        iw[:, 1:] = index
        r = torch.from_numpy(rest).cuda() if k < V else None
        want = head.distill(s, t.float(), index, 1.3, r)
        got = head.distill(wide[:, 3:3 + V], tw[:, 1:1 + k], iw[:, 1:], 1.3, r, grad=out[:, 5:5 + V])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert (out[:, :5] == 5).all() and (out[:, 5 + V:] == 5).all()
        assert torch.equal(head.distill(wide[1:2, 3:3 + V], tw[1:2, 1:1 + k], iw[1:2, 1:], 1.3, None if r is None else r[1:2])[1],
                           want[1][1:2])


def test_rows_past_32_bits(head):
    V, stride = 70001, (1 << 31) + 8
    store = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    s = store.as_strided((3, V), (stride, 1))
    rng = np.random.default_rng(6)
    data, t, index, rest = _case(rng, 3, V, 30, "bf16")
    s.copy_(data)
    r = torch.from_numpy(rest).cuda()
    want = head.distill(data, t, index, 1.0, r)
    got = head.distill(s, t, index, 1.0, r, grad=s)
    assert torch.equal(got[0], want[0]) and torch.equal(s, want[1])


def test_a_row_does_not_depend_on_its_batch(head):
    rng = np.random.default_rng(7)
    for V, k in ((2, 2), (40, 5), (900, 20), (12000, 64), (90000, 64)):
        s, t, index, rest = _case(rng, 600, V, k, "bf16")
        r = torch.from_numpy(rest).cuda() if k < V else None
        whole = head.distill(s, t, index, 2.0, r)
        again = head.distill(s, t, index, 2.0, r)
        assert torch.equal(whole[0], again[0]) and torch.equal(whole[1], again[1])


@pytest.mark.parametrize("V,k", ((65, 9), (700, 9), (5003, 33), (20011, 64), (70001, 20), (150001, 100)))
@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows(head, V, k, dtype):
    """Calls of more rows than workgroups can share: rows picked from all over the batch
    against the plain ones, and against calls of few rows within both calls' bounds."""
    rng = np.random.default_rng(V)
    rows = 700
    s, t, index, rest = _case(rng, 7, V, k, dtype)
    turn = torch.arange(rows, device="cuda") % 7
    weight = torch.from_numpy(rng.uniform(0.5, 2, rows).astype(np.float32)).cuda()
    weight[350] = 0.0
    r = torch.from_numpy(rest).cuda()
    index[3, 1] = index[3, 0]
    index[4] = -1
    r[4] = -math.inf
    rest[4] = -math.inf
    loss, grad = head.distill(s[turn], t[turn], index[turn], 2.0, r[turn], weight)
    assert not grad[350].any()
    sh, th, ih = s.float().cpu().numpy(), t.float().cpu().numpy(), index.cpu().numpy()
    for row in (0, 1, 2, 3, 4, 355, 356, 511, 512, 513, 697, 698, 699):
        j = row % 7
        w = float(weight[row])
        slots = list(zip(ih[j].tolist(), th[j].tolist()))
        want, g = ref.distill_row(sh[j], slots, 2.0, float(rest[j]), w)
        with np.errstate(all="ignore"):
            tl, tg = ref.distill_tolerance(sh[j], slots, 2.0, float(rest[j]), w, BITS[s.dtype])
        _same(loss[row].cpu().numpy(), want, tl, f"loss {row}")
        _same(grad[row].float().cpu().numpy(), g, tg, f"gradient {row}")
    in_place = s[turn]
    again = head.distill(in_place, t[turn], index[turn], 2.0, r[turn], weight, grad=in_place)
    assert torch.equal(again[0], loss) and torch.equal(again[1], grad)


def test_the_loss_moves_as_the_gradient_says(head):
    """Central differences of the kernel's own losses, step h along a direction d of entries
    within [-1, 1].  At tau = 1 the loss is a log-sum-exp less a linear part (with a rest:
    less p_r of another log-sum-exp), whose third derivative along d is at most 8 (16) in
    magnitude, so the difference is off by 16 h^2 / 6, and by the losses' own error over h."""
    rng = np.random.default_rng(8)
    h = 2.0 ** -6
    for V, k in ((5, 2), (200, 9), (30000, 50)):
        s, t, index, rest = _case(rng, 4, V, k, "f32")
        r = torch.from_numpy(rest).cuda()
        d = torch.from_numpy(rng.uniform(-1, 1, (4, V)).astype(np.float32)).cuda()
        _, g = head.distill(s, t, index, 1.0, r)
        up, down = (head.distill(s + x * d, t, index, 1.0, r, grad=False).double() for x in (h, -h))
        slope = ((up - down) / (2 * h)).cpu().numpy()
        want = (g.double() * d.double()).sum(dim=1).cpu().numpy()
        for row in range(4):
            slots = list(zip(index[row].tolist(), t[row].tolist()))
            tol, _ = ref.distill_tolerance(s[row].cpu().numpy(), slots, 1.0, float(rest[row]), 1.0, 24)
            # s +- h d is itself rounded: 2^-24 of the largest logit, times sum |g| <= 2
            off = 16 * h * h / 6 + tol / h + 2 * 2.0 ** -24 * float(s[row].abs().max()) / h
            assert abs(slope[row] - want[row]) <= off, (V, row, slope[row], want[row], off)


def test_autograd(head):
    rng = np.random.default_rng(9)
    for dtype in DTYPES:
        s, t, index, rest = _case(rng, 6, 700, 11, dtype)
        r = torch.from_numpy(rest).cuda()
        leaf = s.clone().requires_grad_()
        loss = head.distill_loss(leaf, t, index, 2.0, r)
        (loss * torch.arange(6, device="cuda")).sum().backward()
        want = head.distill(s, t, index, 2.0, r, weight=torch.arange(6, device="cuda").float())
        assert torch.equal(loss.detach(), want[0]) and torch.equal(leaf.grad, want[1])
        leaf.grad = None
        head.distill_loss(leaf, t, index, 2.0, r).mean().backward()
        mean = head.distill(s, t, index, 2.0, r, weight=torch.full((6,), 1 / 6, device="cuda"))
        assert torch.equal(leaf.grad, mean[1])


def test_graph_replays(head):
    import paper_2207_07736_amd as p
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(10)
    h = p.Head(16, 200000, stream=stream)
    try:
        for V in (2, 500, 30000, 150001):
            s, t, index, rest = _case(rng, 8, V, min(V - 1, 30), "f32")
            r = torch.from_numpy(rest).cuda()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                h.distill(s, t, index, 1.0, r)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = h.distill(s, t, index, 1.0, r)
            for i in range(3):
                s.mul_(0.9)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                with torch.cuda.stream(stream):
                    want = h.distill(s, t, index, 1.0, r)
                stream.synchronize()
                assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    finally:
        h.close()


def test_refusals(head):
    import paper_2207_07736_amd as p
    s = torch.zeros((4, 10), device="cuda")
    g = torch.zeros((4, 10), device="cuda")
    t = torch.zeros((4, 3), device="cuda")
    index = torch.zeros((4, 3), device="cuda", dtype=torch.int32)
    loss = torch.zeros(4, device="cuda")

    def refused(**changes):
        a = p.rlsim_distill(p.RLSIM_F32, s.data_ptr(), 4, 10, 10, p.RLSIM_F32, t.data_ptr(), 3, 4, index.data_ptr(), 3, 3, 1.0,
                            None, None, loss.data_ptr(), g.data_ptr(), 10)
        for key, value in changes.items():
            setattr(a, key, value)
        with pytest.raises(p.RlsimError) as e:
            p.rlsim_head_distill(head.h, a)
        assert e.value.code == p.RLSIM_EINVAL and p.rlsim_head_last_error(head.h)

    for changes in (dict(dtype=5), dict(teacher_dtype=-1), dict(logits=None), dict(teacher=None), dict(index=None),
                    dict(logits=s.data_ptr() + 1), dict(teacher=t.data_ptr() + 2), dict(index=index.data_ptr() + 2),
                    dict(index_bytes=2), dict(index_bytes=8, index=index.data_ptr() + 4), dict(rows=0),
                    dict(rows=(1 << 20) + 1), dict(vocab=0), dict(vocab=11), dict(row_stride=9), dict(teacher_stride=2),
                    dict(index_stride=2), dict(grad_stride=9), dict(k=0), dict(k=1025, teacher_stride=1025, index_stride=1025),
                    dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf),
                    dict(rest=loss.data_ptr() + 1), dict(weight=loss.data_ptr() + 2), dict(loss=loss.data_ptr() + 3),
                    dict(grad=g.data_ptr() + 2), dict(loss=None, grad=None), dict(grad=s.data_ptr() + 4),
                    dict(grad=s.data_ptr(), grad_stride=11), dict(grad=s.data_ptr() - 40)):
        refused(**changes)
    with pytest.raises(p.RlsimError):
        p.rlsim_head_distill(None, p.rlsim_distill())
    assert p.lib.rlsim_head_distill(head.h, None) == p.RLSIM_EINVAL
    good = dict(logits=s, teacher=t, index=index)
    for bad in (dict(logits=s.double()), dict(logits=s.t()), dict(logits=s[0]), dict(teacher=t[:3]), dict(teacher=t.double()),
                dict(index=index.float()), dict(index=index[:, :2]), dict(index=index.cpu()), dict(rest=loss[:3]),
                dict(rest=loss.double()), dict(weight=loss.cpu()), dict(grad=g.half()), dict(grad=g[:, :9]),
                dict(grad=g[:1].expand(4, 10))):
        with pytest.raises(ValueError):
            head.distill(**{**good, **bad})
