"""Distilling rows that one entry dominates on the GPU: loss and gradient lie within bounds
that fp32 statistics would miss (head_sharp.py), in every form for rows of more than 64
entries; of shorter rows, whose gradients have fp32 factors, the losses do."""
import numpy as np
import pytest

import head_sharp as sharp

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DTYPES = {"f32": (torch.float32, 24), "bf16": (torch.bfloat16, 8), "f16": (torch.float16, 11)}
ADDS = 66                                 # the longest thread's: 131,072 fp32 entries on 512 threads


@pytest.fixture(scope="module")
def head():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2207_07736_amd as p
    h = p.Head(1024, 1 << 18)
    yield h
    h.close()


@pytest.mark.parametrize("rows", (6, 700))
@pytest.mark.parametrize("V,k,tau", ((70, 5, 1.0), (700, 9, 1.0), (2500, 20, 0.7), (5003, 33, 2.0), (20011, 64, 0.7), (70001, 9, 1.3),
                                     (131072, 100, 2.0)))
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_student_near_a_sharp_teacher(head, dtype, V, k, tau, rows):
    kind, bits = DTYPES[dtype]
    rng = np.random.default_rng(V)
    s, t, top, rest = sharp.case(rng, 6, V, k, tau)
    dev = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    s, t, top, rest = dev(s).to(kind), dev(t).to(kind), dev(top), dev(rest)
    weight = dev(rng.uniform(0.5, 3.0, 6).astype(np.float32))
    turn = torch.arange(rows, device="cuda") % 6
    loss, grad = head.distill(s[turn], t[turn], top[turn], tau, rest[turn], weight[turn])
    tau = float(np.float32(tau))
    pick = sorted({*range(6), rows - 1, rows // 2})
    loss, grad = loss[pick].cpu().numpy(), grad[pick].float().cpu().numpy()
    s, t, top, rest, weight = (v.cpu().numpy() for v in (s.float(), t.float(), top, rest, weight))
    for at, r in enumerate(pick):
        j = r % 6
        want, g, loss_bound, grad_bound = sharp.bounds(s[j], t[j], top[j], tau, float(rest[j]), float(weight[j]), bits, ADDS)
        assert abs(float(loss[at]) - want) <= loss_bound, (r, float(loss[at]), want, loss_bound)
        off = np.abs(grad[at] - g) - grad_bound
        assert off.max() <= 0, (r, int(off.argmax()), grad[at][off.argmax()], g[off.argmax()], grad_bound[off.argmax()])


@pytest.mark.parametrize("rows", (24, 700))
@pytest.mark.parametrize("V,tau", ((70, 1.0), (700, 1.0), (2500, 0.7), (5003, 2.0), (20011, 0.7), (70001, 1.3), (131072, 2.0)))
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_rest_near_the_students(head, dtype, V, tau, rows):
    kind, bits = DTYPES[dtype]
    rng = np.random.default_rng(V + 1)
    s, t, top, rest = sharp.even_case(rng, 24, V, tau, lambda v: torch.from_numpy(v).to(kind).float().numpy())
    dev = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    weight = dev(rng.uniform(0.5, 3.0, 24).astype(np.float32))
    turn = torch.arange(rows, device="cuda") % 24
    loss, grad = head.distill(dev(s).to(kind)[turn], dev(t).to(kind)[turn], dev(top)[turn], tau, dev(rest)[turn], weight[turn])
    tau = float(np.float32(tau))
    loss, grad, weight = loss.cpu().numpy(), grad[:24].float().cpu().numpy(), weight.cpu().numpy()
    for r in range(24):
        want, g, loss_bound, grad_bound = sharp.even_bounds(s[r], t[r], top[r], tau, float(rest[r]), float(weight[r]), bits)
        assert abs(float(loss[r]) - want) <= loss_bound, (r, float(loss[r]), want, loss_bound)
        off = np.abs(grad[r] - g) - grad_bound
        assert off.max() <= 0, (r, int(off.argmax()), grad[r][off.argmax()], g[off.argmax()], grad_bound[off.argmax()])


@pytest.mark.parametrize("rows", (24, 3000))
@pytest.mark.parametrize("V,k,tau", ((2, 1, 1.0), (2, 2, 2.0), (4, 2, 1.0), (4, 4, 0.7), (8, 3, 2.0), (8, 8, 1.0), (13, 5, 1.0), (16, 16, 2.0),
                                     (30, 8, 0.7), (55, 14, 1.0), (64, 64, 2.0)))
def test_losses_of_short_rows(head, V, k, tau, rows):
    import paper_2207_07736_amd as p
    rng = np.random.default_rng(V + k)
    s, t, top, rest = sharp.case(rng, 24, V, k, tau)
    dev = lambda v: None if v is None else torch.from_numpy(v).cuda()[torch.arange(rows, device="cuda") % 24]  # noqa: E731
    h = p.Head(rows, V)
    try:
        loss = h.distill(dev(s), dev(t), dev(top), tau, dev(rest), grad=False)[:24].cpu().numpy()
    finally:
        h.close()
    tau = float(np.float32(tau))
    for r in range(24):
        want, _, bound, _ = sharp.bounds(s[r], t[r], top[r], tau, None if rest is None else float(rest[r]), 1.0, 24, 8)
        assert abs(float(loss[r]) - want) <= bound, (r, float(loss[r]), want, bound)
