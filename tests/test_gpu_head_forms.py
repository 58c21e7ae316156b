"""Forms of the output head's kernels that calls of few rows do not reach: long rows with a
workgroup each (more rows than are shared among workgroups), losses or gradients alone, and
the same rows in batches of other sizes."""
import math

import numpy as np
import pytest

import head_reference as ref
from test_gpu_head_distill import BITS, DTYPES, _case, _same
from test_gpu_head_sample import _rows, _u

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROWS = 300                                # 257 and more are not shared
LONG = (16391, 50001)                     # 1,024 threads to a row, and a tail behind its vectors


@pytest.fixture(scope="module")
def head():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2207_07736_amd as p
    h = p.Head(1 << 12, 1 << 18)
    yield h
    h.close()


def _check_sample(head, x, dtype, rng, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """ROWS rows that repeat x's, with u of their own; settings are numbers or have a value for
    each row of x.  Each of x's rows is compared twice, at both ends of the batch."""
    n = len(x)
    logits = torch.from_numpy(x).cuda().to(DTYPES[dtype])
    turn = torch.arange(ROWS, device="cuda") % n
    u = _u(rng, ROWS)

    def dev(v, kind):
        return torch.from_numpy(np.asarray(v, dtype=kind)).cuda()[turn] if np.ndim(v) else v

    token, logp = head.sample(logits[turn], torch.from_numpy(u).cuda(), dev(T, np.float32), dev(top_k, np.int32),
                              dev(top_p, np.float32), dev(min_p, np.float32), logp=True)
    l, token, logp = logits.float().cpu().numpy(), token.cpu().numpy(), logp.cpu().numpy()
    at = lambda v, j: v[j] if np.ndim(v) else v  # noqa: E731
    for r in (*range(n), *range(ROWS - n, ROWS)):
        j = r % n
        want, lp = ref.sample_row(l[j], u[r], at(T, j), int(at(top_k, j)), at(top_p, j), at(min_p, j))
        assert token[r] == want, (r, token[r], want)
        if want < 0 or lp == 0.0:
            assert logp[r] == 0.0
            continue
        most = np.nanmax(l[j])
        above = 0.0 if l[j][want] == most else (float(l[j][want]) - float(most)) / float(at(T, j))
        assert abs(logp[r] - lp) <= ref.logp_tolerance(lp, above), (r, logp[r], lp)


@pytest.mark.parametrize("V", LONG)
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_filter(head, V, dtype):
    rng = np.random.default_rng(V)
    for settings in (dict(), dict(T=0.6), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_p=0.8, min_p=0.02),
                     dict(T=1.4, top_k=300, top_p=0.7, min_p=0.001), dict(T=0.0)):
        _check_sample(head, _rows(rng, 6, V), dtype, rng, **settings)


@pytest.mark.parametrize("V", LONG)
@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_infinite_and_equal_entries(head, V, dtype):
    """Also in the last entries, behind the vectors."""
    rng = np.random.default_rng(V + 1)
    x = _rows(rng, 11, V)
    low = float(torch.finfo(DTYPES[dtype]).min)
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = -np.inf
    x[2, V - 1] = -3.0
    x[3] = 1.5
    x[4, ::2] = np.nan
    x[5, V - 1] = np.inf
    x[5, V // 2] = np.inf
    x[6, V // 3:] = low
    x[7] = low
    x[8, 1:] = -np.inf
    x[9] = np.round(x[9])
    x[10, V - 2] = 300.0
    for settings in (dict(), dict(T=0.0), dict(top_k=1), dict(top_k=50), dict(top_p=0.5), dict(min_p=0.2),
                     dict(top_k=90, top_p=0.8, min_p=0.01), dict(T=1e-30)):
        _check_sample(head, x, dtype, rng, **settings)


@pytest.mark.parametrize("dtype", DTYPES)
def test_settings_of_its_own_for_each_row(head, dtype):
    V = 16391
    rng = np.random.default_rng(3)
    T = rng.uniform(0.2, 2.0, 30)
    T[:6] = (0.0, -1.0, np.nan, np.inf, 1e-42, 1e30)
    k = rng.integers(-2, 400, 30)
    p = rng.uniform(0.0, 1.2, 30)
    p[6:9] = (0.0, -0.5, np.nan)
    m = np.where(rng.random(30) < 0.5, rng.uniform(0, 0.3, 30), 0.0)
    m[9:13] = (np.nan, -1.0, 1.0, 7.0)
    _check_sample(head, _rows(rng, 30, V), dtype, rng, T.astype(np.float32), k, p.astype(np.float32), m.astype(np.float32))


@pytest.mark.parametrize("V,flat", ((16391, 0.0), (16391, 0.02), (50001, 0.3)))
@pytest.mark.parametrize("dtype", DTYPES)
def test_cuts_among_many_close_entries(head, V, flat, dtype):
    rng = np.random.default_rng(int(V + 100 * flat))
    x = (rng.standard_normal((3, V)) * flat).astype(np.float32)
    for settings in (dict(top_p=0.5), dict(top_k=V // 2), dict(top_k=V // 3, top_p=0.9), dict(min_p=0.9), dict(top_p=0.999, min_p=0.5)):
        _check_sample(head, x, dtype, rng, **settings)


def _bounds(s, t, index, rest, tau, dtype, weight=1.0):
    slots = list(zip(index.tolist(), t.tolist()))
    with np.errstate(all="ignore"):
        return (*ref.distill_row(s, slots, tau, rest, weight), *ref.distill_tolerance(s, slots, tau, rest, weight, BITS[DTYPES[dtype]]))


@pytest.mark.parametrize("V,k", ((65, 9), (1500, 20), (5003, 33), (20011, 64), (50001, 20), (131072, 100)))
@pytest.mark.parametrize("dtype", DTYPES)
def test_losses_or_gradients_alone(head, V, k, dtype):
    """Of many rows: within the bounds of 64-bit ones, and a gradient alone is the one that comes
    with the losses."""
    rng = np.random.default_rng(V)
    s, t, index, rest = _case(rng, 5, V, k, dtype)
    rest[3] = -math.inf
    index[3] = -1
    r = torch.from_numpy(rest).cuda()
    turn = torch.arange(ROWS, device="cuda") % 5
    call = (s[turn], t[turn], index[turn], 2.0, r[turn])
    both = head.distill(*call)
    loss = head.distill(*call, grad=False)
    assert torch.equal(head.distill(*call, loss=False), both[1])
    sh, th, ih = s.float().cpu().numpy(), t.float().cpu().numpy(), index.cpu().numpy()
    for j in range(5):
        want, g, loss_bound, grad_bound = _bounds(sh[j], th[j], ih[j], float(rest[j]), 2.0, dtype)
        for row in (j, ROWS - 5 + j):
            for got in (loss, both[0]):
                _same(got[row].cpu().numpy(), want, loss_bound, f"loss {row}")
            _same(both[1][row].float().cpu().numpy(), g, grad_bound, f"gradient {row}")


@pytest.mark.parametrize("V,k", ((2, 2), (40, 5), (900, 20), (12000, 64), (90000, 64)))
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_in_smaller_batches(head, V, k, dtype):
    """1, 7 and 100 rows of 600: bit for bit where rows are not shared in either call, else both
    within the bounds of 64-bit rows, as sums of chunks are rounded at other places."""
    rng = np.random.default_rng(V)
    s, t, index, rest = _case(rng, 600, V, k, dtype)
    r = torch.from_numpy(rest).cuda() if k < V else None
    whole = head.distill(s, t, index, 2.0, r)
    for a, b in ((0, 1), (17, 24), (500, 600)):
        part = head.distill(s[a:b], t[a:b], index[a:b], 2.0, None if r is None else r[a:b])
        if V < 4096:
            assert torch.equal(part[0], whole[0][a:b]) and torch.equal(part[1], whole[1][a:b])
            continue
        for row in (a, b - 1):
            want, g, loss_bound, grad_bound = _bounds(s[row].float().cpu().numpy(), t[row].float().cpu().numpy(),
                                                      index[row].cpu().numpy(), float(rest[row]), 2.0, dtype)
            for loss, grad in ((part[0][row - a], part[1][row - a]), (whole[0][row], whole[1][row])):
                _same(loss.cpu().numpy(), want, loss_bound, f"loss {row}")
                _same(grad.float().cpu().numpy(), g, grad_bound, f"gradient {row}")


@pytest.mark.parametrize("rows", (2, ROWS))
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
def test_the_longest_rows(rows, dtype):
    """2^20 entries, and as many teacher slots as a call takes."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2207_07736_amd as p
    V, k = 1 << 20, 1024
    h = p.Head(ROWS, V)
    try:
        rng = np.random.default_rng(rows)
        s, t, index, rest = _case(rng, 2, V, k, dtype)
        turn = torch.arange(rows, device="cuda") % 2
        loss, grad = h.distill(s[turn], t[turn], index[turn], 2.0, torch.from_numpy(rest).cuda()[turn])
        u = _u(rng, rows)
        tokens = [h.sample(s[turn], torch.from_numpy(u).cuda(), **settings).cpu().numpy()
                  for settings in (dict(), dict(top_p=0.9), dict(top_k=1000, min_p=0.01))]
        sh, th, ih = s.float().cpu().numpy(), t.float().cpu().numpy(), index.cpu().numpy()
        for row in (0, rows - 1):
            j = row % 2
            want, g, loss_bound, grad_bound = _bounds(sh[j], th[j], ih[j], float(rest[j]), 2.0, dtype)
            _same(loss[row].cpu().numpy(), want, loss_bound, f"loss {row}")
            _same(grad[row].float().cpu().numpy(), g, grad_bound, f"gradient {row}")
            for token, settings in zip(tokens, (dict(), dict(top_p=0.9), dict(top_k=1000, min_p=0.01))):
                assert token[row] == ref.sample_row(sh[j], u[row], **settings)[0], settings
    finally:
        h.close()


# more rows than a launch has workgroups (or groups of rows) for: each goes through several
@pytest.mark.parametrize("V,rows", ((2, 1 << 29), (9, 1 << 25), (65, 1 << 21), (2100, 1 << 21)))
def test_more_rows_than_a_launch_has_workgroups(V, rows):
    """The first and the last rows are those of a call of their own."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2207_07736_amd as p
    rows, some = rows + 321, 1000
    h = p.Head(rows, V)
    try:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(V)
        logits = torch.empty((rows, V), dtype=torch.bfloat16, device="cuda").normal_(0.0, 2.0, generator=gen)
        u = torch.rand(rows, generator=gen, device="cuda")
        k = min(V, 3)
        teacher = torch.empty((rows, k), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        index = torch.randint(0, V, (rows, k), dtype=torch.int32, generator=gen, device="cuda")
        rest = torch.zeros(rows, device="cuda")
        for settings in (dict(), dict(top_k=2, top_p=0.8), dict(top_p=0.9)):
            whole = h.sample(logits, u, **settings)
            for a in (0, rows - some):
                assert torch.equal(whole[a:a + some], h.sample(logits[a:a + some], u[a:a + some], **settings))
            del whole
        want = [h.distill(logits[a:a + some], teacher[a:a + some], index[a:a + some], rest=rest[a:a + some]) for a in (0, rows - some)]
        loss, grad = h.distill(logits, teacher, index, rest=rest, grad=logits)
        for a, (one, g) in zip((0, rows - some), want):
            assert torch.equal(loss[a:a + some], one) and torch.equal(grad[a:a + some], g)
    finally:
        h.close()
