"""Sampling from rows of logits on the GPU: tokens equal the plain implementation's, whole
numbers on both sides; log-probabilities lie within the derived bound of 64-bit ones."""
import math

import numpy as np
import pytest

import head_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# each side of every change of the kernel's form, ends inside a vector, and long rows
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


def _check(head, logits, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Run on the device and compare every row with the plain implementation.  Settings
    are numbers, or arrays with a value for each row."""
    rows = logits.shape[0]

    def dev(v, dtype):
        return torch.from_numpy(np.asarray(v, dtype=dtype)).cuda() if np.ndim(v) else v

    token, logp = head.sample(logits, torch.from_numpy(u).cuda(), dev(T, np.float32), dev(top_k, np.int32),
                              dev(top_p, np.float32), dev(min_p, np.float32), logp=True)
    l, token, logp = logits.float().cpu().numpy(), token.cpu().numpy(), logp.cpu().numpy()
    pick = lambda v, r: v[r] if np.ndim(v) else v  # noqa: E731
    for r in range(rows):
        want, lp = ref.sample_row(l[r], u[r], pick(T, r), int(pick(top_k, r)), pick(top_p, r), pick(min_p, r))
        assert token[r] == want, (r, token[r], want)
        if want < 0 or lp == 0.0:
            assert logp[r] == 0.0
            continue
        clean = l[r][~np.isnan(l[r])]
        x = 0.0 if l[r][want] == clean.max() else (float(l[r][want]) - float(clean.max())) / float(pick(T, r))
        assert abs(logp[r] - lp) <= ref.logp_tolerance(lp, x), (r, logp[r], lp)
    return token, logp


def _rows(rng, rows, V, scale=2.2):
    return (rng.standard_normal((rows, V)) * scale * rng.uniform(0.1, 2.0, (rows, 1))).astype(np.float32)


def _u(rng, rows):
    return (rng.integers(0, 1 << 24, rows) / 2.0 ** 24).astype(np.float32)


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_filter_at_every_size(head, V, dtype):
    rng = np.random.default_rng(V)
    rows = 8 if V < 5000 else 3
    for settings in (dict(), dict(T=0.6), dict(top_k=min(V, 40)), dict(top_p=0.9), dict(min_p=0.05),
                     dict(T=1.4, top_k=300, top_p=0.7, min_p=0.001)):
        logits = torch.from_numpy(_rows(rng, rows, V)).cuda().to(DTYPES[dtype])
        _check(head, logits, _u(rng, rows), **settings)


@pytest.mark.parametrize("V", (2, 7, 64, 300, 3000, 40000))
def test_settings_of_its_own_for_each_row(head, V):
    rng = np.random.default_rng(V + 1)
    rows = 70 if V < 1000 else 24
    T = rng.uniform(0.2, 2.0, rows)
    T[:6] = (0.0, -1.0, np.nan, np.inf, 1e-42, 1e30)
    k = rng.integers(-2, min(V, 400) + 5, rows)
    p = rng.uniform(0.0, 1.2, rows)
    p[6:9] = (0.0, -0.5, np.nan)
    m = np.where(rng.random(rows) < 0.5, rng.uniform(0, 0.3, rows), 0.0)
    m[9:13] = (np.nan, -1.0, 1.0, 7.0)
    logits = torch.from_numpy(_rows(rng, rows, V)).cuda()
    _check(head, logits, _u(rng, rows), T.astype(np.float32), k, p.astype(np.float32), m.astype(np.float32))


@pytest.mark.parametrize("V", (3, 64, 130, 1500, 9000, 70000))
@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_infinite_and_equal_entries(head, V, dtype):
    """Rows with nothing left, with one entry left, of equal entries, with NaN, +inf and
    the type's lowest value in masked places, and of +0 and -0."""
    rng = np.random.default_rng(V + 2)
    x = _rows(rng, 12, V)
    low = float(torch.finfo(DTYPES[dtype]).min)
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = -np.inf
    x[2, V // 2] = -3.0
    x[3] = 1.5
    x[4, ::2] = np.nan
    x[5, V - 1] = np.inf
    x[5, 0] = np.inf
    x[6, V // 3:] = low
    x[7] = low
    x[8] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
    x[9, 1:] = -np.inf
    x[10] = np.round(x[10])
    x[11, 0] = 300.0
    logits = torch.from_numpy(x).cuda().to(DTYPES[dtype])
    for settings in (dict(), dict(T=0.0), dict(top_k=1), dict(top_k=2), dict(top_k=50), dict(top_p=0.5), dict(top_p=0.0),
                     dict(min_p=0.2), dict(min_p=1.0), dict(top_k=90, top_p=0.8, min_p=0.01), dict(T=1e-30), dict(T=1e30)):
        _check(head, logits, _u(rng, 12), **settings)


@pytest.mark.parametrize("V,flat", ((6000, 0.0), (6000, 0.02), (50000, 0.0), (50000, 0.3), (140000, 0.05)))
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
def test_cuts_among_many_close_entries(head, V, flat, dtype):
    """More entries near the largest than a workgroup can list: cuts in the middle of
    them, and among equal ones."""
    rng = np.random.default_rng(int(V + 100 * flat))
    logits = torch.from_numpy((rng.standard_normal((4, V)) * flat).astype(np.float32)).cuda().to(DTYPES[dtype])
    for settings in (dict(top_p=0.5), dict(top_k=V // 2), dict(top_k=V // 3, top_p=0.9), dict(min_p=0.9), dict(top_p=0.999),
                     dict(top_k=V - 1, min_p=0.5)):
        _check(head, logits, _u(rng, 4), **settings)


@pytest.mark.parametrize("V", (40000, 131072))
def test_fewer_live_entries_than_top_k(head, V):
    """Sharp rows in which fewer than k entries weigh anything, and many lie just past the
    weights' end: all that weigh are kept, whatever the others' number."""
    rng = np.random.default_rng(V + 3)
    x = np.full((6, V), -30.0, np.float32) + rng.uniform(0, 1, (6, V)).astype(np.float32)
    for r, n in enumerate((1, 3, 30, 100, 250, 299)):
        x[r, rng.permutation(V)[:n]] = rng.uniform(-8, 0, n).astype(np.float32)
    for rows in (6, 600):
        logits = torch.from_numpy(np.tile(x, (rows // 6, 1))).cuda()
        u = _u(rng, rows)
        for settings in (dict(top_k=300), dict(top_k=300, top_p=0.0), dict(top_k=300, top_p=0.9), dict(top_k=900, min_p=0.01)):
            got = head.sample(logits, torch.from_numpy(u).cuda(), **settings).cpu().numpy()
            for r in (*range(6), rows - 1):
                assert got[r] == ref.sample_row(x[r % 6], u[r], settings.get("T", 1.0), settings["top_k"],
                                                settings.get("top_p", 1.0), settings.get("min_p", 0.0))[0]


def test_uniform_numbers_at_the_ends(head):
    rng = np.random.default_rng(5)
    u = np.array([0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, np.nan, 0.5, 2.0 ** -25], dtype=np.float32)
    for V in (2, 50, 700, 33000):
        logits = torch.from_numpy(_rows(rng, 8, V)).cuda()
        _check(head, logits, u)
        _check(head, logits, u, top_p=0.9)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_addresses(head, dtype):
    """Rows apart, rows that start at odd elements, and a row count of one."""
    rng = np.random.default_rng(6)
    for V in (2, 63, 1001, 20011):
        wide = torch.from_numpy(_rows(rng, 6, V + 5)).cuda().to(DTYPES[dtype])
        u = _u(rng, 6)
        view = wide[:, 3:3 + V]
        assert not view.is_contiguous()
        got = head.sample(view, torch.from_numpy(u).cuda(), top_p=0.95)
        assert torch.equal(got, head.sample(view.contiguous(), torch.from_numpy(u).cuda(), top_p=0.95))
        _check(head, view, u, top_p=0.95)
        _check(head, wide[2:3, 1:], u[:1])


def test_rows_past_32_bits(head):
    """Row offsets that pass 2^32 bytes, and 2^32 elements."""
    V, stride = 70001, (1 << 31) + 8
    store = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    logits = store.as_strided((3, V), (stride, 1))
    rng = np.random.default_rng(7)
    logits.copy_(torch.from_numpy(_rows(rng, 3, V)).cuda())
    u = _u(rng, 3)
    _check(head, logits, u, top_p=0.9)
    _check(head, store.as_strided((3, 9), (stride, 1)), u)


def test_a_row_does_not_depend_on_its_batch(head):
    rng = np.random.default_rng(8)
    for V in (2, 40, 900, 12000, 90000):
        logits = torch.from_numpy(_rows(rng, 600, V)).cuda().bfloat16()
        u = torch.from_numpy(_u(rng, 600)).cuda()
        for settings in (dict(), dict(top_p=0.9), dict(top_k=20, min_p=0.02)):
            whole = head.sample(logits, u, logp=True, **settings)
            for a, b in ((0, 1), (17, 24), (500, 600)):
                part = head.sample(logits[a:b], u[a:b], logp=True, **settings)
                assert torch.equal(part[0], whole[0][a:b]) and torch.equal(part[1], whole[1][a:b])


def test_frequencies(head):
    """A million draws from one row of two and one of a hundred entries follow its
    probabilities (five standard deviations)."""
    for V in (2, 100):
        n = 1 << 20
        gen = torch.Generator(device="cuda")
        gen.manual_seed(3)
        row = torch.randn(V, generator=gen, device="cuda")
        u = torch.rand(n, generator=gen, device="cuda")
        token = head.sample(row.expand(n, V).contiguous(), u)
        freq = torch.bincount(token, minlength=V).double().cpu() / n
        p = torch.softmax(row.double().cpu(), 0)
        assert torch.all((freq - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n) + 1e-9)


def test_largest_batch_of_two_actions(head):
    """A million rows of two entries: against the probability of the first."""
    n = 1 << 20
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    logits = torch.randn((n, 2), generator=gen, device="cuda")
    u = torch.rand(n, generator=gen, device="cuda")
    token, logp = head.sample(logits, u, logp=True)
    p = torch.softmax(logits.double(), dim=1)
    sure = (p[:, 0] - u).abs() > 1e-6
    assert torch.equal(token[sure], (u >= p[:, 0])[sure].int())
    want = torch.log(p).gather(1, token.long()[:, None])[:, 0]
    assert (logp - want).abs().max() < 1e-5 and sure.float().mean() > 0.9999


def test_own_stream_and_graph():
    """On a stream of its own, and captured: replays follow the inputs of the day."""
    import paper_2207_07736_amd as p
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(9)
    h = p.Head(16, 40000, stream=stream)
    try:
        logits = torch.from_numpy(_rows(rng, 16, 40000)).cuda().bfloat16()
        u = torch.from_numpy(_u(rng, 16)).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            want = h.sample(logits, u, top_p=0.9, top_k=200)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = h.sample(logits, u, top_p=0.9, top_k=200)
        for i in range(4):
            fresh = torch.from_numpy(_u(rng, 16)).cuda() if i else u.clone()
            u.copy_(fresh)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                want = h.sample(logits, u, top_p=0.9, top_k=200)
            stream.synchronize()
            assert torch.equal(out, want)
    finally:
        h.close()


def test_refusals(head):
    import paper_2207_07736_amd as p
    logits = torch.zeros((4, 10), device="cuda")
    u = torch.zeros(4, device="cuda")

    def refused(**changes):
        a = p.rlsim_sample(p.RLSIM_F32, logits.data_ptr(), 4, 10, 10, u.data_ptr(), 1.0, 0, 1.0, 0.0)
        a.token = u.data_ptr()
        for key, value in changes.items():
            setattr(a, key, value)
        with pytest.raises(p.RlsimError) as e:
            p.rlsim_head_sample(head.h, a)
        assert e.value.code == p.RLSIM_EINVAL and p.rlsim_head_last_error(head.h)

    refused(dtype=3)
    refused(dtype=-1)
    refused(logits=None)
    refused(logits=logits.data_ptr() + 2)
    refused(rows=0)
    refused(rows=(1 << 20) + 1)
    refused(vocab=0)
    refused(vocab=(1 << 20) + 1, row_stride=1 << 21)
    refused(row_stride=9)
    refused(row_stride=1 << 41)
    refused(u=None)
    refused(u=u.data_ptr() + 1)
    refused(token=None)
    refused(logp=u.data_ptr() + 2)
    refused(top_k_rows=u.data_ptr() + 1)
    refused(temperature=-1.0)
    refused(temperature=math.inf)
    refused(temperature=math.nan)
    refused(top_p=math.nan)
    refused(top_p=-0.1)
    refused(min_p=-0.1)
    refused(min_p=math.nan)
    with pytest.raises(p.RlsimError):
        p.rlsim_head_sample(None, p.rlsim_sample())
    assert p.lib.rlsim_head_sample(head.h, None) == p.RLSIM_EINVAL
    for bad in (dict(logits=logits.double()), dict(logits=logits[0]), dict(logits=logits.t()), dict(logits=logits.cpu()),
                dict(u=u[:3]), dict(u=u.double()), dict(u=u.cpu()), dict(u=None), dict(temperature=u[:2]),
                dict(top_k=torch.zeros(4, device="cuda")), dict(top_k=-1), dict(logits=logits[:1].expand(4, 10))):
        with pytest.raises(ValueError):
            head.sample(**{**dict(logits=logits, u=u), **bad})
