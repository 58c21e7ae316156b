"""The output layer's cross entropy on the GPU against its formula in 64 bits."""
import pytest

torch = pytest.importorskip("torch")

import learn_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = (torch.float32, torch.bfloat16, torch.float16)


@pytest.fixture(scope="module")
def learner():
    import paper_2207_07736_amd as rl
    made = rl.Learner(2100, 1100, 20000)
    yield made
    made.close()


def _inputs(rows, dim, V, dtype, seed=0, sharp=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    matrix = (torch.randn((V, dim), generator=g, device="cuda") * sharp / dim ** 0.5).to(dtype)
    hidden = torch.randn((rows, dim), generator=g, device="cuda").to(dtype)
    target = torch.randint(0, V, (rows,), generator=g, device="cuda")
    target[torch.rand(rows, generator=g, device="cuda") < 0.1] = -1
    weight = torch.randn(rows, generator=g, device="cuda")
    return hidden, matrix, target, weight


def _check(learner, hidden, matrix, target, weight=None):
    dtype = hidden.dtype
    loss, dhidden, dmatrix = learner.cross_entropy(hidden, matrix, target, weight)
    l, x, w = ref.xent(hidden, matrix, target, weight)
    ref.close(loss, l[0], l[1] + 2.0 ** -24 * l[0].abs(), "loss")
    ref.close(dhidden, x[0], ref.rounded(*x, dtype), "dhidden")
    ref.close(dmatrix, w[0], ref.rounded(*w, dtype), "dmatrix")
    return loss, dhidden, dmatrix


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,V", [(1, 1, 1), (1, 64, 2), (3, 5, 7), (7, 64, 300), (17, 100, 1000), (33, 33, 257), (40, 8, 300), (300, 40, 520),
                                        (32, 128, 129), (64, 192, 64), (130, 65, 515), (257, 320, 777), (1000, 16, 2)])
def test_sizes(learner, rows, dim, V, dtype):
    _check(learner, *_inputs(rows, dim, V, dtype, seed=rows + V))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,V", [(2049, 1024, 8200), (2000, 1001, 20000), (5, 1024, 20000), (700, 1000, 9001)])
def test_larger(learner, rows, dim, V, dtype):
    _check(learner, *_inputs(rows, dim, V, dtype, seed=1))


@pytest.mark.parametrize("dtype", TYPES)
def test_pieces_of_the_vocabulary(dtype):
    """Rows enough for several pieces, the last one of a few entries."""
    import paper_2207_07736_amd as rl
    rows, dim, V = (20000, 64, 3 * 1024 + 5) if dtype == torch.float32 else (30000, 64, 2 * 2048 + 130)
    learner = rl.Learner(rows, dim, V)
    try:
        _check(learner, *_inputs(rows, dim, V, dtype, seed=2))
    finally:
        learner.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("target_type", (torch.uint8, torch.int32, torch.int64))
def test_target_types(learner, target_type, dtype):
    hidden, matrix, target, weight = _inputs(100, 64, 256, dtype)
    if target_type == torch.uint8:
        matrix, target = matrix[:200], target.clamp(min=0)      # 200 .. 255 are outside
    assert target_type == torch.uint8 or (target < 0).any()
    _check(learner, hidden, matrix, target.to(target_type), weight)


@pytest.mark.parametrize("dtype", TYPES)
def test_two_actions_and_many_rows(dtype):
    """A control policy's output layer: more rows than one workgroup weighs."""
    import paper_2207_07736_amd as rl
    learner = rl.Learner(100003, 24, 2)
    try:
        _check(learner, *_inputs(100003, 24, 2, dtype, seed=9))
    finally:
        learner.close()


@pytest.mark.parametrize("scale", (2.0 ** -60, 2.0 ** 60))
def test_fp32_rows_of_any_size(learner, scale):
    """Rows, entries of the vocabulary and weights that differ by powers of two up to 2^120."""
    hidden, matrix, target, weight = _inputs(70, 96, 600, torch.float32)
    by_row = torch.exp2((torch.arange(70, device="cuda") % 9 - 4.0) * 3.0)
    by_entry = torch.exp2(-(torch.arange(600, device="cuda") % 7) * 2.0)
    hidden, matrix = hidden * by_row[:, None] * scale, matrix * by_entry[:, None] / scale
    hidden[3], matrix[11] = 0.0, 0.0
    _check(learner, hidden, matrix, target, weight * torch.exp2((torch.arange(70, device="cuda") % 5) * 6.0 - 12.0))


def test_a_workspace_too_large():
    import paper_2207_07736_amd as rl
    with pytest.raises(rl.RlsimError) as e:
        rl.Learner(1 << 22, 1 << 16, 1 << 20)
    assert e.value.code == rl.RLSIM_ENOMEM
    made = rl.Learner(4, 4, 4)
    x = torch.zeros((4, 4), device="cuda")
    assert float(made.cross_entropy(x, x, torch.zeros(4, dtype=torch.int32, device="cuda"), grad=False)[0]) == pytest.approx(1.386294, abs=1e-6)
    made.close()


def test_targets_outside(learner):
    hidden, matrix, target, _ = _inputs(8, 64, 100, torch.bfloat16)
    target[:] = torch.tensor([0, 99, 100, -1, -100, 2 ** 40, -2 ** 62, 50])
    loss, dhidden, _ = _check(learner, hidden, matrix, target)
    assert not loss[2:7].any() and not dhidden[2:7].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_wider_arrays(learner, dtype):
    hidden, matrix, target, weight = _inputs(90, 64, 300, dtype)
    for pad, off in ((8, 0), (8, 8), (3, 1)):
        wide_h = torch.zeros((90, 64 + pad + off), device="cuda", dtype=dtype)
        wide_m = torch.zeros((300, 64 + pad + off), device="cuda", dtype=dtype)
        wide_h[:, off:off + 64], wide_m[:, off:off + 64] = hidden, matrix
        _check(learner, wide_h[:, off:off + 64], wide_m[:, off:off + 64], target, weight)


@pytest.mark.parametrize("dtype", TYPES)
def test_sharp_rows(learner, dtype):
    """Logits of some hundreds: a softmax that is one entry, right or wrong."""
    hidden, matrix, target, weight = _inputs(70, 64, 500, dtype, sharp=60.0)
    z = hidden.double() @ matrix.double().t()
    target[:35] = z[:35].argmax(dim=1)
    loss, _, _ = _check(learner, hidden, matrix, target, weight)
    assert (loss[35:][target[35:] >= 0] > 50).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_know_their_target(learner, dtype):
    """Losses from 1e-2 to 1e-30: neither they nor the gradients are differences from 1."""
    g = torch.Generator(device="cuda").manual_seed(6)
    matrix = torch.zeros((300, 64), device="cuda")
    matrix[:, :60] = torch.randn((300, 60), generator=g, device="cuda") / 8
    hidden = torch.randn((40, 64), generator=g, device="cuda")
    target = torch.full((40,), 17, device="cuda")
    matrix[17, 60] = 1.0                                       # the target's lead, from row to row
    hidden[:, 60] = torch.linspace(12.0, 75.0, 40, device="cuda")
    hidden, matrix = hidden.to(dtype), matrix.to(dtype)
    loss, dhidden, dmatrix = _check(learner, hidden, matrix, target)
    assert float(loss.max()) < 1e-1 and 0.0 < float(loss.min()) < 1e-25


def test_fp16_gradients_of_a_flat_softmax(learner):
    """20,000 probabilities of 5e-5 each, and weights from 2^-10 to 2^10."""
    hidden, matrix, target, weight = _inputs(40, 64, 20000, torch.float16, sharp=0.01)
    weight = weight.sign() * torch.exp2(torch.arange(40, device="cuda") % 21 - 10.0)
    _check(learner, hidden, matrix, target, weight)


@pytest.mark.parametrize("dtype", TYPES)
def test_padded_rows_may_hold_anything(learner, dtype):
    hidden, matrix, target, weight = _inputs(60, 64, 400, dtype)
    weight[5] = 0.0
    want = learner.cross_entropy(hidden, matrix, target, weight)
    out = target < 0
    hidden[out] = float("nan")
    got = learner.cross_entropy(hidden, matrix, target, weight)
    hidden[5] = float("inf")
    again = learner.cross_entropy(hidden, matrix, target, weight)
    assert not got[0][out].any() and not got[1][out].any() and not again[1][5].any()
    for a, b, c in zip(want[1:], got[1:], again[1:]):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert torch.equal(want[0], got[0])
    # a NaN in a row that counts is the row's and the matrix's
    live = int(torch.nonzero(~out & (weight != 0))[0])
    hidden[live, 3] = float("nan")
    loss, dhidden, dmatrix = learner.cross_entropy(hidden, matrix, target, weight)
    assert torch.isnan(loss[live]) and torch.isnan(dhidden[live]).all() and torch.isnan(dmatrix[:, :]).all()
    others = ~out & (torch.arange(60, device="cuda") != live) & (weight != 0)
    assert torch.equal(loss[others], want[0][others]) and torch.equal(dhidden[others], want[1][others])


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("rows", (5, 50))
def test_rows_that_end_within_a_step_keep_to_themselves(learner, rows, dtype):
    """Rows of 8 k entries inside wider arrays of NaN, for sums of 1 to 11 steps of 32: nothing
    behind a row's end is used."""
    for dim in range(8, 352, 8):
        hidden, matrix, target, weight = _inputs(rows, dim, 70, dtype, seed=dim)
        wide_h = torch.full((rows, dim + 32), float("nan"), device="cuda", dtype=dtype)
        wide_m = torch.full((70, dim + 32), float("nan"), device="cuda", dtype=dtype)
        wide_h[:, 8:dim + 8], wide_m[:, 8:dim + 8] = hidden, matrix
        want = learner.cross_entropy(hidden, matrix, target, weight)
        for a, b in zip(want, learner.cross_entropy(wide_h[:, 8:dim + 8], wide_m[:, 8:dim + 8], target, weight)):
            assert torch.isfinite(a).all() and torch.equal(a, b), dim


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("rows", (5, 50))
def test_a_vocabulary_that_ends_within_a_step_keeps_to_itself(learner, rows, dtype):
    """The first rows of a longer matrix of NaN, for sums over 1 to 15 steps of 32 entries."""
    for V in range(3, 480, 7):
        hidden, matrix, target, weight = _inputs(rows, 64, V, dtype, seed=V)
        long = torch.full((V + 40, 64), float("nan"), device="cuda", dtype=dtype)
        long[:V] = matrix
        want = learner.cross_entropy(hidden, matrix, target, weight)
        for a, b in zip(want, learner.cross_entropy(hidden, long[:V], target, weight)):
            assert torch.isfinite(a).all() and torch.equal(a, b), V


@pytest.mark.parametrize("rows", (7, 100))
def test_parts_of_a_call(learner, rows):
    """Losses, either gradient or both, at once or from the statistics, are the same bits."""
    hidden, matrix, target, weight = _inputs(rows, 128, 700, torch.bfloat16)
    stats = torch.empty((rows, 3), device="cuda")
    loss, dhidden, dmatrix = learner.cross_entropy(hidden, matrix, target, weight, stats=stats)
    assert torch.equal(learner.cross_entropy(hidden, matrix, target, grad=False), loss)
    assert torch.equal(learner.cross_entropy(hidden, matrix, target, weight, grad="hidden")[1], dhidden)
    assert torch.equal(learner.cross_entropy(hidden, matrix, target, weight, grad="matrix")[1], dmatrix)
    later = learner.cross_entropy(hidden, matrix, target, weight, loss=False, stats=stats)
    assert torch.equal(later[0], dhidden) and torch.equal(later[1], dmatrix)
    assert torch.equal(learner.cross_entropy(hidden, matrix, target, weight, loss=False, grad="matrix", stats=stats), dmatrix)
    z = hidden.double() @ matrix.double().t()
    counts = target >= 0
    torch.testing.assert_close(stats[counts, 0].double(), z.max(dim=1).values[counts], rtol=0, atol=1e-4)
    own = torch.exp(z.gather(1, target.clamp(min=0)[:, None])[:, 0] - z.max(dim=1).values)
    torch.testing.assert_close(stats[counts, 2].double(), own[counts], rtol=1e-3, atol=0)


def test_again_and_again(learner):
    hidden, matrix, target, weight = _inputs(500, 256, 5000, torch.bfloat16)
    first = learner.cross_entropy(hidden, matrix, target, weight)
    for _ in range(5):
        for a, b in zip(first, learner.cross_entropy(hidden, matrix, target, weight)):
            assert torch.equal(a, b)


def test_no_rows_and_only_rows_outside(learner):
    matrix = torch.randn((50, 16), device="cuda")
    loss, dhidden, dmatrix = learner.cross_entropy(matrix[:0], matrix, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert loss.shape == (0,) and dhidden.shape == (0, 16) and dmatrix.shape == (50, 16) and not dmatrix.any()
    loss, dhidden, dmatrix = learner.cross_entropy(matrix, matrix, torch.full((50,), -1, dtype=torch.int32, device="cuda"))
    assert not loss.any() and not dhidden.any() and not dmatrix.any()


def test_refusals(learner):
    import paper_2207_07736_amd as rl
    hidden, matrix, target, weight = _inputs(8, 64, 100, torch.bfloat16)
    for bad, match in ((dict(hidden=hidden.double()), "float32"), (dict(hidden=hidden[:, :63]), "matrix"),
                       (dict(matrix=matrix.float()), "matrix"), (dict(target=target.float()), "target"),
                       (dict(target=target[:5]), "target"), (dict(weight=weight.double()), "weight"),
                       (dict(hidden=hidden.t().contiguous().t()), "consecutive"), (dict(grad="both"), "grad"),
                       (dict(loss=False), "stats"), (dict(loss=False, grad=False), "neither"),
                       (dict(matrix=matrix[0]), "vocab"), (dict(hidden=hidden.cpu()), "on cuda")):
        args = dict(hidden=hidden, matrix=matrix, target=target, weight=weight)
        args.update(bad)
        with pytest.raises(ValueError, match=match):
            learner.cross_entropy(**args)
    many = torch.zeros((2101, 4), device="cuda")
    with pytest.raises(rl.RlsimError, match="rows") as e:
        learner.cross_entropy(many, many[:5], torch.zeros(2101, dtype=torch.int64, device="cuda"))
    assert e.value.code == rl.RLSIM_EINVAL
    none = rl.Learner()
    with pytest.raises(rl.RlsimError, match="without an output layer"):
        none.cross_entropy(hidden, matrix, target)
    none.close()
