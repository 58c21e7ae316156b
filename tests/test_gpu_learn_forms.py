"""Forms of the learner's kernels that only large or far-apart arrays reach
(tests/test_learn_forms.py holds the sizes to them), against the formulas in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import learn_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = (torch.float32, torch.bfloat16, torch.float16)


# ---- the recurrence, sequences more than 2^32 bytes apart ----------------------------

def _far(T, d, dtype):
    """[T, 2, d] in an array whose second sequence begins past 2^32 bytes."""
    step, seq = d + 3, (1 << 32) // torch.empty(0, dtype=dtype).element_size() + 64
    base = torch.empty(seq + T * step, dtype=dtype, device="cuda")
    return base.as_strided((T, 2, d), (step, seq, 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (1, 33, 64))
@pytest.mark.parametrize("T", (1, 40, 130))
def test_sequences_far_apart(T, d, dtype):
    import paper_2207_07736_amd as rl
    g = torch.Generator(device="cuda").manual_seed(T + d)
    near = [torch.randn((T, 2, d), generator=g, device="cuda").to(dtype) for _ in range(3)]
    x, gate, dy = (_far(T, d, dtype).copy_(t) for t in near)
    y, dx, dgate = (_far(T, d, dtype) for _ in range(3))
    state, dlast = (torch.randn((2, d), generator=g, device="cuda") for _ in range(2))
    ends = (torch.rand((T, 2), generator=g, device="cuda") < 0.05).to(torch.uint8)
    last, dstate = torch.empty_like(state), torch.empty_like(state)
    marks = torch.empty((-(-T // 16), 2, d), device="cuda")
    kind = {torch.float32: rl.RLSIM_F32, torch.bfloat16: rl.RLSIM_BF16, torch.float16: rl.RLSIM_F16}[dtype]
    h = rl.rlsim_learner_create()
    try:
        args = rl.rlsim_scan(kind, T, 2, d, x.data_ptr(), gate.data_ptr(), *x.stride()[:2], *gate.stride()[:2], state.data_ptr(),
                             ends.data_ptr(), marks.data_ptr(), y.data_ptr(), *y.stride()[:2], last.data_ptr())
        rl.rlsim_learner_scan(h, args)
        rl.rlsim_learner_scan_grad(h, args, rl.rlsim_scan_grad(dy.data_ptr(), *dy.stride()[:2], dlast.data_ptr(), dx.data_ptr(),
                                                               dgate.data_ptr(), *dx.stride()[:2], *dgate.stride()[:2], dstate.data_ptr()))
        torch.cuda.synchronize()
    finally:
        rl.rlsim_learner_destroy(h)
    want = ref.scan(near[0], near[1], state, ends, near[2], dlast)
    for name, got, w in (("y", y, want[0]), ("dx", dx, want[2]), ("dgate", dgate, want[3])):
        ref.close(got, w[0], ref.rounded(*w, dtype), name)
    ref.close(last, *want[1], "last")
    ref.close(dstate, *want[4], "dstate")


def test_far_rows_through_the_binding():
    """The same bits as those of rows side by side."""
    import paper_2207_07736_amd as rl
    learner = rl.Learner()
    g = torch.Generator(device="cuda").manual_seed(0)
    near = [torch.randn((130, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(3)]
    x, gate, dy = (_far(130, 64, torch.bfloat16).copy_(t) for t in near)
    for rows in ((near[0], near[1], near[2]), (x, gate, dy)):
        y, last, marks = learner.scan(rows[0], rows[1], marks=True)
        made = y, last, marks, *learner.scan_grad(rows[0], rows[1], marks, rows[2])
        if rows[0] is x:
            assert all(torch.equal(a, b) for a, b in zip(made, kept))
        kept = made
    learner.close()


# ---- the output layer in tiles of 256 x 256 -------------------------------------------

@pytest.mark.parametrize("dtype,rows,vocab", [(torch.bfloat16, 4096, 8492), (torch.float16, 4096, 8492), (torch.float32, 4096, 4600),
                                              (torch.float32, 1024, 4600)])
def test_large_tiles_and_two_pieces(dtype, rows, vocab):
    import paper_2207_07736_amd as rl
    g = torch.Generator(device="cuda").manual_seed(7)
    matrix = (torch.randn((vocab, 4096), generator=g, device="cuda") / 32).to(dtype)
    hidden = torch.randn((rows, 4096), generator=g, device="cuda").to(dtype)
    target = torch.randint(-1, vocab, (rows,), generator=g, device="cuda")
    weight = torch.randn(rows, generator=g, device="cuda")
    learner = rl.Learner(rows, 4096, vocab)
    try:
        made = learner.cross_entropy(hidden, matrix, target, weight)
        again = learner.cross_entropy(hidden, matrix, target, weight)
        assert all(torch.equal(a, b) for a, b in zip(made, again))
    finally:
        learner.close()
    loss, x, w = ref.xent(hidden, matrix, target, weight)
    ref.close(made[0], loss[0], loss[1] + 2.0 ** -24 * loss[0].abs(), "loss")
    ref.close(made[1], x[0], ref.rounded(*x, dtype), "dhidden")
    ref.close(made[2], w[0], ref.rounded(*w, dtype), "dmatrix")
    # an entry of the last piece, a target of the first one's: both pieces are in dhidden
    assert (target >= vocab - 200).any() and (target < 256).any()


def test_as_many_rows_as_a_handle_takes():
    import paper_2207_07736_amd as rl
    rows, dim, vocab = 1 << 22, 8, 2
    g = torch.Generator(device="cuda").manual_seed(8)
    matrix = torch.randn((vocab, dim), generator=g, device="cuda").bfloat16()
    hidden = torch.randn((rows, dim), generator=g, device="cuda").bfloat16()
    target = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.uint8)
    learner = rl.Learner(rows, dim, vocab)
    try:
        made = learner.cross_entropy(hidden, matrix, target)
    finally:
        learner.close()
    loss, x, w = ref.xent(hidden, matrix, target)
    ref.close(made[0], loss[0], loss[1] + 2.0 ** -24 * loss[0].abs(), "loss")
    ref.close(made[1], x[0], ref.rounded(*x, torch.bfloat16), "dhidden")
    # the reference's bound is of one sum over all rows; 64 workgroups share it, each off by 2 u a
    # row of what its absolutes reach, and dz is off by half a step of fp16
    X, t = hidden.double(), target.long()[:, None]
    p = torch.softmax(X @ matrix.double().t(), dim=1)
    dz = p.scatter_add(1, t, torch.full_like(t, -1, dtype=torch.float64))
    reach = dz.abs().t() @ X.abs()
    assert rows // 64 * 2 * ref.U < 2.0 ** -6
    ref.close(made[2], w[0], ref.rounded(w[0], reach * ((rows // 64 + 64 + 80) * 2.0 * ref.U + 2.0 ** -11 + 2.0 ** -16), torch.bfloat16), "dmatrix")


# ---- clipping ---------------------------------------------------------------------------

@pytest.mark.parametrize("to", (None, torch.float32, torch.bfloat16))
@pytest.mark.parametrize("dtype", TYPES)
def test_more_bytes_than_the_cache_holds(dtype, to):
    """Stores past the cache, in place too."""
    import paper_2207_07736_amd as rl
    g = torch.Generator(device="cuda").manual_seed(9)
    tensors = [torch.randn(k, generator=g, device="cuda").to(dtype) for k in (150000001, 5, 1000003)]
    before = [t.clone() for t in tensors]
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))
    out = None if to is None else [torch.empty_like(t, dtype=to) for t in tensors]
    learner = rl.Learner()
    norm = float(learner.clip(tensors, 3.0, out=out))
    learner.close()
    assert abs(norm - want) <= want * (2.0 ** -24 + 2.0 ** -30)
    for b, t in zip(before, out or tensors):
        value = b.double() * (3.0 / want)
        ref.close(t, value, ref.rounded(value, value.abs() * 2.5 * ref.U, t.dtype))


def test_none_is_skipped():
    import paper_2207_07736_amd as rl
    learner = rl.Learner()
    a = torch.randn((30, 40), device="cuda").t()
    b = torch.randn(70000, device="cuda")
    before = [a.double().clone(), b.double().clone()]
    want = math.sqrt(sum(float((t ** 2).sum()) for t in before))
    for tensors, out in (([None, a, None, b], None), ([a, None, b], [torch.empty_like(a), None, torch.empty_like(b)])):
        a.copy_(before[0])
        b.copy_(before[1])
        norm = float(learner.clip(tensors, 0.5, out=out))
        assert abs(norm - want) <= want * (2.0 ** -24 + 2.0 ** -30)
        for t, w in zip([t for t in out or tensors if t is not None], before):
            value = w * (0.5 / want)
            ref.close(t, value, ref.rounded(value, value.abs() * 2.5 * ref.U, torch.float32))
        if out:
            assert torch.equal(a.double(), before[0]) and torch.equal(b.double(), before[1])
    learner.close()
