"""The learner's operators from their formulas in 64 bits, with bounds of the error that
the kernels' arithmetic can make (torch tensors, any device).

Bounds count roundings: u = 2^-24 for an fp32 operation to nearest, and a half step of the
output's type for its own rounding.  The hardware's exp2 and reciprocal are good to one
unit of the last place (2 u)."""
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def rounded(value, err, dtype):
    """The bound once a value is rounded to dtype."""
    return err + (value.abs() + err) * HALF_STEP[dtype] + SMALLEST[dtype]


def scan(x, gate, state=None, done=None, dy=None, dlast=None):
    """h, last, dx, dgate, dstate (the gradients None without dy and dlast), each as
    (value, bound before the output's rounding)."""
    T, n, d = x.shape
    x64, g = x.double(), gate.double()
    a, take = torch.sigmoid(g), torch.sigmoid(-g)
    # exp2's argument is off by |g| log2(e) u (product) and as much for the constant, its
    # value by 2 u; the sum, the reciprocal after its step, and E r add an u or two each
    gate_err = (2.0 * g.abs() + 8.0) * U
    keep = torch.ones((T, n, 1), dtype=torch.float64, device=x.device)
    if done is not None:
        keep = (done == 0).double()[:, :, None]
    s = torch.zeros((n, d), dtype=torch.float64, device=x.device) if state is None else state.double()
    se = torch.zeros_like(s)
    h, he, into, into_e = [], [], [], []
    for t in range(T):
        into.append(s)
        into_e.append(se)
        parts = (a[t] * s).abs() + (take[t] * x64[t]).abs()
        v = a[t] * s + take[t] * x64[t]
        e = a[t] * se * (1 + 1e-5) + (gate_err[t] + 3.0 * U) * parts
        h.append(v)
        he.append(e)
        s, se = v * keep[t], e * keep[t]
    H, E, I, IE = torch.stack(h), torch.stack(he), torch.stack(into), torch.stack(into_e)
    out = [(H, E), (s, se)]
    if dy is None and dlast is None:
        return out + [None, None, None]
    dy64 = torch.zeros_like(x64) if dy is None else dy.double()
    r = torch.zeros((n, d), dtype=torch.float64, device=x.device) if dlast is None else dlast.double()
    re = torch.zeros_like(r)
    dx, dg = [None] * T, [None] * T
    for t in reversed(range(T)):
        e = dy64[t] + keep[t] * r
        ee = keep[t] * re + 2.0 * U * (dy64[t].abs() + (keep[t] * r).abs())
        w = a[t] * take[t]
        dx[t] = (take[t] * e, take[t] * (ee * (1 + 1e-5) + (gate_err[t] + 2.0 * U) * e.abs()))
        diff = I[t] - x64[t]
        diff_err = IE[t] + U * (I[t].abs() + x64[t].abs())
        dg[t] = (w * diff * e, w * ((2.0 * gate_err[t] + 6.0 * U) * (diff * e).abs() + 1.00001 * (diff_err * e.abs() + ee * (diff.abs() + diff_err))))
        r, re = a[t] * e, a[t] * (ee * (1 + 1e-5) + (gate_err[t] + 2.0 * U) * e.abs())
    stack = lambda p: tuple(torch.stack(q) for q in zip(*p))  # noqa: E731
    return out + [stack(dx), stack(dg), (r, re)]


def xent(hidden, matrix, target, weight=None, grad=True):
    """loss, dhidden, dmatrix, each as (value, bound before the output's rounding)."""
    dtype = hidden.dtype
    X, W = hidden.double(), matrix.double()
    rows, dim = X.shape
    V = W.shape[0]
    counts = (target.long() >= 0) & (target.long() < V)
    t = torch.where(counts, target.long(), 0)[:, None]
    X = torch.where(counts[:, None], X, 0.0)
    z = X @ W.t()
    # Sums of dim products, each step off by at most 2 u of what the sum of absolutes can
    # reach (the matrix units may truncate).  fp32 factors are scaled to below 2^15 by row and
    # cut into two fp16 parts: each is off by 2^-11 of the 2^-11 that the first leaves, 4 u of
    # itself, or by 2^-25 where that part is small, 2^-39 of the row's largest entry (which
    # is 2^14 at least); the product of both second parts, another 4 u, is left out; three sums.
    full = dtype == torch.float32
    steps = (-(-dim // 32) * 32) * (3 if full else 1)
    reach = X.abs() @ W.abs().t()
    ze = reach * (steps * 2.0 * U + 8.0 * U)
    xtop, wtop = X.abs().max(dim=1, keepdim=True).values, W.abs().max(dim=1, keepdim=True).values
    if full:
        ze = ze + reach * 12.1 * U + 2.0 ** -38 * (xtop * W.abs().sum(dim=1)[None] + X.abs().sum(dim=1)[:, None] * wtop.t())
    m = z.max(dim=1, keepdim=True).values
    s = torch.exp(z - m).sum(dim=1, keepdim=True)
    loss = (torch.log(s) + m - z.gather(1, t))[:, 0]
    # a logit's error moves the loss by itself; exponentials (3 u and their argument's), the
    # sum of V of them in fp32, the logarithm, and the differences' roundings
    sums = (V / 16 + 64) * U
    largest = ze.max(dim=1).values
    exp_err = 4.0 * U + (z - m).abs().clamp(max=110.0) * 2.0 * U
    loss_err = 2.0 * largest + sums + (exp_err * torch.exp(z - m)).sum(dim=1) / s[:, 0] + 8.0 * U * (1.0 + loss.abs() + m[:, 0].abs() + z.abs().max(dim=1).values)
    # Of a row whose largest logit is its target's, by more than errors can hide, the loss is
    # log1p of the others' sum: off by the share that this sum is.
    miss = torch.exp(z - m).scatter(1, t, 0.0).sum(dim=1) / s[:, 0]
    others = z.scatter(1, t, -float("inf")).max(dim=1).values
    share = 2.02 * largest + sums + 232.0 * U             # exponentials: 4 u and 110 x 2 u at most
    own = z.gather(1, t)[:, 0]
    knows = own - others > 4.0 * largest
    loss = torch.where(knows, -torch.log1p(-miss), loss)
    loss_err = torch.where(knows, loss * (share + 8.0 * U), loss_err)
    loss = torch.where(counts, loss, 0.0)
    loss_err = torch.where(counts, loss_err, 0.0)
    if not grad:
        return (loss, loss_err), None, None
    w = torch.ones(rows, dtype=torch.float64, device=X.device) if weight is None else weight.double()
    live = counts & (w != 0)
    w = torch.where(live, w, 0.0)[:, None]
    p = torch.exp(z - m) / s
    dz = p.scatter(1, t, -miss[:, None])
    dz = torch.where(live[:, None], dz, 0.0)
    pe = p * (exp_err + 2.0 * largest[:, None] + ze + sums + 8.0 * U)
    # the target's: the others' share of the sum, three roundings and what moves the ratio
    pe = pe.scatter(1, t, (miss * (torch.exp(own - m[:, 0]) / s[:, 0] * share + 4.0 * U))[:, None])
    # the hardware's exp2 gives 0 below the smallest normal number, 2^-126, and so may the
    # matrix units take a factor below it: what is smaller is off by no more than that, twice
    tiny = 2.0 ** -125
    pe = pe + tiny
    half = 4.0 * U if full else HALF_STEP[dtype]
    # fp16: dz is held times 2^13 at least (of the largest weight), its denormals off by 2^-25
    floor = 2.0 ** -38 if dtype == torch.float16 else 0.0
    dze = torch.where(live[:, None], pe + dz.abs() * half + floor, 0.0)
    many = 3 if full else 1
    over_v = (-(-V // 32) * 32 * many + 80) * 2.0 * U
    over_n = (-(-rows // 32) * 32 * many + 80) * 2.0 * U
    xfloor = wfloor = 0.0
    if full:
        # the other factor's cut, the part left out, and its small parts; dz's small parts: it is held
        # times what its partner was divided by, below 2^14 over all, so off by 2^-39 of the largest
        # such, and its partner is below 2^15 then
        over_v, over_n = over_v + 8.1 * U, over_n + 8.1 * U
        tops = wtop.clamp(min=1e-300)
        xfloor = w.abs() * 2.0 ** -38 * ((dz.abs() @ wtop) + (W.abs() / tops).sum(dim=0)[None] * wtop.max())
    half_w = half
    if dtype != torch.float16:
        # for dmatrix bf16 goes by fp16 too, hidden's rows divided by powers of two (exactly, but for
        # what is small): the same small parts
        half_w = 4.0 * U if full else HALF_STEP[torch.float16]
        xt = xtop.clamp(min=1e-300)
        most = (w.abs() * xtop).max() * 2.0
        wfloor = 2.0 ** -38 * ((w * dz).abs().t() @ xtop + (X.abs() / xt * live[:, None]).sum(dim=0)[None] * most)
    dX = w * (dz @ W)
    dXe = w.abs() * (dze @ W.abs() + over_v * (dz.abs() @ W.abs())) * 1.001 + xfloor
    wd = w * dz
    scale = w.abs().max() * 2.0
    wde = w.abs() * (pe + dz.abs() * (half_w + 2.0 * U)) + ((floor * scale if floor else 0.0) + tiny) * live[:, None]
    dW = wd.t() @ X
    dWe = (wde.t() @ X.abs() + over_n * (wd.abs().t() @ X.abs())) * 1.001 + wfloor
    return (loss, loss_err), (dX, dXe), (dW, dWe)


def close(got, want, bound, what=""):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs() - bound
    assert not torch.isnan(off).any(), f"{what}: NaN"
    worst = int(off.reshape(-1).argmax()) if off.numel() else 0
    assert off.numel() == 0 or float(off.max()) <= 0.0, (what, worst, float(got.reshape(-1)[worst]), float(want.reshape(-1)[worst]),
                                                         float(bound.expand_as(want).reshape(-1)[worst]))
