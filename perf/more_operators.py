"""Performance cases of a learner's operators: a gated linear recurrence over recorded
rows, the cross entropy of an output layer, and clipping by the gradients' global norm.

A case is a dict of plain values:
  kind      "scan", "xent" or "clip"
  dtype     "f32", "bf16" or "f16"
 scan:
  T, n, d   steps, sequences (environments), channels
  order     "time": rows [T][n][d]; "batch": [n][T][d], seen as [T][n][d]
  done      episodes end within the rows
  grad      the backward pass too
 xent:
  rows, D, V   rows, width of the hidden state, entries of the vocabulary
  weighted  a weight for each row (advantages)
  grad      gradients of the hidden state and the matrix beside the losses
 clip:
  tensors, total   how many gradients, and their elements together
  mixed     every other gradient is fp32, whatever dtype says
  clipped   the norm is above the limit; the clipped gradients go to tensors of
            their own. Otherwise it is below, in place, and nothing changes.

Recurrence: a_t = sigmoid(gate_t), h_t = a_t h'_{t-1} + (1 - a_t) x_t, where h'_t is 0
after a step that ends an episode, and h_t otherwise; h'_{-1} is the state given.
Outputs are the h_t and h'_{T-1}.

Cross entropy: z = hidden matrix^T, loss = log sum exp z - z_target; the gradient is
that of sum(weight * loss). A row whose target is outside the vocabulary has loss 0
and adds nothing to a gradient.

Clipping: norm = sqrt(sum of all squares); where norm > limit (and finite) each gradient
is multiplied by limit / norm.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


def _scan(name, T, n, d, dtype, order="time", done=False, grad=False):
    return dict(name=name, kind="scan", T=T, n=n, d=d, dtype=dtype, order=order, done=done, grad=grad)


def _xent(name, rows, D, V, dtype, weighted=False, grad=True):
    return dict(name=name, kind="xent", rows=rows, D=D, V=V, dtype=dtype, weighted=weighted, grad=grad)


def _clip(name, tensors, total, dtype, mixed=False, clipped=True):
    return dict(name=name, kind="clip", tensors=tensors, total=total, dtype=dtype, mixed=mixed, clipped=clipped)


def listed():
    return [
        # one sequence answers one token: latency
        _scan("step-1x1024", 1, 1, 1024, "bf16"),
        # a recurrent policy acts once in every environment of a mid-size batch
        _scan("step-4096x256", 1, 4096, 256, "f32", done=True),
        # a learner's pass over a recorded rollout of 200 steps, episodes ending in it
        _scan("rollout-200x4096x64", 200, 4096, 64, "f32", done=True, grad=True),
        # ragged sizes, batch-major rows, a sequence model's forward and backward
        _scan("ragged-1023x37x333", 1023, 37, 333, "f16", order="batch", done=True, grad=True),
        # one very long sequence: few channels, so time itself has to be shared out
        _scan("long-65536x2048", 65536, 1, 2048, "bf16", grad=True),
        # a few rows teach a mid-size vocabulary: the matrix and its gradient set the pace
        _xent("few-7x1024x32000", 7, 1024, 32000, "bf16"),
        # fp32 training of a discretised policy from advantages
        _xent("policy-2048x256x4096", 2048, 256, 4096, "f32", weighted=True),
        # validation on odd sizes: the losses alone
        _xent("eval-1023x1000x50001", 1023, 1000, 50001, "f16", grad=False),
        # the largest: a training step's tokens, a wide model, a large vocabulary
        _xent("train-4096x4096x131072", 4096, 4096, 131072, "bf16", weighted=True),
        # the gradients of a small control policy: latency
        _clip("policy-8", 8, 9000, "f32"),
        # a mid-size model in mixed precision, norm within the limit, as in most steps
        _clip("within-61x50M", 61, 50000003, "bf16", mixed=True, clipped=False),
        # a large model's gradients, clipped
        _clip("clip-48x400M", 48, 400000000, "bf16"),
    ]


def _log_int(rng, lo, hi):
    """Log-uniform over [lo, hi]; about one value in four a power of two."""
    if hi <= lo:
        return lo
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    v = 2.0 ** round(math.log2(v)) if rng.random() < 0.25 else v
    return max(lo, min(hi, int(round(v))))


def draw(rng):
    dtype = rng.choice(("f32", "bf16", "f16"))
    kind = rng.choice(("scan", "xent", "clip"))
    if kind == "scan":
        T = 1 if rng.random() < 0.2 else _log_int(rng, 2, 65536)
        d = _log_int(rng, 1, min(4096, (1 << 27) // T))
        n = _log_int(rng, 1, min(65536, (1 << 27) // (T * d)))
        return _scan("", T, n, d, dtype, order=rng.choice(("time", "batch")), done=rng.random() < 0.5,
                     grad=rng.random() < 0.7)
    if kind == "xent":
        V, D = _log_int(rng, 512, 131072), _log_int(rng, 16, 4096)
        most = 1 << (37 if dtype == "f32" else 40)
        return _xent("", _log_int(rng, 1, max(1, min(8192, most // (V * D)))), D, V, dtype,
                     weighted=rng.random() < 0.5, grad=rng.random() < 0.75)
    tensors = rng.randint(1, 60)
    return _clip("", tensors, _log_int(rng, 60 * 16, 200000000), dtype, mixed=rng.random() < 0.3,
                 clipped=rng.random() < 0.6)


def _sizes(case):
    """Elements of each gradient: from large to small, odd ones among them."""
    count, total = case["tensors"], case["total"]
    share = [1.0 / (1 + (5 * i) % count) for i in range(count)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    sizes[0] += max(0, total - sum(sizes))
    return sizes


def _type_of(case, i):
    return torch.float32 if case["mixed"] and i % 2 else DTYPES[case["dtype"]]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=DEVICE)

    state = dict(case=case)
    if case["kind"] == "scan":
        T, n, d = case["T"], case["n"], case["d"]

        def rows(make):
            if case["order"] == "batch":
                return make(n, T, d).transpose(0, 1)
            return make(T, n, d)

        # channels that forget within a few steps and ones that remember for hundreds
        memory = uniform(d) * 6.0 - 1.0
        state["x"] = rows(lambda *s: normal(*s).to(dtype))
        state["gate"] = rows(lambda *s: normal(*s).add_(memory).to(dtype))
        state["state"] = normal(n, d)
        state["done"] = (uniform(T, n) < 1.0 / 64).to(torch.uint8) if case["done"] else None
        state["dy"] = rows(lambda *s: normal(*s).to(dtype)) if case["grad"] else None
    elif case["kind"] == "xent":
        N, D, V = case["rows"], case["D"], case["V"]
        matrix = (normal(V, D) * (2.0 / math.sqrt(D))).to(dtype)
        target = torch.randint(0, V, (N,), generator=gen, device=DEVICE)
        # half of the rows know their target more or less, the others do not
        known = torch.where(uniform(N, 1) < 0.5, 4.0 * uniform(N, 1), 0.0)
        state["hidden"] = (normal(N, D) + known * matrix[target].float()).to(dtype)
        state["matrix"] = matrix
        # rows that only pad the batch
        state["target"] = torch.where((uniform(N) < 0.1) & (torch.arange(N, device=DEVICE) > 0), -1, target)
        state["weight"] = normal(N) if case["weighted"] else None
    else:
        state["grads"] = [(normal(k) * (0.01 * (1.0 + i % 7))).to(_type_of(case, i)) for i, k in enumerate(_sizes(case))]
        state["out"] = [torch.empty_like(g) for g in state["grads"]] if case["clipped"] else None
        about = math.sqrt(sum(k * (0.01 * (1.0 + i % 7)) ** 2 for i, k in enumerate(_sizes(case))))
        state["limit"] = about * (0.3 if case["clipped"] else 2.0)
    if own:
        import paper_2207_07736_amd as rl
        if case["kind"] == "xent":
            state["learner"] = rl.Learner(case["rows"], case["D"], case["V"])
        else:
            state["learner"] = rl.Learner()
    return state


def _running(a, b):
    """h_t = a_t h_{t-1} + b_t over the first dimension (h_{-1} = 0): pairs of
    neighbours joined, then pairs of pairs, and so on."""
    reach = 1
    while reach < a.shape[0]:
        b = torch.cat((b[:reach], b[reach:] + a[reach:] * b[:-reach]))
        a = torch.cat((a[:reach], a[reach:] * a[:-reach]))
        reach *= 2
    return b


def _plain_scan(state):
    case = state["case"]
    dtype = DTYPES[case["dtype"]]
    x, gate = state["x"].float(), state["gate"].float()
    a = 1.0 / (1.0 + torch.exp(-gate))
    take = 1.0 / (1.0 + torch.exp(gate))
    ones = torch.ones((case["T"], case["n"], 1), device=x.device)
    keep = ones if state["done"] is None else (state["done"] == 0)[:, :, None].float()
    # keep of the step before: what reaches step t of the state after step t - 1
    before = torch.cat((ones[:1], keep[:-1]))
    carried = a * before
    b = take * x
    b[0] += a[0] * state["state"]
    h = _running(carried, b)
    last = h[-1] * keep[-1]
    if not case["grad"]:
        return h.to(dtype), last
    dy = state["dy"].float()
    # e_t = dy_t + carried_{t+1} e_{t+1}: the same recurrence from the end
    after = torch.cat((carried[1:], torch.zeros_like(carried[:1])))
    e = _running(after.flip(0), dy.flip(0)).flip(0)
    previous = torch.cat((state["state"][None], h[:-1])) * before
    dx = take * e
    dgate = a * take * (previous - x) * e
    return h.to(dtype), last, dx.to(dtype), dgate.to(dtype), a[0] * e[0]


def _plain_xent(state):
    case = state["case"]
    dtype = DTYPES[case["dtype"]]
    hidden, matrix, target = state["hidden"].float(), state["matrix"].float(), state["target"]
    counts = (target >= 0) & (target < case["V"])
    at = torch.where(counts, target, 0)[:, None]
    z = hidden @ matrix.t()
    z -= z.max(dim=1, keepdim=True).values
    chosen = torch.gather(z, 1, at)
    e = z.exp_()
    total = e.sum(dim=1, keepdim=True)
    loss = torch.where(counts, (torch.log(total) - chosen)[:, 0], 0.0)
    if not case["grad"]:
        return loss
    dz = e.div_(total)
    dz.scatter_add_(1, at, torch.full_like(chosen, -1.0))
    weight = counts.float() if state["weight"] is None else torch.where(counts, state["weight"], 0.0)
    dz *= weight[:, None]
    return loss, (dz @ matrix).to(dtype), (dz.t() @ hidden).to(dtype)


def _plain_clip(state):
    grads, limit = state["grads"], state["limit"]
    total = torch.stack([g.double().square().sum() for g in grads]).sum()
    norm = total.sqrt()
    scale = torch.where((norm > limit) & torch.isfinite(norm), limit / norm, 1.0)
    if state["out"] is None:
        return norm.float(), [g.mul_(scale.to(g.dtype)) for g in grads]
    return norm.float(), [o.copy_(g.float() * scale.float()) for o, g in zip(state["out"], grads)]


def run(state):
    case = state["case"]
    if not own:
        return {"scan": _plain_scan, "xent": _plain_xent, "clip": _plain_clip}[case["kind"]](state)
    learner = state["learner"]
    if case["kind"] == "scan":
        if not case["grad"]:
            return learner.scan(state["x"], state["gate"], state["state"], state["done"])
        y, last, marks = learner.scan(state["x"], state["gate"], state["state"], state["done"], marks=True)
        dx, dgate, dstate = learner.scan_grad(state["x"], state["gate"], marks, state["dy"], state["done"])
        return y, last, dx, dgate, dstate
    if case["kind"] == "xent":
        return learner.cross_entropy(state["hidden"], state["matrix"], state["target"], state["weight"],
                                     grad=case["grad"])
    norm = learner.clip(state["grads"], state["limit"], out=state["out"])
    return norm, state["grads"] if state["out"] is None else state["out"]


def work(case):
    e = SIZES[case["dtype"]]
    if case["kind"] == "scan":
        T, n, d = case["T"], case["n"], case["d"]
        # x, gate, done and the state in, y and the last state out; a sigmoid and its
        # complement, two products and a sum.  Backward: dy in too, dx, dgate and dstate
        # out; the recurrence again and three products for each gradient
        rows, ends = T * n * d, n * d * 4
        moved = 3 * rows * e + 2 * ends + (T * n if case["done"] else 0)
        if case["grad"]:
            moved += 3 * rows * e + ends
        return dict(bytes=moved, flops=rows * (16 if case["grad"] else 7))
    if case["kind"] == "xent":
        N, D, V = case["rows"], case["D"], case["V"]
        moved = (N + V) * D * e + N * 12 + (N * 4 if case["weighted"] else 0)
        if case["grad"]:
            moved += (N + V) * D * e
        return dict(bytes=moved, flops=2 * N * D * V * (3 if case["grad"] else 1) + 4 * N * V)
    sizes = _sizes(case)
    moved = sum(k * (4 if case["mixed"] and i % 2 else e) for i, k in enumerate(sizes))
    return dict(bytes=moved * (2 if case["clipped"] else 1), flops=sum(sizes) * (3 if case["clipped"] else 2))


def _exact_scan(case, state):
    T = case["T"]
    # whole tensors on one step at a time, in 64 bits
    x, gate = state["x"].double(), state["gate"].double()
    a = torch.sigmoid(gate)
    keep = torch.ones((T, case["n"], 1), device=x.device, dtype=torch.float64)
    if state["done"] is not None:
        keep.masked_fill_(state["done"].bool()[:, :, None], 0.0)
    h = torch.empty_like(x, memory_format=torch.contiguous_format)
    into = torch.empty_like(h)                      # the state each step starts from
    s = state["state"].double()
    b = (1.0 - a) * x
    for t in range(T):
        into[t] = s
        torch.addcmul(b[t], a[t], s, out=h[t])
        s = h[t] * keep[t]
    if not case["grad"]:
        return h, s
    e = torch.empty_like(h)
    back = torch.zeros_like(s)
    dy = state["dy"].double()
    for t in reversed(range(T)):
        torch.add(dy[t], back, out=e[t])
        back = e[t] * a[t]
        if t:
            back = back * keep[t - 1]
    # 1 - sigmoid(g) = sigmoid(-g), without the difference
    take = torch.sigmoid(-gate)
    return h, s, take * e, a * take * (into - x) * e, back


def _exact_xent(case, state):
    V, N = case["V"], case["rows"]
    matrix = state["matrix"].double()
    losses, dhidden, dmatrix = [], [], torch.zeros_like(matrix)
    block = max(1, (1 << 28) // V)
    for r in range(0, N, block):
        x, t = state["hidden"][r:r + block].double(), state["target"][r:r + block]
        rows = torch.nonzero((t >= 0) & (t < V))[:, 0]
        lq = torch.log_softmax(x[rows] @ matrix.t(), dim=1)
        loss = torch.zeros(t.shape[0], device=x.device, dtype=torch.float64)
        loss[rows] = -lq[torch.arange(rows.shape[0], device=x.device), t[rows]]
        losses.append(loss)
        if case["grad"]:
            g = lq.exp_()
            g[torch.arange(rows.shape[0], device=x.device), t[rows]] -= 1.0
            if state["weight"] is not None:
                g *= state["weight"][r:r + block][rows, None].double()
            dx = torch.zeros_like(x)
            dx[rows] = g @ matrix
            dhidden.append(dx)
            dmatrix += g.t() @ x[rows]
    return (torch.cat(losses), torch.cat(dhidden), dmatrix) if case["grad"] else torch.cat(losses)


def _exact_clip(case, state):
    square = sum(float((g.double() ** 2).sum()) for g in state["grads"])
    norm = math.sqrt(square)
    factor = state["limit"] / norm if norm > state["limit"] else 1.0
    return torch.tensor(norm, dtype=torch.float64), [g.double() * factor for g in state["grads"]]


def exact(case, seed):
    return {"scan": _exact_scan, "xent": _exact_xent, "clip": _exact_clip}[case["kind"]](case, prepare(case, seed))
