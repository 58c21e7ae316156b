"""distill_loss on streams other than the handle's: its forward and backward wait for what
comes before on the current stream, and what comes after waits for them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("current_own", (False, True))
@pytest.mark.parametrize("handle_own", (False, True))
def test_gradients_off_the_handles_stream(handle_own, current_own):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2207_07736_amd as p
    handle = torch.cuda.Stream() if handle_own else None
    current = torch.cuda.Stream() if current_own else torch.cuda.default_stream()
    head, plain = p.Head(512, 30000, stream=handle), p.Head(512, 30000)
    rng = np.random.default_rng(0)
    busy = torch.zeros((4096, 4096), device="cuda", dtype=torch.bfloat16)
    try:
        for rows, V in ((6, 700), (8, 30000), (512, 5003)):
            teacher = torch.from_numpy(rng.standard_normal((rows, 9)).astype(np.float32)).cuda()
            index = torch.from_numpy(np.argsort(rng.random((rows, V)), axis=1)[:, :9].astype(np.int32)).cuda()
            for turn in range(4):
                x = torch.from_numpy(rng.standard_normal((rows, V)).astype(np.float32)).cuda()
                want = plain.distill(x * 2.0, teacher, index, weight=torch.full((rows,), 1 / rows, device="cuda"))
                torch.cuda.synchronize()
                with torch.cuda.stream(current):
                    leaf = x.clone().requires_grad_()
                    for _ in range(12):                      # a millisecond of work ahead of the student's rows
                        busy = busy @ busy
                    student = leaf * (2.0 + busy[0, 0].float())
                    losses = head.distill_loss(student, teacher, index)
                    kept = losses.detach().clone()
                    for _ in range(12):                      # and of the losses' gradient
                        busy = busy @ busy
                    (losses.mean() * (1.0 + busy[0, 0].float())).backward()
                    grad = leaf.grad.clone()
                    del losses, student, leaf
                    torch.full((rows, V), float("nan"), device="cuda")       # over whatever was freed
                torch.cuda.synchronize()
                assert torch.equal(kept, want[0]) and torch.equal(grad, want[1] * 2.0), (rows, V, turn)
    finally:
        head.close()
        plain.close()
