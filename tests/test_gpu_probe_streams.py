"""probe_store on the default stream or a raw one, called with another current stream, comes
after what that has been given."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("own", ("none", "raw"))
def test_a_store_follows_a_fill_of_the_current_stream(own):
    from paper_2207_07736_amd import Trajectory
    from paper_2207_07736_amd.probe import probe_store
    n, K = 1 << 16, 8
    tr = Trajectory(K, n, stats=False)
    busy = torch.empty(1 << 28, dtype=torch.float32, device="cuda")
    current, kept = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(current):
            for _ in range(10):
                busy.fill_(1.0)                   # the fill of done waits for these
            tr.done.fill_(9)
            probe_store(n, K, tr.obs, tr.action, tr.reward, tr.done, stream=None if own == "none" else kept.cuda_stream)
        torch.cuda.synchronize()
        assert int((tr.done == 9).sum()) == 0
