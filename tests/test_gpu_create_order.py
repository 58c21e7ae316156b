"""A handle's memory is cleared before its creation returns, whatever the null stream has to do."""
import numpy as np
import pytest

import workloads

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("D", [40, 300])
def test_first_steps_of_a_wide_handle_behind_a_busy_null_stream(D):
    """Steps on a stream that does not wait for the null stream leave the same state after
    the first reset as after a second one, when everything before has ended."""
    from paper_2207_07736_amd import Simulator
    n, T, seed = 3000, 20, 4
    busy = torch.empty(1 << 28, dtype=torch.float32, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        busy.fill_(1.0)                           # on the null stream, some 4 ms
    sim = Simulator(n, D, workloads.CARTPOLE, stream=s)
    try:
        states = []
        for _ in range(2):
            sim.reset(seed)
            for _ in range(T):
                sim.step(1)
            states.append(sim.get_state())
            torch.cuda.synchronize()
        assert np.any(states[1][0][4:])
        assert np.array_equal(states[0][0].view(np.uint32), states[1][0].view(np.uint32))
        assert np.array_equal(states[0][1], states[1][1])
    finally:
        sim.close()
