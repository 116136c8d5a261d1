"""AdamW with a learning rate of zero: the states move, no weight does, whatever the quotient of its moments."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [4096, 3001])
def test_weights_stay_at_a_learning_rate_of_zero(niti, bits, n):
    """Moments with a zero second moment (beta2 = 0, no gradient) at the smallest eps, beside weights of zero and small ones."""
    rng = np.random.default_rng(1)
    p = torch.from_numpy((10.0 ** rng.uniform(-38, 2, n) * rng.choice([-1, 0, 1], n)).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda()
    m, v, s_m, s_v = niti.adamw_state(p, bits)
    plan = niti.adamw_tensors([p], [g], [m], [v], s_m=[s_m] if bits == 8 else None, s_v=[s_v] if bits == 8 else None, weight_decay=0.5)
    p0 = p.clone()
    step = torch.ones(1, dtype=torch.int32, device="cuda")
    for lr in (0.0, 0.0, 1e-31):
        niti.adamw(plan, step, lr, (0.9, 0.0), 1e-20)
        assert torch.equal(p, p0) and m.any()
        step += 1
        g.zero_()
    niti.adamw(plan, step, 1e-3, (0.9, 0.0), 1e-20)
    assert not torch.equal(p, p0)
    assert niti.check() == 0
