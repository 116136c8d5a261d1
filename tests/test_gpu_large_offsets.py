"""Tensors of more than 2^31 elements: the far end is computed from the right places."""
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
    torch.cuda.empty_cache()


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def test_norm(niti):
    M, C = 530000, 4096
    x = torch.zeros((M, C), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    some = torch.randn((5, C), device="cuda", generator=g).to(torch.bfloat16)
    x[-5:] = some
    gain = torch.ones(C, device="cuda")
    y, s, _, r = niti.rmsnorm_fwd(x, gain)
    ys, ss, _, rs = niti.rmsnorm_fwd(some, gain)
    assert torch.equal(y[-5:], ys) and torch.equal(s[-5:], ss) and torch.equal(r[-5:], rs) and not y[:-5].any()
    v = niti.dequantize(y, s, dtype=torch.bfloat16)
    assert torch.equal(v[-5:], niti.dequantize(ys, ss, dtype=torch.bfloat16))
    del y, v
    dx, _ = niti.rmsnorm_bwd(x, x, gain, r, need_dgain=False)
    ds, _ = niti.rmsnorm_bwd(some, some, gain, rs, need_dgain=False)
    assert torch.equal(dx[-5:], ds)
    del dx
    q, sq = niti.quantize(x, rows=False)
    qs, sqs = niti.quantize(some, rows=False)
    assert torch.equal(q[-5:], qs) and torch.equal(sq, sqs)


@pytest.mark.parametrize("M", [4, 70000])
def test_linear(niti, M):
    """M = 4: weights of more than 2^31 bytes; M = 70000: as many outputs."""
    N, K = (70000, 32768) if M == 4 else (32768, 64)
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.zeros((N, K), dtype=torch.int8, device="cuda")
    a = torch.zeros((M, K), dtype=torch.int8, device="cuda")
    s = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    w[-40:] = torch.randint(-127, 128, (40, K), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
    a[-3:] = torch.randint(-127, 128, (3, K), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
    out, _ = niti.linear_act_fwd(a, s, w, s, dtype=torch.bfloat16)
    want = (a[-3:].double() @ w[-40:].double().t()) * 2.0 ** -18
    assert torch.equal(out[-3:, -40:], want.float().to(torch.bfloat16)) and not out[:, :-40].any() and not out[:-3].any()


def test_adamw(niti):
    n = (1 << 31) + 5000
    p = torch.zeros(n, device="cuda")
    grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v, sm, sv = niti.adamw_state(p, 8)
    tail = torch.linspace(-1, 1, 3000, device="cuda").to(torch.bfloat16)
    grad[-3000:] = tail
    p[-3000:] = 1.0
    step = torch.ones(1, dtype=torch.int32, device="cuda")
    niti.adamw(niti.adamw_tensors([p], [grad], [m], [v], s_m=[sm], s_v=[sv]), step, 1e-2)
    # first step: every element with a gradient moves by lr, against its sign (eps is 1e-8 of a root above 1e-5)
    want = np.where(tail.float().cpu().numpy() == 0, 1.0, 1.0 - 1e-2 * np.sign(tail.float().cpu().numpy()))
    assert np.allclose(p[-3000:].cpu().numpy(), want, atol=2e-6) and not p[:-3000].any()
    values = niti.dequantize(m, sm, dtype=torch.bfloat16, block=256)
    # a code is within one part in eight of its value
    assert np.all(np.abs(values[-3000:].float().cpu().numpy() - 0.1 * tail.float().cpu().numpy()) <= 0.1 * tail.float().abs().cpu().numpy() / 8 + 1e-5)
    assert not values[:-3000].any() and niti.check() == 0
