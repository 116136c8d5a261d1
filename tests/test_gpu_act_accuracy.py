"""GELU, SiLU and their slopes in float32 over their whole range, against 64 bits.  The argument is a bias beside sums of zeros, so
that it is exact; the slope is the bias gradient of one row with an error of one.

Bounds.  With a = |z|, Q the tail of the normal distribution, GELU is max(z, 0) - a Q(a).  The tail takes one reciprocal (2^-23)
and one exponential (2^-22), a polynomial whose argument carries the reciprocal's error and the rounding of two operations
(2^-22, which moves it by no more than as much), its own roundings and fit (2^-23), and two products: below 5 * 2^-22.  The
exponent z^2 / 2 is rounded twice, and its factor once: z^2 2^-23.7.  SiLU: exponential, reciprocal and five roundings, below 2^-21."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TAIL = 5 * 2.0 ** -22
STEP = 2.0 ** -24
LEAST = 2.0 ** -118               # (exponentials and reciprocals below the normal numbers are 0; times |z|)


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _points(n):
    rng = np.random.default_rng(3)
    z = np.concatenate([rng.uniform(-13, 13, n // 2), rng.uniform(-3, 3, n // 4), 10.0 ** rng.uniform(-6, 2, n - n // 2 - n // 4) * rng.choice([-1, 1], n - n // 2 - n // 4)])
    z[:8] = [0.0, -0.0, -5.0, -5.6, -6.0, -12.9, 40.0, -40.0]
    return z.astype(np.float32)


def _tail(z):
    # (ndtr() is 0 below -8.4)
    return torch.special.erfc(torch.from_numpy(np.abs(z)) / np.sqrt(2.0)).numpy() / 2


def _forward(niti, z, act, M):
    a, w = torch.zeros((M, 32), dtype=torch.int8, device="cuda"), torch.zeros((z.size, 32), dtype=torch.int8, device="cuda")
    s = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = niti.linear_act_fwd(a, s, w, s, bias=torch.from_numpy(z).cuda(), act=act, dtype=torch.float32)
    assert all(torch.equal(out[i], out[0]) for i in (M // 2, M - 1))
    return out[0].cpu().numpy().astype(float)


def _slope(niti, z, act):
    a, w = torch.zeros((1, 32), dtype=torch.int8, device="cuda"), torch.zeros((z.size, 32), dtype=torch.int8, device="cuda")
    s = torch.zeros(1, dtype=torch.int32, device="cuda")
    _, _, db = niti.linear_act_bwd(a, s, w, s, torch.ones((1, z.size), device="cuda"), z=torch.from_numpy(z).cuda().view(1, -1), act=act)
    return db.cpu().numpy().astype(float)


# rows that are streamed, and tiles with whole and with ragged rows of results
@pytest.mark.parametrize("M,N", [(1, 16384), (200, 4096), (200, 4095)])
def test_gelu(niti, M, N):
    z = _points(N)
    got, z = _forward(niti, z, "gelu", M), z.astype(float)
    part = np.abs(z) * _tail(z)
    want = np.maximum(z, 0) - part
    assert np.all(np.abs(got - want) <= (TAIL + z * z * 2.0 ** -23) * part + STEP * np.abs(want) + LEAST)


@pytest.mark.parametrize("M,N", [(1, 16384), (200, 4096), (200, 4095)])
def test_silu(niti, M, N):
    z = _points(N)
    got, z = _forward(niti, z, "silu", M), z.astype(float)
    want = z * torch.sigmoid(torch.from_numpy(z)).numpy()
    assert np.all(np.abs(got - want) <= 2.0 ** -21 * np.abs(want) + LEAST)


@pytest.mark.parametrize("N", [16384, 4095])
def test_gelu_slope(niti, N):
    """u = phi(a) a - Q(a): 1 + u, or -u for negative z."""
    z = _points(N)
    got, z = _slope(niti, z, "gelu"), z.astype(float)
    q, bell = _tail(z), np.abs(z) * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    want = np.where(z < 0, q - bell, 1 - q + bell)
    off = (TAIL + z * z * 2.0 ** -23) * (q + bell)
    assert np.all(np.abs(got - want) <= off + 2 * STEP * np.abs(want) + LEAST)


@pytest.mark.parametrize("N", [16384, 4095])
def test_silu_slope(niti, N):
    """s (1 + z (1 - s)): s is off by 2^-21 of itself, 1 - s by that of s and half a step."""
    z = _points(N)
    got, z = _slope(niti, z, "silu"), z.astype(float)
    s, t = torch.sigmoid(torch.from_numpy(z)).numpy(), torch.sigmoid(torch.from_numpy(-z)).numpy()
    want = s * (1 + z * t)
    off = s * (2.0 ** -21 * (np.abs(1 + z * t) + np.abs(z) * s) + 3 * STEP * (1 + np.abs(z) * t) + STEP * np.abs(z))
    assert np.all(np.abs(got - want) <= off + LEAST)


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_arguments_that_are_not_finite(niti, act):
    """The limits at both ends, and NaN for NaN."""
    z = np.array([np.inf, -np.inf, np.nan, 3e38, -3e38, 1.0, -1.0, 0.0], dtype=np.float32)
    for M in (1, 200):
        got = _forward_any(niti, z, act, M)
        assert got[0] == np.inf and got[1] == 0 and np.isnan(got[2]) and got[3] == np.float32(3e38) and got[4] == 0 and np.isfinite(got[5:]).all()
    from paper_2009_13108_b200 import NitiError
    got = _slope(niti, z, act)
    assert got[0] == 1 and got[1] == 0 and np.isnan(got[2]) and got[3] == 1 and got[4] == 0 and np.isfinite(got[5:]).all()
    with pytest.raises(NitiError):
        niti.check()


def _forward_any(niti, z, act, M):
    a, w = torch.zeros((M, 32), dtype=torch.int8, device="cuda"), torch.zeros((z.size, 32), dtype=torch.int8, device="cuda")
    s = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = niti.linear_act_fwd(a, s, w, s, bias=torch.from_numpy(z).cuda(), act=act, dtype=torch.float32)
    return out[M - 1].cpu().numpy().astype(float)
