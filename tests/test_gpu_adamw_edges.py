"""AdamW where its numbers are at the ends of float32: second moments that are subnormal, weights that are not finite."""
import numpy as np
import pytest
import torch

from floatref import decode_e4m3, random_bits, split_e4m3

pytestmark = pytest.mark.gpu
F = np.float32
LR, B1, B2, EPS = 1e-2, 0.9, 0.999, 1e-20
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _step(t):
    return torch.full((1,), t, dtype=torch.int32, device="cuda")


def _gradients(n, seed, lo=-24.0, hi=-17.0):
    """Magnitudes from 10^lo to 10^hi, of both signs."""
    rng = np.random.default_rng(seed)
    return (10.0 ** rng.uniform(lo, hi, n) * rng.choice([-1.0, 1.0], n)).astype(F)


def _weights_follow(got, p, m, v, t, eps=EPS):
    """float32 m and v are given: the update is off by a few steps (approximate reciprocal, the factors' roundings), the weight
    by half a step of each term."""
    upd = LR / (1 - B1 ** t) * m.astype(float) / (np.sqrt(v.astype(float) / (1 - B2 ** t)) + eps)
    assert np.all(np.abs(got.astype(float) - (p - upd)) <= 24 * STEP * np.abs(upd) + 3 * STEP * np.abs(p.astype(float)))


@pytest.mark.parametrize("offset", [0, 1])
def test_small_second_moments_in_32_bits(niti, offset):
    """Roots of v from 2^-149 to 2^-96, on both sides of the smallest normal number; zeros among them."""
    n = 4096 + offset
    rng = np.random.default_rng(1)
    v = np.ldexp(rng.uniform(1, 2, n), rng.integers(-150, -96, n)).astype(F)
    edge = np.float32(2.0 ** -126)
    v[:6] = [edge, np.nextafter(edge, F(0)), np.nextafter(edge, F(1)), F(2.0 ** -149), F(0), F(1e-39)]
    v[100:400:7] = 0
    m = (np.sqrt(v.astype(float)) * rng.standard_normal(n)).astype(F)
    g, p = _gradients(n, 2), (0.05 * rng.standard_normal(n)).astype(F)
    g[::3] = 0
    dev = [torch.from_numpy(np.concatenate([np.zeros(offset, F), x])).cuda()[offset:] for x in (p, g, m, v)]
    niti.adamw(niti.adamw_tensors(*[[x] for x in dev]), _step(3), LR, (B1, B2), EPS)
    m, v = F(B1) * m + F(1 - B1) * g, F(B2) * v + (F(1 - B2) * g) * g
    assert m.dtype == v.dtype == F
    assert np.array_equal(dev[2].cpu().numpy(), m) and np.array_equal(dev[3].cpu().numpy(), v)
    _weights_follow(dev[0].cpu().numpy(), p, m, v, 3)
    assert niti.check() == 0


@pytest.mark.parametrize("n", [2048 * 4, 3001])
def test_small_second_moments_in_8_bits(niti, n):
    """The codes are those of float32 arithmetic, in a first step from zero states and in the next without gradients."""
    g, p = _gradients(n, 5), np.zeros(n, F)
    dev = {"p": torch.zeros(n, device="cuda"), "g": torch.from_numpy(g).cuda()}
    m8, v8, s_m, s_v = niti.adamw_state(dev["p"])
    plan = niti.adamw_tensors([dev["p"]], [dev["g"]], [m8], [v8], s_m=[s_m], s_v=[s_v])
    for t in (1, 2):
        m = decode_e4m3(m8.cpu().numpy(), s_m.cpu().numpy()).astype(F)
        r = decode_e4m3(v8.cpu().numpy(), s_v.cpu().numpy()).astype(F)
        m, v = F(B1) * m + F(1 - B1) * g, F(B2) * (r * r) + (F(1 - B2) * g) * g
        r = np.sqrt(v)
        p = dev["p"].cpu().numpy()
        niti.adamw(plan, _step(t), LR, (B1, B2), EPS)
        _weights_follow(dev["p"].cpu().numpy(), p, m, v, t)
        x = random_bits(n, t)
        for code8, s8, value, draw, least in ((m8, s_m, np.abs(m), x >> 16, 0), (v8, s_v, r, x & 65535, r > 0)):
            s, code, frac, _ = split_e4m3(value.astype(np.float64))
            assert np.array_equal(s8.cpu().numpy(), s)
            want = np.maximum(code + ((np.floor(frac).astype(np.int64) + draw) >> 16), least)
            assert np.array_equal(code8.cpu().numpy().astype(np.int64) & 127, want)
        dev["g"].zero_()
        g = np.zeros(n, F)
    assert niti.check() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_elements_do_not_depend_on_their_neighbours_gradients(niti, bits):
    """Beside a gradient that is not finite every other element gets the weight that it gets without it."""
    from paper_2009_13108_b200 import NitiError
    n = 4096
    g = _gradients(n, 7, -24.0, -2.0)
    runs = []
    for bad in (False, True):
        p = torch.from_numpy((0.05 * np.random.default_rng(8).standard_normal(n)).astype(F)).cuda()
        gd = torch.from_numpy(g).cuda()
        gd[5::64] = float("nan") if bad else 0.0
        m, v, s_m, s_v = niti.adamw_state(p, bits)
        niti.adamw(niti.adamw_tensors([p], [gd], [m], [v], s_m=[s_m] if bits == 8 else None, s_v=[s_v] if bits == 8 else None),
                   _step(1), LR, (B1, B2), EPS)
        runs.append((p, m, v))
    with pytest.raises(NitiError):
        niti.check()
    keep = torch.ones(n, dtype=torch.bool)
    keep[5::64] = False
    for a, b in zip(*runs):
        assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("w8", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n,at", [(2048 * 3, 2048 + 77), (300, 299)])
def test_weights_that_are_not_finite_raise_the_status(niti, bits, w8, n, at):
    from paper_2009_13108_b200 import NitiError
    for x in (float("inf"), float("-inf"), float("nan")):
        p = torch.from_numpy((0.05 * np.random.default_rng(8).standard_normal(n)).astype(F)).cuda()
        g = torch.from_numpy(_gradients(n, 9, -4.0, -2.0)).cuda()
        m, v, s_m, s_v = niti.adamw_state(p, bits)
        w = torch.zeros(n, dtype=torch.int8, device="cuda")
        plan = niti.adamw_tensors([p], [g], [m], [v], s_m=[s_m] if bits == 8 else None, s_v=[s_v] if bits == 8 else None,
                                  w8=[w] if w8 else None, s_w=[niti.scalar(-9)] if w8 else None)
        niti.adamw(plan, _step(1), LR)
        assert niti.check() == 0
        p[at] = x
        niti.adamw(plan, _step(2), LR)
        with pytest.raises(NitiError, match="0x40|64|status"):
            niti.check()
        rest = torch.ones(n, dtype=torch.bool)
        rest[at] = False
        assert torch.isfinite(p[rest]).all() and not torch.isfinite(p[at])
        if w8:
            assert abs(int(w[at])) == 127


@pytest.mark.parametrize("bits", [32, 8])
def test_replaced_gradients_are_the_ones_used(niti, bits):
    """A list whose gradients are replaced, by others of another type and alignment, goes on as a list built with them."""
    n = 5000
    first, second = torch.from_numpy(_gradients(n, 1, -4.0, -2.0)).cuda(), torch.from_numpy(_gradients(n + 1, 2, -4.0, -2.0)).cuda().to(torch.bfloat16)[1:]
    runs = []
    for replace in (False, True):
        p = torch.from_numpy((0.05 * np.random.default_rng(8).standard_normal(n)).astype(F)).cuda()
        m, v, s_m, s_v = niti.adamw_state(p, bits)
        build = lambda g: niti.adamw_tensors([p], [g], [m], [v], s_m=[s_m] if bits == 8 else None, s_v=[s_v] if bits == 8 else None)      # noqa: E731
        plan = build(first)
        niti.adamw(plan, _step(1), LR)
        if replace:
            plan.set_grads([second])
        else:
            plan = build(second)
        niti.adamw(plan, _step(2), LR)
        runs.append((p, m, v))
    assert all(torch.equal(a, b) for a, b in zip(*runs)) and niti.check() == 0


@pytest.mark.parametrize("n", [2048, 300])
def test_int8_weights_at_the_ends_of_the_exponents(niti, n):
    """floor(|p| 2^-s + 1/2) for the smallest and the largest exponents, of weights that are subnormal and nearly infinite (a
    learning rate of zero leaves them as they are)."""
    rng = np.random.default_rng(4)
    small = np.ldexp(rng.uniform(1, 2, n), rng.integers(-149, -119, n)).astype(F)
    large = np.ldexp(rng.uniform(1, 1.99, n), rng.integers(118, 128, n)).astype(F)
    for s, p in [(-127, small), (-126, small), (-125, small), (125, large), (126, large), (127, large)]:
        p = p * rng.choice([-1, 1], n).astype(F)
        dev, w, z = torch.from_numpy(p).cuda(), torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, device="cuda")
        niti.adamw(niti.adamw_tensors([dev], [z], [z.clone()], [z.clone()], w8=[w], s_w=[niti.scalar(s)]), _step(1), 0.0)
        assert np.array_equal(dev.cpu().numpy(), p)
        want = np.minimum(np.floor(np.abs(p.astype(float)) * 2.0 ** -s + 0.5), 127)
        assert want.max() >= 2 and np.array_equal(w.cpu().numpy(), np.sign(p) * want), s
    assert niti.check() == 0
