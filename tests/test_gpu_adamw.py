"""AdamW against its formula in 64 bits, states in 32 and in 8 bits."""
import numpy as np
import pytest
import torch

from floatref import block_exponents, decode_e4m3, random_bits, split_e4m3

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS = 1e-2, 0.9, 0.999, 1e-8
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _np(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def _problem(sizes, bits, gtype, w8, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n: torch.randn(n, device="cuda", generator=g)                    # noqa: E731
    ps, gs = [0.05 * rnd(n) for n in sizes], [(1e-2 * rnd(n)).to(gtype) for n in sizes]
    out = {"p": ps, "g": gs, "decay": [0.1 * (i % 2) for i in range(len(sizes))]}
    if bits == 8:
        code = lambda n, top: torch.randint(0, top, (n,), device="cuda", generator=g).to(torch.uint8)      # noqa: E731
        # codes of a magnitude below 256 (120), with a sign for the first moment
        out["m"] = [code(n, 121) | (code(n, 2) << 7) for n in sizes]
        out["v"] = [code(n, 121) for n in sizes]
        exps = lambda n, lo: torch.randint(lo, lo + 3, (-(-n // 256),), device="cuda", generator=g).to(torch.int8)   # noqa: E731
        out["s_m"], out["s_v"] = [exps(n, -17) for n in sizes], [exps(n, -15) for n in sizes]
    else:
        out["m"], out["v"] = [1e-3 * rnd(n) for n in sizes], [1e-4 * rnd(n).square() for n in sizes]
    if w8:
        out["w8"] = [torch.zeros(n, dtype=torch.int8, device="cuda") for n in sizes]
        out["s_w"] = [torch.full((1,), -9 - i % 3, dtype=torch.int32, device="cuda") for i in range(len(sizes))]
    return out


def _plan(niti, pr):
    return niti.adamw_tensors(pr["p"], pr["g"], pr["m"], pr["v"], s_m=pr.get("s_m"), s_v=pr.get("s_v"), w8=pr.get("w8"),
                              s_w=pr.get("s_w"), weight_decay=pr["decay"])


def _expected(pr, i, bits, t, scale=1.0):
    """The formulas, and by how much float32 arithmetic can miss m and v."""
    p, g = _np(pr["p"][i]), _np(pr["g"][i]) * scale
    if bits == 8:
        m = decode_e4m3(pr["m"][i].cpu().numpy(), pr["s_m"][i].cpu().numpy())
        v = decode_e4m3(pr["v"][i].cpu().numpy(), pr["s_v"][i].cpu().numpy()) ** 2
    else:
        m, v = _np(pr["m"][i]), _np(pr["v"][i])
    m_slack = 4 * STEP * (np.abs(B1 * m) + np.abs((1 - B1) * g))
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    upd = LR / (1 - B1 ** t) * m / (np.sqrt(v / (1 - B2 ** t)) + EPS)
    # the update is off by that of m, a few steps of the quotient (approximate division and root: 2 steps each) and of the
    # bias corrections; the weight by half a step of each of its terms
    p_slack = (LR / (1 - B1 ** t) * m_slack / (np.sqrt(v / (1 - B2 ** t)) + EPS) + 24 * STEP * np.abs(upd) + 3 * STEP * np.abs(p))
    return p * (1 - LR * pr["decay"][i]) - upd, m, v, p_slack, m_slack


SIZES = [[1], [255, 256, 257], [1000, 8, 70001, 3], [5] * 40, [300 + 17 * i for i in range(300)], [2048 * 40]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w8", [False, True])
def test_one_step(niti, sizes, gtype, bits, w8, pr=None):
    pr = pr or _problem(sizes, bits, gtype, w8)
    t = 7
    want = [_expected(pr, i, bits, t) for i in range(len(sizes))]
    niti.adamw(_plan(niti, pr), torch.full((1,), t, dtype=torch.int32, device="cuda"), LR, (B1, B2), EPS)
    for i, (p, m, v, p_slack, m_slack) in enumerate(want):
        got = _np(pr["p"][i])
        assert np.all(np.abs(got - p) <= p_slack)
        if bits == 32:
            assert np.all(np.abs(_np(pr["m"][i]) - m) <= m_slack)
            assert np.all(np.abs(_np(pr["v"][i]) - v) <= 6 * STEP * v + 1e-45)
        else:
            _check_codes(pr, i, m, v, m_slack, t)
        if w8:
            u = np.abs(got) * 2.0 ** -int(pr["s_w"][i])          # (of the stored weight: exact)
            assert np.array_equal(_np(pr["w8"][i]), np.sign(got) * np.minimum(np.floor(u + 0.5), 127))
    assert niti.check() == 0


def test_many_chunks(niti):
    """Enough elements that a CTA takes several chunks in a row and stores their exponents together; the tensors end inside
    chunks, and their exponents start on no particular boundary."""
    sizes = [9_000_001, 300, 5_500_123, 2_100_000]
    pr = _problem(sizes, 8, torch.bfloat16, True)
    whole = torch.zeros(sum(x.numel() for x in pr["s_m"]) + 3, dtype=torch.int8, device="cuda")
    at = 3
    for i, e in enumerate(pr["s_m"]):
        whole[at:at + e.numel()] = e
        pr["s_m"][i] = whole[at:at + e.numel()]
        at += e.numel()
    before = pr["p"][1].clone()
    test_one_step(niti, sizes, torch.bfloat16, 8, True, pr=pr)
    assert not torch.equal(before, pr["p"][1]) and not whole[:3].any()


def test_tensors_that_are_copied_in_bulk_among_others(niti):
    """A CTA's chunks come from aligned tensors, whose operands are fetched ahead, and from others, in turn: the exponents of
    one bulk chunk must not meet those of the next where a warp runs ahead over the chunks between them."""
    sizes = [2048 * 25 + 200 * (i % 3) for i in range(160)]
    pr = _problem(sizes, 8, torch.bfloat16, True)
    for i in range(0, len(sizes), 2):
        buf = torch.zeros(sizes[i] + 1, device="cuda")
        buf[1:] = pr["p"][i]
        pr["p"][i] = buf[1:]
    test_one_step(niti, sizes, torch.bfloat16, 8, True, pr=pr)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_whose_squares_overflow_leave_their_elements(niti, bits):
    from paper_2009_13108_b200 import NitiError
    pr = _problem([4000, 300], bits, torch.float32, True)
    big = torch.tensor([2.0 ** 63, -3e19, 3e38, 2.0 ** 100], device="cuda")
    for i, at in ((0, 700), (1, 296)):
        pr["g"][i][at:at + 4] = big
        pr["g"][i][at - 1] = 2.0 ** 62
    was = [(p.clone(), m.clone(), v.clone()) for p, m, v in zip(pr["p"], pr["m"], pr["v"])]
    niti.adamw(_plan(niti, pr), torch.ones(1, dtype=torch.int32, device="cuda"), LR, (B1, B2), EPS)
    with pytest.raises(NitiError):
        niti.check()
    for i, at in ((0, 700), (1, 296)):
        assert torch.equal(pr["p"][i][at:at + 4], was[i][0][at:at + 4]) and torch.isfinite(pr["p"][i]).all()
        # the smaller one is taken: a first step's m / sqrt(v) is about 1 beside its neighbours' states
        assert not torch.equal(pr["p"][i][at - 1], was[i][0][at - 1])
        if bits == 32:
            assert torch.equal(pr["m"][i][at:at + 4], was[i][1][at:at + 4]) and torch.equal(pr["v"][i][at:at + 4], was[i][2][at:at + 4])
            assert torch.isfinite(pr["v"][i]).all()
        else:
            for codes in (pr["m"][i], pr["v"][i]):
                assert int((codes & 127).max()) <= 126
            assert int(pr["v"][i].max()) <= 126 and int(pr["s_v"][i].max()) <= 63


def test_a_learning_rate_of_zero_changes_the_states_alone(niti):
    for bits in (32, 8):
        pr = _problem([5000], bits, torch.float32, False)
        for k in ("g", "m", "v"):
            pr[k][0][::2] = 0                     # (no gradient, no states)
        p0, m0 = pr["p"][0].clone(), pr["m"][0].clone()
        niti.adamw(_plan(niti, pr), torch.ones(1, dtype=torch.int32, device="cuda"), 0.0, (0.9, 0.99999), 1e-8)
        assert torch.equal(pr["p"][0], p0) and not torch.equal(pr["m"][0], m0)


def _check_codes(pr, i, m, v, m_slack, t):
    r = np.sqrt(v)
    # a maximum that float32 can carry over a power of two may have either exponent (0.9 m + 0.1 g of short numbers meets
    # powers of two exactly)
    s_m, s_r = pr["s_m"][i].cpu().numpy().astype(np.int64), pr["s_v"][i].cpu().numpy().astype(np.int64)
    for s, x, slack in ((s_m, np.abs(m), m_slack), (s_r, r, 4 * STEP * r)):
        assert np.all((s == block_exponents(np.maximum(x - slack, 0))) | (s == block_exponents(x + slack)))
    _, code_m, f_m, unit_m = split_e4m3(np.abs(m), s_m)
    _, code_r, f_r, unit_r = split_e4m3(r, s_r)
    got_m, got_r = pr["m"][i].cpu().numpy().astype(np.int64), pr["v"][i].cpu().numpy().astype(np.int64)
    assert np.all((np.abs(m) <= m_slack) | ((got_m >= 128) == (m < 0)) | (got_m & 127 == 0))
    x = random_bits(m.size, t)
    for got, code, f, draw, slack, least in ((got_m & 127, code_m, f_m, x >> 16, m_slack * unit_m, 0), (got_r, code_r, f_r, x & 65535, 4 * STEP * r * unit_r, r > 0)):
        off = slack * 65536 + 1
        total = np.floor(f) + draw
        # float32 can change neither the whole part nor whether the sum carries
        sure = (np.abs(total - 65536) > off) & (f > off) & (f < 65536 - off)
        want = np.maximum(code + (total >= 65536), least)
        assert np.array_equal(got[sure], want[sure]) and np.all(np.abs(got - want) <= 1)
        if m.size > 5000:
            assert sure.mean() > 0.8


def test_codes_follow_from_float32_operations(niti):
    """Every product and sum rounded to float32, the root correctly rounded: the codes are exactly those of numpy's float32."""
    n, t = 1 << 20, 9
    f = np.float32
    pr = _problem([n], 8, torch.bfloat16, False, seed=5)
    g = pr["g"][0].float().cpu().numpy()
    m = decode_e4m3(pr["m"][0].cpu().numpy(), pr["s_m"][0].cpu().numpy()).astype(f)          # (exact)
    r = decode_e4m3(pr["v"][0].cpu().numpy(), pr["s_v"][0].cpu().numpy()).astype(f)
    m = f(B1) * m + f(1 - B1) * g
    r = np.sqrt(f(B2) * (r * r) + f(1 - B2) * g * g)
    assert m.dtype == r.dtype == f
    niti.adamw(_plan(niti, pr), torch.full((1,), t, dtype=torch.int32, device="cuda"), LR, (B1, B2), EPS)
    x = random_bits(n, t)
    for name, value, draw, least in (("m", np.abs(m), x >> 16, 0), ("v", r, x & 65535, r > 0)):
        s, code, frac, _ = split_e4m3(value.astype(np.float64))
        want = np.maximum(code + ((np.floor(frac).astype(np.int64) + draw) >> 16), least)
        assert np.array_equal(pr["s_" + name][0].cpu().numpy(), s)
        got = pr[name][0].cpu().numpy().astype(np.int64)
        assert np.array_equal(got & 127, want)
    assert np.array_equal(pr["m"][0].cpu().numpy() >= 128, m < 0)


def test_32_bit_states_are_numpys(niti):
    n, f = 1 << 20, np.float32
    pr = _problem([n], 32, torch.bfloat16, False, seed=6)
    g, m, v = pr["g"][0].float().cpu().numpy(), pr["m"][0].cpu().numpy(), pr["v"][0].cpu().numpy()
    niti.adamw(_plan(niti, pr), torch.ones(1, dtype=torch.int32, device="cuda"), LR, (B1, B2), EPS)
    assert np.array_equal(pr["m"][0].cpu().numpy(), f(B1) * m + f(1 - B1) * g)
    assert np.array_equal(pr["v"][0].cpu().numpy(), f(B2) * v + f(1 - B2) * g * g)


def test_rounding_of_states_is_unbiased(niti):
    """bfloat16 gradients and short codes, whose weighted sums have repeating bits."""
    n = 1 << 20
    pr = _problem([n], 8, torch.bfloat16, False, seed=3)
    _, m, v, _, _ = _expected(pr, 0, 8, 5)
    niti.adamw(_plan(niti, pr), torch.full((1,), 5, dtype=torch.int32, device="cuda"), LR, (B1, B2), EPS)
    for x, name in ((m, "m"), (np.sqrt(v), "v")):
        s, _, _, unit = split_e4m3(np.abs(x))
        got = decode_e4m3(pr[name][0].cpu().numpy(), pr["s_" + name][0].cpu().numpy())
        err = (np.abs(got) - np.abs(x)) * unit                # in units of the code's last place
        assert np.abs(err).max() <= 1 + 1e-3
        # errors between two neighbours have a deviation of at most half a unit, their mean one of 0.5 / sqrt(n); the
        # truncation to 16 bits costs less than 2^-16, roots that are kept from zero are at most one in 120
        assert abs(err.mean()) < 2.0 ** -16 + 5 * 0.5 / np.sqrt(n), name


def test_states_without_a_gradient_decay(niti):
    """No code is a fixed point: with zero gradients every root shrinks by sqrt(0.999) a step on average."""
    n, steps = 1 << 14, 400
    pr = _problem([n], 8, torch.float32, False)
    pr["g"][0].zero_(); pr["s_v"][0].zero_(); pr["s_m"][0].zero_()
    pr["v"][0].copy_(torch.arange(n, device="cuda") % 56 + 64)                # normal codes
    old = decode_e4m3(pr["v"][0].cpu().numpy(), pr["s_v"][0].cpu().numpy())
    step, plan = torch.zeros(1, dtype=torch.int32, device="cuda"), _plan(niti, pr)
    for _ in range(steps):
        step += 1
        niti.adamw(plan, step, LR, (B1, B2), EPS)
    new = decode_e4m3(pr["v"][0].cpu().numpy(), pr["s_v"][0].cpu().numpy())
    ratio = (new / old).mean()
    # a walk of unbiased steps: each moves by one unit (at most 1 / 8 of the value) with the probability that the decay
    # (1 / 2000 of the value, at most 1 / 125 of a unit) asks for, so a value's variance after 400 steps is below
    # 400 / 2000 / 8 of its square, and the mean of 16384 is within 5 * sqrt(0.025 / 16384) = 0.007
    assert abs(ratio - B2 ** (steps / 2)) < 0.007


def test_steps_in_8_bits_follow_those_in_32(niti):
    """Twenty steps on the same gradients.  Each step's states carry relative errors up to 2^-3 (m) and 2^-3 (r) of zero
    mean, so an update of magnitude lr is off by less than lr / 4 + lr / 4, and the weights by less than 20 times that."""
    n = 4096
    a, b = _problem([n], 32, torch.float32, False), _problem([n], 8, torch.float32, False)
    for x in ("m", "v"):
        a[x][0].zero_(); b[x][0].zero_()
        b["s_" + x][0].zero_()
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    pa, pb = _plan(niti, a), _plan(niti, b)
    g = torch.Generator(device="cuda").manual_seed(9)
    start = a["p"][0].clone()
    for _ in range(20):
        step += 1
        a["g"][0].copy_(1e-2 * (torch.randn(n, device="cuda", generator=g) + 1))
        b["g"][0].copy_(a["g"][0])
        niti.adamw(pa, step, LR, (B1, B2), EPS)
        niti.adamw(pb, step, LR, (B1, B2), EPS)
    assert (a["p"][0] - start).abs().mean() > 5 * LR
    assert (a["p"][0] - b["p"][0]).abs().max() < 20 * LR / 2


def test_gradients_that_are_not_finite_leave_their_elements(niti):
    from paper_2009_13108_b200 import NitiError
    for bits in (32, 8):
        pr = _problem([600], bits, torch.float32, False)
        p0, m0, v0 = pr["p"][0].clone(), pr["m"][0].clone(), pr["v"][0].clone()
        bad = [0, 255, 256, 599]
        for i, x in zip(bad, (float("nan"), float("inf"), float("-inf"), float("nan"))):
            pr["g"][0][i] = x
        niti.adamw(_plan(niti, pr), torch.ones(1, dtype=torch.int32, device="cuda"), LR)
        with pytest.raises(NitiError):
            niti.check()
        assert torch.equal(pr["p"][0][bad], p0[bad]) and torch.isfinite(pr["p"][0]).all()
        ok = torch.ones(600, dtype=torch.bool)
        ok[bad] = False
        assert (pr["p"][0].cpu()[ok] != p0.cpu()[ok]).all()
        if bits == 32:
            assert torch.equal(pr["m"][0][bad], m0[bad]) and torch.equal(pr["v"][0][bad], v0[bad])


def test_gradient_scale_and_zero_gradients(niti):
    pr, qr = _problem([1000], 32, torch.float32, False), _problem([1000], 32, torch.float32, False)
    step = torch.full((1,), 3, dtype=torch.int32, device="cuda")
    qr["g"][0].mul_(4.0)
    niti.adamw(_plan(niti, pr), step, LR)
    niti.adamw(_plan(niti, qr), step, LR, grad_scale=torch.full((1,), 0.25, device="cuda"))
    assert torch.equal(pr["p"][0], qr["p"][0]) and torch.equal(pr["m"][0], qr["m"][0])
    # no gradient and no states: only the decay
    zr = _problem([512], 8, torch.float32, False)
    zr["decay"] = [0.5]
    for k in ("g", "m", "v", "s_m", "s_v"):
        zr[k][0].zero_()
    p0 = zr["p"][0].clone()
    niti.adamw(_plan(niti, zr), step, LR)
    assert np.allclose(_np(zr["p"][0]), _np(p0) * (1 - LR * 0.5), rtol=2 * STEP, atol=0)
    assert not zr["m"][0].any() and not zr["v"][0].any()
    assert niti.check() == 0


def test_slices_of_one_buffer(niti):
    """Tensors that start on no vector boundary, gaps between them untouched."""
    n = 3000
    for bits in (32, 8):
        pr = _problem([n], bits, torch.bfloat16, True)
        cut = [(1, 700), (703, 1301), (1500, 2999)]
        view = lambda x: [x[0][a:b] for a, b in cut]                              # noqa: E731
        sub = {k: view(pr[k]) for k in ("p", "g", "m", "v", "w8")}
        sub["decay"], sub["s_w"] = [0.0, 0.1, 0.0], [pr["s_w"][0]] * 3
        if bits == 8:
            for k in ("s_m", "s_v"):
                sub[k] = [torch.full((-(-(b - a) // 256),), -12, dtype=torch.int8, device="cuda") for a, b in cut]
        want = [_expected(sub, i, bits, 2) for i in range(3)]
        before = {k: pr[k][0].clone() for k in ("p", "m", "v", "w8")}
        niti.adamw(_plan(niti, sub), torch.full((1,), 2, dtype=torch.int32, device="cuda"), LR)
        for i, (p, m, v, p_slack, m_slack) in enumerate(want):
            assert np.all(np.abs(_np(sub["p"][i]) - p) <= p_slack)
        for k, old in before.items():
            for gap in (slice(0, 1), slice(700, 703), slice(1301, 1500), slice(2999, 3000)):
                assert torch.equal(pr[k][0][gap], old[gap])


def test_replays_of_a_captured_step_count_on(niti):
    a, b = _problem([5000, 300], 8, torch.bfloat16, True), _problem([5000, 300], 8, torch.bfloat16, True)
    pa, pb = _plan(niti, a), _plan(niti, b)
    sa, sb = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        sa += 1
        niti.adamw(pa, sa, LR)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        graph.replay()
        sb += 1
        niti.adamw(pb, sb, LR)
    for k in ("p", "m", "v", "w8", "s_m", "s_v"):
        for x, y in zip(a[k], b[k]):
            assert torch.equal(x, y)


def test_a_step_number_below_one_updates_nothing(niti):
    from paper_2009_13108_b200 import NitiError
    pr = _problem([400], 32, torch.float32, False)
    p0 = pr["p"][0].clone()
    niti.adamw(_plan(niti, pr), torch.zeros(1, dtype=torch.int32, device="cuda"), LR)
    with pytest.raises(NitiError):
        niti.check()
    assert torch.equal(p0, pr["p"][0])


def test_refusals(niti):
    from paper_2009_13108_b200 import NitiError
    pr = _problem([512, 10], 32, torch.float32, True)
    plan = _plan(niti, pr)
    step = torch.ones(1, dtype=torch.int32, device="cuda")
    p0 = [p.clone() for p in pr["p"]]
    for kw in ({"lr": -1.0}, {"lr": float("nan")}, {"lr": LR, "betas": (1.0, 0.9)}, {"lr": LR, "betas": (0.9, -0.1)}, {"lr": LR, "eps": 0.0}):
        with pytest.raises(NitiError):
            niti.adamw(plan, step, **kw)
    with pytest.raises(NitiError):
        niti.adamw(plan, step.float(), LR)
    bad = [dict(pr, p=[p.double() for p in pr["p"]]), dict(pr, g=pr["g"][:1]), dict(pr, m=[m[:5] for m in pr["m"]]),
           dict(pr, m=[m.to(torch.bfloat16) for m in pr["m"]]), dict(pr, s_w=None), dict(pr, w8=[w.int() for w in pr["w8"]]),
           dict(pr, p=[p.cpu() for p in pr["p"]]), dict(pr, decay=[0.1])]
    for x in bad:
        with pytest.raises(NitiError):
            _plan(niti, x)
    with pytest.raises(NitiError):
        niti.adamw(_plan(niti, dict(pr, decay=[-0.1, 0.0])), step, LR)
    assert all(torch.equal(a, b) for a, b in zip(p0, pr["p"]))
    niti.adamw(niti.adamw_tensors([], [], [], []), step, LR)                   # nothing to do
    assert niti.check() == 0
