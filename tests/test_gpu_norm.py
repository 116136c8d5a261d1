"""Norm, quantisation and their inverse against 64-bit definitions.

How far a float32 payload magnitude u < 128 can be off before it is rounded, in units of the result: the sum of squares of a
row passes through at most 32 (or C / 1024, long rows) sequential and 10 pairwise additions, half a relative step 2^-24
each, and half of that remains after the root; the reciprocal root, the mean, the two products and the scale add 8 steps.
"""
import numpy as np
import pytest
import torch

from floatref import check_payload, exponents, decode_e4m3

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _slack(C):
    return 128 * 2.0 ** -24 * ((max(32, C / 512) + 10) / 2 + 8)


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _np(t):
    return t.detach().double().cpu().numpy()


def _rows(seed, M, C, t):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, C), device="cuda", generator=g) * torch.exp(torch.randn((M, 1), device="cuda", generator=g))
    return x.to(t)


SIZES = [(1, 1), (1, 4096), (3, 8), (7, 33), (130, 1000), (257, 1001), (64, 2056), (5, 8192), (3, 16384), (2, 16400), (2, 5001),
         (700, 72), (2000, 16)]


@pytest.mark.parametrize("M,C", SIZES)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("mode", [0, 1])
def test_norm_forward(niti, M, C, kind, residual, rows, mode):
    t = TYPES[kind]
    x, gain = _rows(1, M, C, t), 1 + 0.3 * torch.randn(C, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    res = _rows(3, M, C, t) if residual else None
    y, s, h, rstd = niti.rmsnorm_fwd(x, gain, residual=res, rows=rows, eps=1e-5, round_mode=mode)
    hd = x if res is None else (x.float() + res.float()).to(t)
    assert torch.equal(h, hd)
    hd = _np(hd)
    r = 1 / np.sqrt((hd ** 2).mean(1) + 1e-5)
    # (half of the sum's error, and the root's)
    assert np.all(np.abs(_np(rstd) / r - 1) <= _slack(C) / 128)
    v = hd * r[:, None] * _np(gain)
    top = np.abs(v).max(1, keepdims=True) if rows else np.abs(v).max().reshape(1, 1)
    want = exponents(top)
    got = s.cpu().numpy().reshape(-1, 1)
    off = np.abs(np.log2(np.maximum(top, 1e-300)) - np.round(np.log2(np.maximum(top, 1e-300)))) > 1e-5     # away from powers of two
    assert np.array_equal(got[off], want[off])
    check_payload(y.cpu().numpy(), got, v, mode, _slack(C))
    assert niti.check() == 0


@pytest.mark.parametrize("place", ["x", "residual"])
def test_h_in_the_place_of_a_summand(niti, place):
    x, res = _rows(1, 300, 1024, torch.bfloat16), _rows(2, 300, 1024, torch.bfloat16)
    gain = torch.ones(1024, device="cuda")
    y0, s0, h0, _ = niti.rmsnorm_fwd(x, gain, residual=res)
    a, b = x.clone(), res.clone()
    y1, s1, h1, _ = niti.rmsnorm_fwd(a, gain, residual=b, h=a if place == "x" else b)
    assert torch.equal(h0, h1) and torch.equal(y0, y1) and torch.equal(s0, s1)


def test_zero_rows_have_exponent_zero_and_payload_zero(niti):
    x = torch.zeros((3, 64), device="cuda")
    x[1] = 1.0
    y, s, _, rstd = niti.rmsnorm_fwd(x, torch.ones(64, device="cuda"), eps=1e-6)
    assert s.tolist()[0] == 0 and s.tolist()[2] == 0 and not y[0].any() and not y[2].any() and y[1].any()
    assert abs(float(rstd[0]) - 1000) < 1
    q, s = niti.quantize(x, rows=False)
    assert int(s) == -6 and torch.equal(q.float() / 64, x)
    q, s = niti.quantize(torch.zeros((2, 5), device="cuda"))
    assert s.tolist() == [0, 0] and not q.any()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite_raise_the_status_and_stay_in_their_row(niti, bad):
    from paper_2009_13108_b200 import NitiError
    x = _rows(5, 4, 256, torch.float32)
    gain = torch.ones(256, device="cuda")
    y0, s0, _, _ = niti.rmsnorm_fwd(x, gain)
    niti.check()
    x[2, 17] = bad
    y1, s1, _, _ = niti.rmsnorm_fwd(x, gain)
    with pytest.raises(NitiError):
        niti.check()
    for row in (0, 1, 3):
        assert torch.equal(y0[row], y1[row]) and s0[row] == s1[row]
    q, s = niti.quantize(x)
    with pytest.raises(NitiError):
        niti.check()
    assert int(s[2]) == 121 and abs(int(q[2, 17])) == 127
    assert niti.check() == 0


def test_squares_beyond_the_float_range_raise_the_status(niti):
    from paper_2009_13108_b200 import NitiError
    niti.rmsnorm_fwd(torch.full((1, 64), 1e30, device="cuda"), torch.ones(64, device="cuda"))
    with pytest.raises(NitiError):
        niti.check()


@pytest.mark.parametrize("value", [1e-38, 2.0 ** -130, 3e38, 1.0, 127.99])
def test_extreme_magnitudes_keep_the_exponents_bounds(niti, value):
    x = torch.full((2, 32), value, device="cuda")
    q, s = niti.quantize(x)
    want = int(exponents(float(x[0, 0])))
    assert s.tolist() == [want, want]
    assert np.array_equal(_np(q), np.minimum(np.floor(_np(x) * 2.0 ** -want + 0.5), 127))
    assert niti.check() == 0


def test_rounding_to_nearest_is_exact_beside_halves(niti):
    """Magnitudes k + 1/2 and the floats around them, in units: 2^-25 below 1/2 is 0, and every half goes up."""
    half = np.arange(0, 127, dtype=np.float32) + np.float32(0.5)
    u = np.concatenate([half, np.nextafter(half, np.float32(0)), np.nextafter(half, np.float32(200))])
    u = np.concatenate([u, -u, [np.float32(127)]]).astype(np.float32)
    want = np.sign(u) * np.minimum(np.floor(np.abs(u.astype(np.float64)) + 0.5), 127)
    for pad in (0, 2):                                    # (rows of whole vectors, and of single elements)
        x = torch.from_numpy(np.pad(u, (0, -u.size % 4 + pad))).cuda().view(1, -1)
        q, s = niti.quantize(x)
        assert int(s) == 0 and np.array_equal(_np(q)[0, :u.size], want)


@pytest.mark.parametrize("C", [33, 256, 16400])
@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("power", [-123, -118, -90])
def test_rows_near_zero_with_a_tiny_eps(niti, C, rows, mode, power):
    """1 / rms is 1e6 here, and together with 2^100 and the 16 fraction bits it is no float32."""
    x = _rows(31, 5, C, torch.float32) * 2.0 ** power
    x[:, ::3] = 0
    x[3] = 0
    gain = 1 + 0.3 * torch.randn(C, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    y, s, _, rstd = niti.rmsnorm_fwd(x, gain, rows=rows, eps=1e-12, round_mode=mode)
    v = _np(x) * _np(gain) / np.sqrt((_np(x) ** 2).mean(1, keepdims=True) + float(np.float32(1e-12)))
    top = np.abs(v).max(1, keepdims=True) if rows else np.abs(v).max().reshape(1, 1)
    assert np.array_equal(s.cpu().numpy().reshape(-1, 1), exponents(top))
    # (products below 2^-126 lose bits: up to 2^-150 of h gain, times 1e6 and 2^100, in units)
    check_payload(y.cpu().numpy(), s.cpu().numpy().reshape(-1, 1), v, mode, _slack(C) + 2.0 ** -149 * 1e6 * 2.0 ** 100)
    assert not y[:, ::3].any() and not y[3].any() and niti.check() == 0


@pytest.mark.parametrize("C", [256, 16400])
def test_backward_of_rows_near_zero(niti, C):
    """r is 2^50: its cube is no float32, what it is multiplied with makes the product one."""
    h, dy = _rows(32, 3, C, torch.float32) * 2.0 ** -50, _rows(33, 3, C, torch.float32) * 2.0 ** -50
    rstd = torch.rsqrt(h.double().square().mean(1)).float()
    dx, _ = niti.rmsnorm_bwd(dy, h, torch.ones(C, device="cuda"), rstd)
    H, Y, r = _np(h), _np(dy), _np(rstd)[:, None]
    want = r * Y - H * r ** 3 * (Y * H).mean(1, keepdims=True)
    terms = np.abs(r * Y) + np.abs(H) * r ** 3 * np.abs(Y * H).mean(1, keepdims=True)
    assert np.all(np.abs(_np(dx) - want) <= terms * (max(32, C / 512) + 20) * 2.0 ** -24)


def test_dequantize_at_the_ends_of_the_exponents(niti):
    q = torch.tensor([[0, 1, 127, -127] * 8] * 6, dtype=torch.int8, device="cuda")
    s = torch.tensor([127, 200, -126, -127, -128, -200], dtype=torch.int32, device="cuda")
    for shape in (q, q[:, :4].contiguous()):
        v = _np(niti.dequantize(shape, s))
        want = _np(shape) * np.exp2(np.clip(s.cpu().numpy().astype(float), -128, 127))[:, None]
        want[np.abs(want) >= 2.0 ** 128] = np.inf * np.sign(want[np.abs(want) >= 2.0 ** 128])
        assert np.array_equal(v, want)
    one = niti.dequantize(torch.tensor(5, dtype=torch.int8, device="cuda"), s[2:3])
    assert one.shape == () and float(one) == 5 * 2.0 ** -126


def test_calls_without_rows_do_nothing(niti):
    gain = torch.ones(64, device="cuda")
    y, s, h, rstd = niti.rmsnorm_fwd(torch.empty((0, 64), device="cuda"), gain)
    assert y.shape == (0, 64) and s.numel() == 0 and rstd.numel() == 0
    empty = torch.empty((0, 64), device="cuda")
    dx, dgain = niti.rmsnorm_bwd(empty, empty, gain, torch.empty(0, device="cuda"), dgain=torch.ones(64, device="cuda"))
    assert dx.shape == (0, 64) and not dgain.any()
    assert niti.dequantize(torch.empty((0, 4), dtype=torch.int8, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 4)


@pytest.mark.parametrize("M,C", SIZES)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("with_dh", [False, True])
def test_norm_backward(niti, M, C, kind, with_dh):
    t = TYPES[kind]
    h, dy = _rows(1, M, C, t), _rows(2, M, C, t)
    dh = _rows(3, M, C, t) if with_dh else None
    gain = 1 + 0.3 * torch.randn(C, device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    dx, dgain = niti.rmsnorm_bwd(dy, h, gain, rstd, dh=dh)
    H, Y, G, r = _np(h), _np(dy), _np(gain), _np(rstd)[:, None]
    d = _np(dh) if with_dh else 0.0
    gy = Y * G
    mean = (gy * H).mean(1, keepdims=True)
    want = d + (r * gy - H * r ** 3 * mean)
    # each term is off by a few relative steps of float32, the mean by its summation; then the rounding to the type
    steps = (max(32, C / 512) + 20) * 2.0 ** -24
    terms = np.abs(d) + np.abs(r * gy) + np.abs(H) * r ** 3 * np.abs(gy * H).mean(1, keepdims=True)
    tiny = 2.0 ** -25 if t == torch.float16 else 2.0 ** -133
    bound = terms * steps + np.abs(want) * torch.finfo(t).eps / 2 * (1 + 2.0 ** -10) + tiny
    assert np.all(np.abs(_np(dx) - want) <= bound)
    contrib = Y * (H * r)
    # rows are added one after the other in at most M steps, blocks then in at most 320 / 8 + 8
    bound = np.abs(contrib).sum(0) * (min(M, M / 100 + 64) + 50) * 2.0 ** -24 + 1e-30
    assert np.all(np.abs(_np(dgain) - contrib.sum(0)) <= bound)
    again = niti.rmsnorm_bwd(dy, h, gain, rstd, dh=dh)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain)          # the same order of additions
    alone, none = niti.rmsnorm_bwd(dy, h, gain, rstd, dh=dh, need_dgain=False)
    assert none is None and torch.equal(alone, dx)


def test_norm_backward_is_the_derivative(niti):
    """Against central differences of the 64-bit norm (error of order step^2 = 1e-8 of the third derivative)."""
    M, C = 3, 40
    h, w = _rows(7, M, C, torch.float32), _rows(8, M, C, torch.float32)
    gain = 1 + 0.2 * torch.randn(C, device="cuda", generator=torch.Generator("cuda").manual_seed(9))
    rstd = torch.rsqrt(h.square().mean(1) + 1e-3)
    dx, dgain = niti.rmsnorm_bwd(w, h, gain, rstd)

    def loss(hh, gg):
        return float((hh / np.sqrt((hh ** 2).mean(1, keepdims=True) + 1e-3) * gg * W).sum())

    H, W, G = _np(h), _np(w), _np(gain)
    for (i, j) in [(0, 0), (1, 7), (2, 39)]:
        e = np.zeros_like(H)
        e[i, j] = 1e-4
        assert abs((loss(H + e, G) - loss(H - e, G)) / 2e-4 - float(dx[i, j])) <= 1e-5 * np.abs(W[i]).sum()
    e = np.zeros(C)
    e[11] = 1e-4
    assert abs((loss(H, G + e) - loss(H, G - e)) / 2e-4 - float(dgain[11])) <= 1e-5 * np.abs(W).sum()


@pytest.mark.parametrize("place", ["dy", "dh", "h"])
@pytest.mark.parametrize("C", [1024, 16400])
def test_dx_in_the_place_of_an_operand(niti, place, C):
    t = {"dy": _rows(1, 200, C, torch.bfloat16), "h": _rows(2, 200, C, torch.bfloat16), "dh": _rows(3, 200, C, torch.bfloat16)}
    gain, rstd = torch.ones(C, device="cuda"), torch.rsqrt(t["h"].float().square().mean(1))
    dx0, dg0 = niti.rmsnorm_bwd(t["dy"], t["h"], gain, rstd, dh=t["dh"])
    c = {k: v.clone() for k, v in t.items()}
    dx1, dg1 = niti.rmsnorm_bwd(c["dy"], c["h"], gain, rstd, dh=c["dh"], dx=c[place])
    assert torch.equal(dx0, dx1) and torch.equal(dg0, dg1)


@pytest.mark.parametrize("offset", [1, 2, 4])
def test_tensors_that_start_anywhere(niti, offset):
    """Slices of a larger buffer whose first byte is on no 16-byte boundary."""
    M, C = 33, 256
    whole = _rows(1, 1, M * C + 8, torch.bfloat16).view(-1)
    x = whole[offset:offset + M * C].view(M, C)
    gain = torch.ones(C, device="cuda")
    y0, s0, _, r0 = niti.rmsnorm_fwd(x.clone(), gain, round_mode=0)
    y1, s1, _, r1 = niti.rmsnorm_fwd(x, gain, round_mode=0)
    # (another order of the sums: the payloads of both are the definition's, the roots equal to a few steps)
    assert torch.allclose(r0, r1, rtol=2.0 ** -18, atol=0) and (y0.int() - y1.int()).abs().max() <= 1
    d0 = niti.rmsnorm_bwd(x.clone(), x.clone(), gain, r0)[0]
    d1 = niti.rmsnorm_bwd(x, x, gain, r0)[0]
    assert torch.allclose(d0.float(), d1.float(), rtol=2.0 ** -7, atol=1e-4)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("M,C", SIZES)
def test_quantize_and_back(niti, kind, rows, M, C):
    x = _rows(11, M, C, TYPES[kind])
    q, s = niti.quantize(x, rows=rows)
    top = np.abs(_np(x)).max(1, keepdims=True) if rows else np.abs(_np(x)).max().reshape(1, 1)
    e = exponents(top)
    assert np.array_equal(s.cpu().numpy().reshape(-1, 1), e)
    want = np.sign(_np(x)) * np.minimum(np.floor(np.abs(_np(x)) * np.exp2(-e.astype(float)) + 0.5), 127)
    assert np.array_equal(_np(q), want)                   # (scaling by a power of two is exact)
    for out_kind, t in TYPES.items():
        if out_kind == "f16" and np.abs(want * np.exp2(e.astype(float))).max() > 6e4:
            continue
        v = niti.dequantize(q, s, dtype=t)
        exact = want * np.exp2(e.astype(float))
        if out_kind == "f16":
            assert np.all(np.abs(_np(v) - exact) <= 2.0 ** -25)              # (subnormals)
        else:
            assert np.array_equal(_np(v), exact)
    assert niti.check() == 0


def test_quantize_float32_pseudo_stochastic(niti):
    x = _rows(12, 100, 500, torch.float32)
    q, s = niti.quantize(x, round_mode=0)
    share = check_payload(q.cpu().numpy(), s.cpu().numpy().reshape(-1, 1), _np(x), 0, 0.0)
    assert share > 0.95
    err = (_np(q) - _np(x) * np.exp2(-s.cpu().numpy().astype(float))[:, None])
    # (uniform discarded bits: rounded up less often by the ties of the two halves, 2^-9 a value; 50000 values of variance 1 / 4)
    assert abs((err * np.sign(_np(x))).mean()) < 2.0 ** -9 + 5 * 0.5 / np.sqrt(err.size)


@pytest.mark.parametrize("n,block", [(256, 256), (1000, 256), (4096, 256), (77, 16), (100, 7)])
def test_dequantize_codes(niti, n, block):
    g = np.random.default_rng(n)
    code = g.integers(0, 256, n).astype(np.uint8)
    code[(code & 127) == 127] = 0                         # (not a code)
    s = g.integers(-30, 30, -(-n // block)).astype(np.int8)
    v = niti.dequantize(torch.from_numpy(code).cuda(), torch.from_numpy(s).cuda(), dtype=torch.float32, block=block)
    assert np.array_equal(_np(v), decode_e4m3(code, s, block))


def test_refusals(niti):
    from paper_2009_13108_b200 import NitiError
    x, gain = _rows(1, 4, 64, torch.bfloat16), torch.ones(64, device="cuda")
    r = torch.ones(4, device="cuda")
    wrong = [lambda: niti.rmsnorm_fwd(x, gain[:32]), lambda: niti.rmsnorm_fwd(x, gain.double()), lambda: niti.rmsnorm_fwd(x.double(), gain),
             lambda: niti.rmsnorm_fwd(x.t(), gain), lambda: niti.rmsnorm_fwd(x, gain, residual=x.float()),
             lambda: niti.rmsnorm_fwd(x, gain, h=x), lambda: niti.rmsnorm_fwd(x.cpu(), gain), lambda: niti.rmsnorm_fwd(x, gain, eps=-1.0),
             lambda: niti.rmsnorm_fwd(x, gain, eps=float("nan")), lambda: niti.rmsnorm_fwd(x, gain, round_mode=2),
             lambda: niti.rmsnorm_bwd(x, x.float(), gain, r), lambda: niti.rmsnorm_bwd(x, x, gain, r[:2]),
             lambda: niti.quantize(x, round_mode=0), lambda: niti.quantize(x[:, ::2]),
             lambda: niti.dequantize(x, torch.zeros(1, dtype=torch.int32, device="cuda")),
             lambda: niti.dequantize(torch.zeros((4, 4), dtype=torch.int8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))]
    before = niti.launch_count()
    for call in wrong:
        with pytest.raises(NitiError):
            call()
    assert niti.launch_count() == before and niti.check() == 0


@pytest.mark.parametrize("rows", [True, False])
def test_captured_calls_replay_on_new_inputs(niti, rows):
    x, gain = _rows(1, 64, 512, torch.bfloat16), torch.ones(512, device="cuda")
    out = niti.rmsnorm_fwd(x, gain, rows=rows)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        y, s, _, _ = niti.rmsnorm_fwd(x, gain, rows=rows)
    torch.cuda.current_stream().wait_stream(side)
    keep = niti.buffers()
    for k in range(3):
        x.copy_(_rows(20 + k, 64, 512, torch.bfloat16))
        graph.replay()
        y0, s0, _, _ = niti.rmsnorm_fwd(x, gain, rows=rows)
        assert torch.equal(y, y0) and torch.equal(s, s0)
    del keep, out
