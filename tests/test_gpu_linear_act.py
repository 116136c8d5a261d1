"""Fully connected layers with a float epilogue and their backward pass, against 64-bit definitions.

int32 sums and the scale are exact.  z = sum 2^s + bias is off by a step 2^-24 of each term; activations and their slopes by
2^-20 of their argument's size (polynomial 7.1.26 of Abramowitz and Stegun 0.75e-7, hardware exponential and division a few
steps of 2^-22 each on factors of at most one); results then round to their type."""
import numpy as np
import pytest
import torch

from floatref import exponents, round_units, steady

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEP = 2.0 ** -24
ACT_STEP = 2.0 ** -20


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _np(t):
    return t.detach().double().cpu().numpy()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i8(seed, *shape):
    return torch.randint(-127, 128, shape, device="cuda", generator=_gen(seed), dtype=torch.int32).to(torch.int8)


def _exp(M, rows, K, seed=5):
    base = -round(np.log2(73 * 73 * np.sqrt(K)) / 2)
    if rows:
        return torch.randint(base - 1, base + 2, (M,), device="cuda", generator=_gen(seed), dtype=torch.int32)
    return torch.full((1,), base, device="cuda", dtype=torch.int32)


def _act(z, act):
    """Values and slopes in 64 bits."""
    t = torch.from_numpy(z)
    if act == "relu":
        return np.maximum(z, 0), (z > 0).astype(float)
    if act == "gelu":
        cdf = torch.special.ndtr(t).numpy()
        return z * cdf, cdf + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if act == "silu":
        s = torch.sigmoid(t).numpy()
        return z * s, s * (1 + z * (1 - s))
    return z, np.ones_like(z)


def _half_step(want, t):
    """Rounding to a type: half a step of the value, or of the smallest numbers."""
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[t]
    return np.abs(want) * torch.finfo(t).eps / 2 * (1 + 2.0 ** -8) + tiny


def _matmul(a, b):
    """a b^T of whole numbers, exact in 64 bits."""
    return (a.double() @ b.double().t()).cpu().numpy()


def _check_forward(niti, M, N, K, kind, act, rows, bias, residual, keep_z, seed=0):
    t = TYPES[kind]
    a, w = _i8(seed + 1, M, K), _i8(seed + 2, N, K)
    s_a, s_w = _exp(M, rows, K), torch.full((1,), -round(np.log2(73 * 73 * np.sqrt(K)) / 2), device="cuda", dtype=torch.int32)
    b = torch.randn(N, device="cuda", generator=_gen(3)) if bias else None
    res = torch.randn((M, N), device="cuda", generator=_gen(4)).to(t) if residual else None
    out, z = niti.linear_act_fwd(a, s_a, w, s_w, bias=b, residual=res, act=act, keep_z=keep_z, dtype=t)
    prod = _matmul(a, w) * np.exp2(_np(s_a) + _np(s_w))[:, None]
    want_z = prod + (_np(b) if bias else 0.0)
    z_off = STEP * (np.abs(prod) + np.abs(want_z))
    want, _ = _act(want_z, act)
    off = 1.2 * z_off + (ACT_STEP * np.abs(want_z) if act in ("gelu", "silu") else 0.0)      # (slopes are at most 1.13)
    if residual:
        want = want + _np(res)
    off = off + 2 * STEP * np.abs(want)
    assert np.all(np.abs(_np(out) - want) <= off + _half_step(np.abs(want) + off, t))
    if keep_z:
        assert np.all(np.abs(_np(z) - want_z) <= z_off + _half_step(np.abs(want_z) + z_off, t))
    else:
        assert z is None
    assert niti.check() == 0


SIZES = [(1, 1, 1), (1, 32, 32), (1, 4096, 4096), (3, 5, 7), (2, 1000, 512), (16, 4096, 512), (31, 48, 100), (64, 2048, 1024), (128, 256, 128),
         (130, 1000, 777), (17, 10, 256), (513, 96, 1000), (300, 520, 40), (700, 700, 64), (2048, 512, 4096), (257, 33, 16),
         (1100, 2064, 96), (150, 3000, 2000), (8, 20000, 128), (5000, 24, 300), (100, 100, 20000)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("kind", TYPES)
def test_forward(niti, M, N, K, kind):
    for i, (act, rows, bias, residual, keep_z) in enumerate([("none", True, False, False, False), ("gelu", True, True, True, True),
                                                             ("silu", False, True, False, False), ("relu", False, False, True, True)]):
        _check_forward(niti, M, N, K, kind, act, rows, bias, residual, keep_z, seed=10 * i)


def test_the_largest_sums_are_exact(niti):
    """127 * 127 * 131072 stays below 2^31, in a sum that is split over CTAs."""
    M, N, K = 2, 64, 131072
    a = torch.full((M, K), 127, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), 127, dtype=torch.int8, device="cuda")
    w[::2] = -127
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = niti.linear_act_fwd(a, zero, w, zero, dtype=torch.float32)
    want = 127.0 * 127 * K
    assert abs(want) < 2 ** 31
    assert out[:, 1::2].eq(float(np.float32(want))).all() and out[:, ::2].eq(-float(np.float32(want))).all()


def test_out_in_the_place_of_the_residual(niti):
    for M, N, K in ((200, 512, 256), (33, 77, 50), (1, 256, 256)):
        a, w, s = _i8(1, M, K), _i8(2, N, K), torch.full((1,), -8, dtype=torch.int32, device="cuda")
        res = torch.randn((M, N), device="cuda", generator=_gen(3)).to(torch.bfloat16)
        want, _ = niti.linear_act_fwd(a, s, w, s, residual=res, act="gelu")
        got, _ = niti.linear_act_fwd(a, s, w, s, residual=res, act="gelu", out=res)
        assert got is res and torch.equal(want, got)


def test_results_do_not_depend_on_the_other_rows(niti):
    """With an exponent per row, a row alone and the same row in a batch give the same bits (sums are exact)."""
    N, K = 1536, 1024
    a, w = _i8(1, 300, K), _i8(2, N, K)
    s_a, s_w = _exp(300, True, K), torch.full((1,), -9, dtype=torch.int32, device="cuda")
    whole, _ = niti.linear_act_fwd(a, s_a, w, s_w, act="silu")
    for lo, hi in ((0, 1), (7, 9), (100, 116), (30, 94), (0, 129)):
        part, _ = niti.linear_act_fwd(a[lo:hi].contiguous(), s_a[lo:hi].contiguous(), w, s_w, act="silu")
        assert torch.equal(part, whole[lo:hi])


@pytest.mark.parametrize("M,N,K", [(8, 520, 3001), (9, 4400, 3001), (16, 512, 3001), (17, 600, 3001), (32, 520, 3001), (12, 12304, 4096), (32, 6144, 4096),
                                   (20, 7136, 2048), (20, 7136, 512)])
def test_few_rows_of_large_layers(niti, M, N, K):
    """On both sides of the sizes from which on a few rows go by tiles, and each row as it is alone."""
    _check_forward(niti, M, N, K, "bf16", "gelu", True, True, True, True)
    a, w = _i8(1, M, K), _i8(2, N, K)
    s_a, s_w = _exp(M, True, K), _exp(1, False, K)
    out, _ = niti.linear_act_fwd(a, s_a, w, s_w, dtype=torch.float32)
    for m in (0, M - 1):
        one, _ = niti.linear_act_fwd(a[m:m + 1].clone(), s_a[m:m + 1].clone(), w, s_w, dtype=torch.float32)
        assert torch.equal(one[0], out[m])


def test_rows_behind_the_last_one_stay(niti):
    M, N, K = 37, 100, 64
    a, w, s = _i8(1, M, K), _i8(2, N, K), torch.full((1,), -8, dtype=torch.int32, device="cuda")
    buf = torch.full((M * N + 200,), 5.0, dtype=torch.bfloat16, device="cuda")
    niti.linear_act_fwd(a, s, w, s, out=buf[:M * N].view(M, N))
    assert (buf[M * N:] == 5.0).all()


def test_exponent_sums_beyond_int8_raise_the_status(niti):
    from paper_2009_13108_b200 import NitiError
    for sa in (-100, 100):
        for M in (3, 200):
            a, w = _i8(1, M, 64), _i8(2, 64, 64)
            s = torch.full((1,), sa, dtype=torch.int32, device="cuda")
            niti.linear_act_fwd(a, s, w, s)
            with pytest.raises(NitiError):
                niti.check()
    assert niti.check() == 0


def _check_backward(niti, M, N, K, kind, act, mode, dw_kind, seed=0):
    t, tw = TYPES[kind], TYPES[dw_kind]
    a, w = _i8(seed + 1, M, K), _i8(seed + 2, N, K)
    s_a, s_w = torch.full((1,), -9, dtype=torch.int32, device="cuda"), torch.full((1,), -8, dtype=torch.int32, device="cuda")
    z = torch.randn((M, N), device="cuda", generator=_gen(seed + 3)).to(t) if act != "none" else None
    dout = (0.1 * torch.randn((M, N), device="cuda", generator=_gen(seed + 4))).to(t)
    dx, dw, dbias = niti.linear_act_bwd(a, s_a, w, s_w, dout, z=z, act=act, dw_dtype=tw, round_mode=mode)
    D = _np(dout)
    slope = _act(_np(z), act)[1] if z is not None else np.ones_like(D)
    e = D * slope
    inexact = act in ("gelu", "silu")
    e_off = (np.abs(D) * ACT_STEP * (1 + np.abs(_np(z))) + STEP * np.abs(e)) if inexact else np.zeros_like(e)
    s_e = int(exponents(np.abs(e).max()))
    u = np.abs(e) * 2.0 ** -s_e
    sure = steady(u, e_off.max() * 2.0 ** -s_e, mode) if inexact else np.ones_like(e, dtype=bool)
    q = np.sign(e) * np.minimum(round_units(u, mode), 127)
    # where float32 may decide otherwise the payload can be one off
    loose = torch.from_numpy((~sure).astype(np.float64)).cuda()
    Q, A, W = torch.from_numpy(q).cuda(), a.double(), w.double()
    for got, exact, room, s, typ in ((dx, Q @ W, loose @ W.abs(), s_e - 8, t), (dw, Q.t() @ A, loose.t() @ A.abs(), s_e - 9, tw)):
        want, room = exact.cpu().numpy() * 2.0 ** s, room.cpu().numpy() * 2.0 ** s
        off = room + STEP * np.abs(want)
        assert np.all(np.abs(_np(got) - want) <= off + _half_step(np.abs(want) + off, typ))
    rows = M / 64 + 200
    assert np.all(np.abs(_np(dbias) - e.sum(0)) <= np.abs(e).sum(0) * rows * STEP + e_off.sum(0))
    assert niti.check() == 0
    again = niti.linear_act_bwd(a, s_a, w, s_w, dout, z=z, act=act, dw_dtype=tw, round_mode=mode)
    assert all(torch.equal(x, y) for x, y in zip((dx, dw, dbias), again))


BWD_SIZES = [(1, 1, 1), (1, 64, 32), (5, 7, 3), (128, 256, 128), (130, 1000, 777), (64, 10, 256), (1000, 96, 100), (300, 520, 40),
             (2000, 520, 256), (4096, 128, 64), (257, 33, 2000), (512, 2048, 640)]


@pytest.mark.parametrize("M,N,K", BWD_SIZES)
@pytest.mark.parametrize("kind", TYPES)
def test_backward(niti, M, N, K, kind):
    for i, (act, mode, dw_kind) in enumerate([("none", 1, "f32"), ("gelu", 0, "bf16"), ("silu", 1, "f32"), ("relu", 1, "f16")]):
        _check_backward(niti, M, N, K, kind, act, mode, dw_kind, seed=20 * i)


@pytest.mark.parametrize("act", ["none", "relu"])
def test_backward_pseudo_stochastic_float32(niti, act):
    _check_backward(niti, 300, 200, 100, "f32", act, 0, "f32")


def test_backward_is_the_derivative(niti):
    """The exact gradients against central differences of the layer in 64 bits, and the returned ones within the rounding of
    the error to int8 (half a step 2^s_e per element)."""
    M, N, K = 6, 5, 9
    a, w = _i8(1, M, K), _i8(2, N, K)
    s_a, s_w = torch.full((1,), -7, dtype=torch.int32, device="cuda"), torch.full((1,), -7, dtype=torch.int32, device="cuda")
    b = 0.1 * torch.randn(N, device="cuda", generator=_gen(3))
    dout = torch.randn((M, N), device="cuda", generator=_gen(4))
    for act in ("gelu", "silu"):
        out, z = niti.linear_act_fwd(a, s_a, w, s_w, bias=b, act=act, keep_z=True, dtype=torch.float32)
        dx, dw, db = niti.linear_act_bwd(a, s_a, w, s_w, dout, z=z, act=act)
        A, W, B, D = _np(a) * 2.0 ** -7, _np(w) * 2.0 ** -7, _np(b), _np(dout)

        def loss(A, W, B):
            return (_act(A @ W.T + B, act)[0] * D).sum()

        e = D * _act(A @ W.T + B, act)[1]
        step = 2.0 ** int(exponents(np.abs(e).max()))
        h = 1e-5
        for got, room, vary in ((dx, 0.51 * step * np.abs(W).sum(0)[None], 0), (dw, 0.51 * step * np.abs(A).sum(0)[None], 1),
                                (db, 1e-4 * np.ones((1, N)), 2)):
            base = [A, W, B][vary]
            num = np.zeros_like(base)
            for i in np.ndindex(base.shape):
                d = np.zeros_like(base)
                d[i] = h
                args = [A, W, B]
                args[vary] = base + d
                up = loss(*args)
                args[vary] = base - d
                num[i] = (up - loss(*args)) / (2 * h)
            assert np.all(np.abs(_np(got) - num) <= room + 1e-6)


def test_parts_of_the_backward_pass(niti):
    M, N, K = 200, 96, 160
    a, w, s = _i8(1, M, K), _i8(2, N, K), torch.full((1,), -8, dtype=torch.int32, device="cuda")
    dout = torch.randn((M, N), device="cuda", generator=_gen(3)).to(torch.bfloat16)
    dx, dw, db = niti.linear_act_bwd(a, s, w, s, dout)
    none, dw1, db1 = niti.linear_act_bwd(a, s, w, s, dout, need_dx=False)
    assert none is None and torch.equal(dw, dw1) and torch.equal(db, db1)
    sq = _i8(4, N, M).t().contiguous()                                     # [M][N] operand: dx in the place of dout
    ww = _i8(5, N, N)
    want = niti.linear_act_bwd(sq, s, ww, s, dout)[0]
    got = niti.linear_act_bwd(sq, s, ww, s, dout, dx=dout)[0]
    assert got is dout and torch.equal(want, got)


def test_zero_errors_and_errors_that_are_not_finite(niti):
    from paper_2009_13108_b200 import NitiError
    M, N, K = 40, 48, 32
    a, w, s = _i8(1, M, K), _i8(2, N, K), torch.full((1,), -8, dtype=torch.int32, device="cuda")
    dout = torch.zeros((M, N), device="cuda")
    dx, dw, db = niti.linear_act_bwd(a, s, w, s, dout)
    assert not dx.any() and not dw.any() and not db.any() and niti.check() == 0
    for bad in (float("nan"), float("inf")):
        dout[3, 4] = bad
        niti.linear_act_bwd(a, s, w, s, dout)
        with pytest.raises(NitiError):
            niti.check()


def test_no_rows(niti):
    a, w, s = torch.empty((0, 64), dtype=torch.int8, device="cuda"), _i8(2, 32, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    out, z = niti.linear_act_fwd(a, s, w, s, keep_z=True)
    assert out.shape == (0, 32) and z.shape == (0, 32)
    dx, dw, db = niti.linear_act_bwd(a, s, w, s, torch.empty((0, 32), device="cuda"), dw=torch.ones((32, 64), device="cuda"))
    assert dx.shape == (0, 64) and not dw.any() and not db.any()


def test_refusals(niti):
    from paper_2009_13108_b200 import NitiError
    M, N, K = 8, 16, 32
    a, w, s = _i8(1, M, K), _i8(2, N, K), torch.zeros(1, dtype=torch.int32, device="cuda")
    r = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    wide = _i8(3, M, 131073)
    wrong = [lambda: niti.linear_act_fwd(a, s, _i8(2, N, K + 1), s), lambda: niti.linear_act_fwd(a.int(), s, w, s),
             lambda: niti.linear_act_fwd(a, s.float(), w, s), lambda: niti.linear_act_fwd(a, torch.zeros(3, dtype=torch.int32, device="cuda"), w, s),
             lambda: niti.linear_act_fwd(a, s, w, torch.zeros(N, dtype=torch.int32, device="cuda")), lambda: niti.linear_act_fwd(a, s, w, s, act="tanh"),
             lambda: niti.linear_act_fwd(a, s, w, s, residual=r.float()), lambda: niti.linear_act_fwd(a, s, w, s, bias=torch.zeros(N + 1, device="cuda")),
             lambda: niti.linear_act_fwd(a.t(), s, w, s), lambda: niti.linear_act_fwd(a.cpu(), s, w, s),
             lambda: niti.linear_act_fwd(a, s, w, s, out=r, z=r), lambda: niti.linear_act_fwd(a, s, w, s, residual=r, z=r),
             lambda: niti.linear_act_fwd(_i8(1, 1, 1 + M * K).view(-1)[1:].view(M, K), s, w, s),
             lambda: niti.linear_act_fwd(wide, s, _i8(4, N, 131073), s), lambda: niti.linear_act_fwd(a, s, w, s, dtype=torch.float64),
             lambda: niti.linear_act_bwd(a, s, w, s, r, act="gelu"), lambda: niti.linear_act_bwd(a, s, w, s, r, round_mode=0),
             lambda: niti.linear_act_bwd(a, s, w, s, r, z=r, act="relu", round_mode=0),
             lambda: niti.linear_act_bwd(a, torch.zeros(M, dtype=torch.int32, device="cuda"), w, s, r),
             lambda: niti.linear_act_bwd(a, s, w, s, r, z=r.float(), act="gelu"), lambda: niti.linear_act_bwd(a, s, w, s, r[:4]),
             lambda: niti.linear_act_bwd(a, s, w, s, r, dw=torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"))]
    before = niti.launch_count()
    for call in wrong:
        with pytest.raises(NitiError):
            call()
    assert niti.launch_count() == before and niti.check() == 0


def test_captured_layers_replay_on_new_inputs(niti):
    """Forward and backward of one layer in a graph, split contractions among them, next to eager calls on the same workspace."""
    M, N, K = 300, 256, 2048
    a, w, s = _i8(1, M, K), _i8(2, N, K), torch.full((1,), -9, dtype=torch.int32, device="cuda")
    dout = torch.randn((M, N), device="cuda", generator=_gen(3)).to(torch.bfloat16)

    def both():
        out, z = niti.linear_act_fwd(a, s, w, s, act="gelu", keep_z=True)
        return (out, z) + niti.linear_act_bwd(a, s, w, s, dout, z=z, act="gelu", round_mode=0)

    both()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    keep = niti.buffers()
    for k in range(3):
        a.copy_(_i8(30 + k, M, K))
        dout.copy_(torch.randn((M, N), device="cuda", generator=_gen(40 + k)))
        graph.replay()
        for x, y in zip(got, both()):
            assert torch.equal(x, y)
    del keep
