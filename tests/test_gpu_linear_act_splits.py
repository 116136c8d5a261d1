"""The linear layer's multiplies where a contraction is split over CTAs: sums at the end of int32, both multiplies of a backward
pass at once, sizes in turn on one workspace; and operands that start between vectors."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i8(seed, *shape):
    return torch.randint(-127, 128, shape, device="cuda", generator=_gen(seed), dtype=torch.int32).to(torch.int8)


def _s(v):
    return torch.full((1,), v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("M,N", [(64, 64), (33, 50), (200, 96)])
def test_the_largest_sums_of_tiles_are_exact(niti, M, N):
    """127 * 127 * 131072 stays below 2^31 in the sums of a tile whose contraction many CTAs share (the rows are too many to be
    streamed), with signs that cancel inside the shares of some columns and between the shares of others."""
    K = 131072
    assert 127 * 127 * K < 2 ** 31
    a = torch.full((M, K), 127, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), 127, dtype=torch.int8, device="cuda")
    w[1::4] = -127
    w[2::4, K // 2:] = -127
    w[3::4, ::2] = -127
    w[3::4, 0] = 127
    want = (a[:1].double() @ w.double().t()).float()
    assert float(want[0, 0]) == np.float32(127.0 * 127 * K) and float(want[0, 3]) != 0
    for k in range(3):
        out, _ = niti.linear_act_fwd(a, _s(0), w, _s(0), dtype=torch.float32)
        assert torch.equal(out, want.expand(M, N)), k
        small, _ = niti.linear_act_fwd(a[:, :4096].contiguous(), _s(0), w[:, :4096].contiguous(), _s(0), dtype=torch.float32)
        assert torch.equal(small, (a[:1, :4096].double() @ w[:, :4096].double().t()).float().expand(M, N)), k
    assert niti.check() == 0


def _backward(niti, M, N, K, seed, dw_dtype=torch.float32, dtype=torch.float32):
    """Errors that are payloads already: nothing is rounded, and both products are exact sums."""
    a, w, e = _i8(seed, M, K), _i8(seed + 1, N, K), _i8(seed + 2, M, N)
    e[0, 0] = 127
    dx, dw, db = niti.linear_act_bwd(a, _s(-3), w, _s(-5), e.to(dtype), dw_dtype=dw_dtype)
    want_x, want_w = (e.double() @ w.double()) * 2.0 ** -5, (e.double().t() @ a.double()) * 2.0 ** -3
    assert torch.equal(dx, want_x.float().to(dtype)) and torch.equal(dw, want_w.float().to(dw_dtype))
    assert torch.equal(db.double(), e.double().sum(0))


# both contractions (over N for dx, over M for dw) are long and the output tiles are few: two or three shares each
SPLIT = [(2900, 2600, 64), (3500, 3500, 60), (2600, 2700, 33), (4100, 3000, 48), (3000, 4200, 64), (4096, 3400, 16)]


@pytest.mark.parametrize("M,N,K", SPLIT)
def test_both_backward_contractions_split(niti, M, N, K):
    _backward(niti, M, N, K, 1)


def test_split_sizes_take_turns(niti):
    """Counters and slabs of one call must not show in the next."""
    for k in range(4):
        for i, (M, N, K) in enumerate(SPLIT):
            _backward(niti, M, N, K, 10 * k + i, dw_dtype=torch.bfloat16 if k & 1 else torch.float32, dtype=torch.bfloat16 if k & 2 else torch.float32)
    niti.begin_step()
    for M, N, K in SPLIT:
        _backward(niti, M, N, K, 50)
    niti.end_step()
    assert niti.check() == 0


def _shifted(t, off=1):
    """The same matrix `off` elements behind a vector boundary."""
    buf = torch.empty(t.numel() + off, dtype=t.dtype, device="cuda")
    buf[off:] = t.reshape(-1)
    return buf[off:].view(t.shape)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M", [3, 20, 300])
def test_forward_tensors_between_vectors(niti, M, dtype):
    """Widths of whole vectors, one tensor at a time off its boundary: the results of the aligned call."""
    N, K = 512, 256
    a, w, b = _i8(1, M, K), _i8(2, N, K), torch.randn(N, device="cuda", generator=_gen(3))
    res = torch.randn((M, N), device="cuda", generator=_gen(4)).to(dtype)
    call = lambda **kw: niti.linear_act_fwd(a, _s(-8), w, _s(-7), act="gelu", keep_z=True, dtype=dtype,               # noqa: E731
                                            **{**dict(bias=b, residual=res), **kw})
    out, z = call()
    spare = torch.empty((M, N), dtype=dtype, device="cuda")
    for kw in (dict(out=_shifted(spare)), dict(z=_shifted(spare)), dict(residual=_shifted(res)), dict(bias=_shifted(b)), dict(out=_shifted(spare, 3), residual=_shifted(res, 5))):
        got, gz = call(**kw)
        assert torch.equal(got, out) and torch.equal(gz, z), list(kw)
    assert niti.check() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_backward_tensors_between_vectors(niti, dtype):
    """dbias is summed by other threads then, so that it agrees to rounding only: a column of 300 numbers below 1, the
    differences of partial sums at most 300 steps each."""
    M, N, K = 300, 512, 256
    a, w = _i8(1, M, K), _i8(2, N, K)
    dout = torch.rand((M, N), device="cuda", generator=_gen(3)).to(dtype)
    z = torch.randn((M, N), device="cuda", generator=_gen(4)).to(dtype)
    call = lambda **kw: niti.linear_act_bwd(a, _s(-8), w, _s(-7), act="relu", **{**dict(dout=dout, z=z), **kw})       # noqa: E731
    dx, dw, db = call()
    for kw in (dict(dout=_shifted(dout)), dict(z=_shifted(z)), dict(dx=_shifted(torch.empty_like(dx))), dict(dw=_shifted(torch.empty_like(dw), 3)),
               dict(dbias=_shifted(torch.empty_like(db)))):
        gx, gw, gb = call(**kw)
        assert torch.equal(gx, dx) and torch.equal(gw, dw), list(kw)
        assert (gb - db).abs().max() <= 300 * 300 * 2 * STEP
    assert niti.check() == 0
