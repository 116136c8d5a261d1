"""The linear layer's backward pass for every choice of outputs: the results of the full call, and the same status."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu
CHOICES = [c for c in itertools.product((False, True), repeat=3) if any(c)]


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _operands(M, N, K, dtype, act):
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    i8 = lambda *s: torch.randint(-127, 128, s, device="cuda", generator=gen, dtype=torch.int32).to(torch.int8)      # noqa: E731
    s = torch.full((1,), -8, dtype=torch.int32, device="cuda")
    z = torch.randn((M, N), device="cuda", generator=gen).to(dtype) if act != "none" else None
    return (i8(M, K), s, i8(N, K), s, torch.randn((M, N), device="cuda", generator=gen).to(dtype)), z


@pytest.mark.parametrize("choice", CHOICES, ids=lambda c: "".join("xwb"[i] for i in range(3) if c[i]))
@pytest.mark.parametrize("M,N,K,dtype,act", [(200, 96, 160, torch.bfloat16, "gelu"), (130, 50, 77, torch.float32, "none"), (1, 33, 16, torch.float16, "relu")])
def test_outputs_are_those_of_the_full_call(niti, M, N, K, dtype, act, choice):
    args, z = _operands(M, N, K, dtype, act)
    want = niti.linear_act_bwd(*args, z=z, act=act)
    got = niti.linear_act_bwd(*args, z=z, act=act, need_dx=choice[0], need_dw=choice[1], need_dbias=choice[2])
    for need, g, w in zip(choice, got, want):
        assert torch.equal(g, w) if need else g is None
    assert niti.check() == 0


@pytest.mark.parametrize("choice", CHOICES, ids=lambda c: "".join("xwb"[i] for i in range(3) if c[i]))
@pytest.mark.parametrize("where", ["dout", "z"])
@pytest.mark.parametrize("M,N,K", [(200, 96, 160), (700, 50, 32), (3, 4100, 32)])
def test_errors_that_are_not_finite_raise_the_status(niti, M, N, K, where, choice):
    """In the first or the last element, whatever outputs are wanted."""
    from paper_2009_13108_b200 import NitiError
    for at in ((0, 0), (M - 1, N - 1)):
        for x in (float("nan"), float("inf")):
            args, z = _operands(M, N, K, torch.float32, "gelu" if where == "z" else "none")
            call = lambda: niti.linear_act_bwd(*args, z=z, act="none" if z is None else "gelu", need_dx=choice[0], need_dw=choice[1], need_dbias=choice[2])  # noqa: E731
            call()
            assert niti.check() == 0
            if where == "z":
                z[at] = float("nan")
            else:
                args[4][at] = x
            call()
            with pytest.raises(NitiError, match="0x40"):
                niti.check()
