"""The exponent of a tensor without rows is that of a tensor of zeros."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def test_the_exponent_of_a_tensor_without_rows_is_zero(niti):
    empty, gain, s = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda"), torch.full((1,), 7, dtype=torch.int32, device="cuda")
    q, got = niti.quantize(empty, s=s, rows=False)
    assert got is s and q.shape == (0, 64) and int(s) == 0
    s.fill_(7)
    y, got, h, _ = niti.rmsnorm_fwd(empty, gain, s_y=s, rows=False)
    assert got is s and y.shape == (0, 64) and int(s) == 0
    assert niti.dequantize(q, s).shape == (0, 64) and niti.check() == 0
