"""Norms of rows whose squares, and an eps, are at the lower end of fp32."""
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.rows_harness import check_rotated, frequencies
from tests.test_gpu_rows import _cu, _dev, _gains, _qkv

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.mark.parametrize("spread", [1e-25, 1e-21, 7e-20, 1e-19, 2e-19, 1e-17, 1e-12])
@pytest.mark.parametrize("eps", [1.2e-38, 1e-36, 1e-30])
def test_squares_below_the_normal_numbers(spread, eps):
    q, k, _ = _qkv(9, 4, 2, 64, BF, spread=spread)
    q[3, 1] = 0
    freq = frequencies(64)
    qg, kg = _gains(64)
    r = nb.make_rotation(freq, qg, kg, eps=eps)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    nb.np_attn_rotate(r, q, k, qo, ko, _cu([9]), _dev([50]))
    torch.cuda.synchronize()
    eps = torch.tensor(eps).item()
    check_rotated(qo, q, qg, eps, range(50, 59), freq, False)
    check_rotated(ko, k, kg, eps, range(50, 59), freq, False)
    assert (qo[3, 1] == 0).all()
