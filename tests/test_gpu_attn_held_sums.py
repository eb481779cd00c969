"""Attention over 8 bits where values' powers of two lie as far apart as the form allows: the sum of the weights is that of all tokens, in any order."""
import math

import numpy as np
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.rows_harness import Held, check_held_rows
from tests.test_gpu_attn_held import _set, _workspace

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _decode(c, q, scale=None):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, q.shape[1], q.shape[0]), scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == 0
    return out, lse


def _fill(c, n, exponents, seed=1, keys=127):
    """A sequence of n tokens, values of 0.25 to 100 times 2^(exponents - 127), keys around 1."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(2, c.hkv, n, c.hd, generator=g, device="cuda")
    x[1] = (x[1].abs() * 30 + 0.25).clamp(max=100)
    e = torch.full((2, c.hkv, n), keys, dtype=torch.uint8, device="cuda")
    e[1] = torch.as_tensor(exponents, dtype=torch.uint8, device="cuda")
    _set(c, 0, 0, x.to(torch.float8_e4m3fn).view(torch.uint8), e)


# where the second power begins: another warp, the same warp's next tokens, another block, the last token
SPLITS = [(17, 16), (80, 64), (144, 128), (300, 128), (9000, 4500), (9000, 8999), (9000, 1)]


@pytest.mark.parametrize("hq,hd", [(2, 64), (2, 128), (16, 64), (16, 128)])
@pytest.mark.parametrize("n,at", SPLITS)
@pytest.mark.parametrize("first,second", [(67, 247), (247, 67), (67, 200), (220, 90)])
def test_sums_of_tokens_whose_values_are_far_apart(hq, hd, n, at, first, second):
    """Queries of 0: every token has the same weight, and the log of the sum is that of their number.

    A weight is the square of a power of two that is off by 2^-22, so off by 2^-21; a maximum that grows, in a warp and at three joins (of warps, of blocks,
    of joined ones), brings a factor that is off by 2^-21 each; fp32 sums, in a chain of a lane's tokens (of a block's, at most 200 of them), 3 exchanges,
    4 warps, 8 parts and 8 joined ones.  The logarithm of the sum's mantissa is off by 2^-21, and its product with ln 2 and the maximum's by half a step of the result each."""
    c = Held(dtype=BF, hkv=1, hd=hd, P=64, n_pages=-(-n // 64) + 1, max_seqs=1)
    c.grow([0], [n])
    _fill(c, n, np.where(np.arange(n) < at, first, second))
    q = torch.zeros(1, hq, hd, dtype=BF, device="cuda")
    out, lse = _decode(c, q)
    off = 5 * 2.0 ** -21 + 2.0 ** -21 + (200 + 23) * 2.0 ** -24 + 2 * math.log(n) * 2.0 ** -23
    assert (lse.double() - math.log(n)).abs().max() <= off
    check_held_rows(out, lse, q, lambda i: c.tokens(0, 0), hd ** -0.5)


@pytest.mark.parametrize("hq,hd", [(4, 64), (16, 128)])
@pytest.mark.parametrize("seed", range(4))
def test_sums_of_tokens_in_any_order(hq, hd, seed):
    """Random powers of two over the whole range, scores of some size: out and the log of the sum, rows of two lengths."""
    c = Held(dtype=HF if seed % 2 else BF, hkv=2, hd=hd, P=16, n_pages=200, max_seqs=1)
    n = (700, 2500)[seed // 2]
    c.grow([0], [n])
    r = np.random.default_rng(seed)
    e = r.choice([67, 100, 130] if c.dtype == HF else [67, 120, 247], (2, n))
    _fill(c, n, e, seed=seed)
    q = torch.randn(1, hq, hd, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(c.dtype)
    out, lse = _decode(c, q)
    check_held_rows(out, lse, q, lambda i: c.tokens(0, 0), hd ** -0.5)
