"""Weights of shared tokens in two terms of the rows' type: np_attn_decode_shared is as near to the 64-bit oracle as np_attn_decode, whichever way a
group takes."""
import numpy as np
import pytest
import torch

from tests.attn_harness import check_rows, f64
from tests.test_gpu_attn_shared import _branches, _shared, _workspace

from paper_2608_22643_b200 import binding as nb

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd,P,groups,tails", [
    (4, 2, 64, 16, [500], [[5, 0] * 10]),                       # one tile
    (8, 1, 128, 64, [1408], [[9] * 40]),                        # two tiles; the last tile half full
    (6, 2, 128, 32, [320, 64], [[1] * 30, [70, 0] * 16]),
    (12, 12, 64, 256, [4096], [[0] * 150]),
    (2, 2, 64, 16, [160], [[3, 7]]),                            # few columns: the other kernel
])
def test_as_exact_as_decode(dtype, hq, hkv, hd, P, groups, tails):
    c, seqs, cu = _branches(dtype, hkv, hd, P, groups, tails)
    n = len(seqs)
    q = torch.randn(n, hq, hd, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).to(dtype)
    out, lse = torch.empty_like(q), torch.empty(n, hq, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, hq, n), c.dev(cu), _shared(c, seqs, cu), seqs=c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    kept = {s: c.tokens(0, s) for s in seqs}
    check_rows(out, lse, q, lambda i: kept[seqs[i]], hd ** -0.5, False)


@pytest.mark.parametrize("dtype,power", [(BF, 8), (HF, 11)])
def test_roundings_that_agree(dtype, power):
    """All tokens but one have a weight of (1 + 0.95 2^-power) / 4, which the type rounds to 1 / 4, and values of 1; the one with a weight of 1 has what makes
    the rounded sum 0.  What is left of the sum is what the rounding took."""
    hd, ways, tokens = 64, 40, 65
    c, seqs, cu = _branches(dtype, 1, hd, 16, [80], [[0] * ways])
    weight = (1 + 0.95 * 2.0 ** -power) / 4
    pages = torch.tensor(c.pool.pages[0], device="cuda")
    at = torch.arange(80, device="cuda")
    k, v = torch.zeros(80, hd, device="cuda"), torch.zeros(80, hd, device="cuda")
    k[0, 0] = 1.0                                                       # its score: the others' are 0
    v[1:tokens] = 1.0
    v[0] = -(tokens - 1) / 4
    k[tokens:, 1] = -64.0                                               # the rest are far below
    c.cache[0, pages[at // 16], 0, 0, at % 16], c.cache[0, pages[at // 16], 1, 0, at % 16] = k.to(dtype), v.to(dtype)
    q = torch.zeros(ways, 2, hd, dtype=dtype, device="cuda")
    q[..., :2] = 1.0
    scale = -np.log(weight)
    out, lse = torch.empty_like(q), torch.empty(ways, 2, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 2, ways), c.dev(cu), c.dev([80]), seqs=c.dev(seqs), scale=scale, lse=lse)
    torch.cuda.synchronize()
    total = 1 + (tokens - 1) * weight
    want = (tokens - 1) * (weight - 0.25) / total
    # the score is off by 10 roundings of values below 2 and the exponential by 2^-21, of 64 weights; two terms by 2^-16 (2^-22) of a weight
    off = (tokens - 1) / 4 * (10 * 2.0 ** -23 + 2.0 ** -21 + (2.0 ** -16 if dtype == BF else 2.0 ** -22)) / total
    assert (np.abs(f64(out) - want) <= 2.0 ** -power * want + (1 + 2.0 ** -power) * off).all(), (f64(out).min(), f64(out).max(), want)
    assert off < want / 2
