"""Scores of up to 2^68, finite: the softmax is of their differences, however large they are themselves.

Each query has one element that is not 0 and the keys' elements there are small whole numbers times a power of two, so scores are exact in fp32;
with `scale` 1 two that differ are 2^13 apart at least, and a row's result is the mean of the values at its largest score."""
import numpy as np
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, check_rows, f64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _steps(n, order, rng):
    """Whole numbers, one for each token, as the keys have them: rising, falling, any, all below zero, every one twice."""
    a = np.arange(1, n + 1) % 128 + 1
    return {"rising": np.minimum(np.arange(n) // 3 + 1, 255), "falling": np.maximum(250 - np.arange(n), 1), "any": rng.permutation(a),
            "negative": -rng.permutation(a), "zero": rng.permutation(a) - 64}[order]


def _check(out, lse, v, scores, half, p_half):
    """One row: the mean of the values at the largest score.  fp32 sums of m equal weights, each off by m 2^-24, a division good to
    2^-22, weights good to `p_half`, one rounding of the result (2^-25 below fp16's normal range)."""
    top = scores.max()
    at = v[scores == top]
    m, want, mean = len(at), at.mean(0), np.abs(at).mean(0)
    tol = half * np.abs(want) + (1 + half) * mean * ((m + 4) * 2.0 ** -23 + p_half) + 2.0 ** -25
    assert (np.abs(out - want) <= tol).all(), np.abs(out - want).max()
    # the score times log2(e), both rounded, times ln(2): four roundings; the logarithm of the sum is good to 2^-20
    assert abs(lse - (top + np.log(m))) <= abs(top) * 2.0 ** -21 + np.log(m) * 2.0 ** -20 + 2.0 ** -20


# (type, power of two that the whole numbers are multiplied by)
POWERS = [(HF, 13), (HF, 21), (HF, 22), (BF, 13), (BF, 21), (BF, 30), (BF, 45), (BF, 60)]


def _factors(dtype, power):
    """(query's element, power of two of the keys'): the keys' times 255 is in the type's range, 65504 in fp16."""
    p = min(power // 2, 8) if dtype == HF else power // 2
    return 2.0 ** (power - p), 2.0 ** p


@pytest.mark.parametrize("dtype,power", POWERS)
@pytest.mark.parametrize("order", ["rising", "falling", "any", "negative", "zero"])
@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_of_large_scores(dtype, power, order, hd):
    n, hq = 300, 3
    rng = np.random.default_rng(power)
    g = torch.Generator(device="cuda").manual_seed(power)
    fq, fk = _factors(dtype, power)
    qkv = torch.randn(n, hq + 2, hd, generator=g, device="cuda")
    qkv[:, 0] = 0
    qkv[:, 0, 5] = fq                                  # head 0: large scores
    qkv[:, 1:hq, 5] = 0                                # the others, rows of the same warps: ordinary ones
    qkv[:, hq, 5] = torch.tensor(_steps(n, order, rng), device="cuda") * fk
    qkv = qkv.to(dtype)
    out, lse = torch.empty(n, hq, hd, dtype=dtype, device="cuda"), torch.empty(n, hq, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(qkv[:, :hq], qkv[:, hq:hq + 1], qkv[:, hq + 1:], torch.tensor([0, n], dtype=torch.int32, device="cuda"), out, status, scale=1.0, lse=lse)
    assert nb.np_attn_check(status) == nb.NP_OK
    k, v, o, ln = f64(qkv[:, hq]), f64(qkv[:, hq + 1]), f64(out), f64(lse)
    half = 2.0 ** -11 if dtype == HF else 2.0 ** -8
    for r in range(n):
        _check(o[r, 0], ln[r, 0], v[:r + 1], k[:r + 1, 5] * fq, half, half)
    # the others' tolerance without the column that only head 0 looks at (their queries are 0 there)
    k[:, 5] = 0
    check_rows(out[:, 1:], lse[:, 1:], qkv[:, 1:hq], lambda i: (k[:i + 1, None], v[:i + 1, None]), 1.0, True)


@pytest.mark.parametrize("dtype,power", POWERS)
@pytest.mark.parametrize("hq", [2, 12])
def test_decode_of_large_scores(dtype, power, hq):
    lens = [1, 3, 64, 300, 2000]
    c = Cache(dtype=dtype, hkv=1, hd=128, P=16, n_pages=160, max_seqs=len(lens))
    c.grow(list(range(len(lens))), lens)
    rng = np.random.default_rng(power)
    fq, fk = _factors(dtype, power)
    for s, n in enumerate(lens):
        a = torch.tensor(_steps(n, ["any", "negative", "rising", "zero", "falling"][s], rng) * fk, device="cuda")
        j = torch.arange(n, device="cuda")
        c.cache[0, torch.tensor(c.pool.pages[s], device="cuda")[j // 16], 0, 0, j % 16, 5] = a.to(dtype)
    q = torch.zeros(len(lens), hq, 128, dtype=dtype, device="cuda")
    q[:, :, 5] = fq
    out, lse = torch.empty_like(q), torch.empty(len(lens), hq, device="cuda")
    ws = torch.zeros(nb.np_attn_workspace_bytes(c.desc, hq, len(lens)), dtype=torch.uint8, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, ws, scale=1.0, lse=lse)
    torch.cuda.synchronize()
    o, ln, half = f64(out), f64(lse), 2.0 ** -11 if dtype == HF else 2.0 ** -8
    for i in range(len(lens)):
        k, v = c.tokens(0, i)
        for h in range(hq):
            _check(o[i, h], ln[i, h], v[:, 0], k[:, 0, 5] * fq, half, half * half)
