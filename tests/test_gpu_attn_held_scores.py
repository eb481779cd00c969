"""Attention over 8 bits at the ends of what scores, scales and queries may be."""
import numpy as np
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import f64
from tests.rows_harness import Held, check_held_rows
from tests.test_gpu_attn_held import _set, _workspace

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _decode(c, q, scale):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, q.shape[1], q.shape[0]), scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == 0
    return out, lse


def _e4m3(x):
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("hq", [3, 12])
@pytest.mark.parametrize("q_power,k_power,scale_power", [(-100, 247, -27), (-120, 240, -2), (-60, 247, -67), (-100, 247, -30), (20, 67, 32), (-30, 67, 82), (100, 67, -48)])
def test_ordinary_scores_of_products_at_the_ends(hq, q_power, k_power, scale_power):
    """Scores of a few units, made of very small queries and scales with very large keys, and the other way round."""
    hd, n = 64, 150
    c = Held(dtype=BF, hkv=1, hd=hd, P=16, n_pages=12, max_seqs=1)
    c.grow([0], [n])
    g = torch.Generator(device="cuda").manual_seed(q_power)
    x = (torch.randn(2, 1, n, hd, generator=g, device="cuda") * 100).clamp(-448, 448)
    e = torch.full((2, 1, n), 120, dtype=torch.uint8, device="cuda")
    e[0] = k_power
    _set(c, 0, 0, _e4m3(x), e)
    q = (torch.randn(1, hq, hd, generator=g, device="cuda").clamp(-2, 2) * 2.0 ** q_power).to(BF)
    scale = 2.0 ** scale_power
    out, lse = _decode(c, q, scale)
    check_held_rows(out, lse, q, lambda i: c.tokens(0, 0), scale)
    assert 1 < abs(f64(lse)).max() < 100


@pytest.mark.parametrize("hq,hd", [(2, 64), (2, 128), (12, 64), (12, 128)])
@pytest.mark.parametrize("order", ["rising", "falling", "any"])
@pytest.mark.parametrize("power,ends", [(p, e) for p in (13, 18, 21) for e in ((127, 127), (117, 137), (67, 230))] + [(p, (117, 137)) for p in (25, 33, 45, 60)])
def test_large_scores(power, hq, hd, order, ends):
    """Scores are whole numbers times 2^power, times powers of two that go back and forth among values: one that is not the largest has no weight, and a
    result is the mean of the values at the largest score.

    Each of them is off by 2^-4 2^-21 (a weight in two terms of fp16, and exponentials), by 2^-24 of the largest where its own power is far below; fp32 sums of
    up to a few equal weights, a division, one rounding."""
    n = 700
    c = Held(dtype=BF, hkv=1, hd=hd, P=16, n_pages=50, max_seqs=1)
    c.grow([0], [n])
    r = np.random.default_rng(power)
    a = {"rising": np.arange(n) // 6, "falling": 120 - np.arange(n) // 6, "any": r.permutation(np.arange(n) % 120)}[order]
    a = np.maximum(a - 60, -60)                                # 240 steps of e4m3 hold these: whole numbers of up to 16, and even, and fourfold ones
    a = np.sign(a) * np.where(abs(a) <= 16, abs(a), np.where(abs(a) <= 32, abs(a) // 2 * 2, abs(a) // 4 * 4))
    g = torch.Generator(device="cuda").manual_seed(power)
    x = torch.randn(2, 1, n, hd, generator=g, device="cuda") * 60
    x[0] = 0
    x[0, 0, :, 5] = torch.as_tensor(a, device="cuda", dtype=torch.float32)
    e = torch.full((2, 1, n), 127, dtype=torch.uint8, device="cuda")
    e[1] = torch.randint(ends[0], ends[1] + 1, (1, n), generator=g, device="cuda").to(torch.uint8)
    _set(c, 0, 0, _e4m3(x.clamp(-448, 448)), e)
    q = torch.zeros(1, hq, hd, dtype=BF, device="cuda")
    q[:, :, 5] = 2.0 ** power
    out, lse = _decode(c, q, 1.0)
    k, v = c.tokens(0, 0)
    s = k[:, 0, 5] * 2.0 ** power
    at = v[s == s.max(), 0]
    m, want = len(at), at.mean(0)
    tol = 2.0 ** -8 * np.abs(want) + 2 * np.abs(at).max() * ((m + 4) * 2.0 ** -23 + 2.0 ** -20)
    assert (np.abs(f64(out)[0] - want) <= tol).all(), np.abs(f64(out)[0] - want).max()
    assert (np.abs(f64(lse)[0] - (s.max() + np.log(m))) <= abs(s.max()) * 2.0 ** -21 + np.log(m) * 2.0 ** -20 + 2.0 ** -16).all()
