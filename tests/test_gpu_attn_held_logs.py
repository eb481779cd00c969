"""The log of the sum over a cache of 8 bits, within the bound that its arithmetic gives: where values' powers of two are ordinary, that of 16 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import f64
from tests.rows_harness import Held
from tests.test_gpu_attn_held import _set, _workspace

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hd", [(4, 64), (4, 128), (16, 128)])
@pytest.mark.parametrize("exponents", [(127, 127), (120, 130), (247, 247), (67, 67), (180, 185)])
@pytest.mark.parametrize("n", [1, 3, 40, 1500])
def test_logs_of_sums(dtype, hq, hd, exponents, n):
    """Beside attn_oracle.tolerances: a score less the maximum, which has an exponent v of the values in it, is rounded at the scale of |v| and the scores (in
    base two), and so is the maximum with what the sum takes back: half a step of that each."""
    c = Held(dtype=dtype, hkv=1, hd=hd, P=32, n_pages=-(-n // 32) + 1, max_seqs=1)
    c.grow([0], [n])
    g = torch.Generator(device="cuda").manual_seed(n)
    x = (torch.randn(2, 1, n, hd, generator=g, device="cuda") * 30).clamp(-100, 100).to(torch.float8_e4m3fn).view(torch.uint8)
    e = torch.full((2, 1, n), 122, dtype=torch.uint8, device="cuda")
    e[1] = torch.randint(exponents[0], exponents[1] + 1, (1, n), generator=g, device="cuda").to(torch.uint8)
    _set(c, 0, 0, x, e)
    q = torch.randn(1, hq, hd, generator=g, device="cuda").to(dtype)
    out, lse = torch.empty_like(q), torch.empty(1, hq, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, hq, 1), lse=lse)
    torch.cuda.synchronize()
    k, v = c.tokens(0, 0)
    qn, ln, scale = f64(q), f64(lse), hd ** -0.5
    for h in range(hq):
        want, wl, mean, amp = A.attend(qn[0, h], k[:, 0], v[:, 0], scale)
        _, tl = A.tolerances(want, wl, mean, amp, n, hd, dtype == HF, False, np.abs(v).max())
        size = max(abs(x - 127) for x in exponents) + 2 * np.abs(k[:, 0] @ qn[0, h] * scale).max() / math.log(2) + 1
        half_step = 2.0 ** (math.ceil(math.log2(size)) - 25)
        assert abs(ln[0, h] - wl) <= tl + math.log(2) * 2 * half_step, (h, ln[0, h], wl)
