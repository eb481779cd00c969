"""`scale` at the ends of fp32's range."""
import ctypes as C
import math

import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild

P = 0x1000      # stands for any aligned address: these calls end before it is used


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_past_the_range_in_base_two_is_refused(scale):
    """Scores are kept in base two: scale * log2(e) has to be a number, too (else 0 * inf in every row)."""
    nbuild.build()
    lib, b = nb.load(), C.byref
    d, t, r = nb.make_kv_desc(torch.bfloat16, 2, 4, 128, 64, 100, 8, 50), nb.np_kv_tables(P, P, P, P, P), nb.np_rows(P, 512, 128)
    assert lib.np_attn_decode(b(d), P, 0, b(t), b(r), 8, P, 2, scale, b(r), None, P, 1 << 40, None) == nb.NP_E_INVAL
    assert "scale" in lib.np_attn_last_error().decode()
    assert lib.np_attn_prompt(b(nb.np_attn_shape(0, 8, 4, 128)), b(r), b(r), b(r), P, 2, 9, scale, b(r), None, P, None) == nb.NP_E_INVAL
    assert "scale" in lib.np_attn_last_error().decode()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-45, 1e-39, 7e-39, 1.2e-38, 2.3e38])
@pytest.mark.parametrize("hq", [3, 12])
def test_scales_that_are_hardly_numbers(scale, hq):
    """The smallest: plain means of the values, a key of -inf left out.  The largest: queries of 0, the same."""
    from tests.attn_harness import Cache, f64
    n, bad = 50, 20
    c = Cache(hkv=1, hd=64, P=16, n_pages=4, max_seqs=1)
    c.grow([0], [n])
    k, v = c.tokens(0, 0)
    q = torch.rand(n, hq, 64, device="cuda").to(torch.bfloat16) + 0.1
    if scale > 1:
        q.zero_()
    else:
        c.cache[0, c.pool.pages[0][bad // 16], 0, 0, bad % 16] = -math.inf
    kk, vv = (torch.tensor(x, device="cuda").to(torch.bfloat16) for x in (k, v))
    if scale < 1:
        kk[bad] = -math.inf
    o1, l1 = torch.empty(1, hq, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, device="cuda")
    ws = torch.zeros(nb.np_attn_workspace_bytes(c.desc, hq, 1), dtype=torch.uint8, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q[-1:], o1, ws, scale=scale, lse=l1)
    o2, l2, status = torch.empty_like(q), torch.empty(n, hq, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(q, kk, vv, torch.tensor([0, n], dtype=torch.int32, device="cuda"), o2, status, scale=scale, lse=l2)
    assert nb.np_attn_check(status) == nb.NP_OK
    got = [(f64(o1)[0], f64(l1)[0], n)] + [(f64(o2)[r], f64(l2)[r], r + 1) for r in (0, 5, bad, bad + 1, n - 1)]
    for o, lse, seen in got:
        at = [j for j in range(seen) if scale > 1 or j != bad]
        want, mean = v[at, 0].mean(0), abs(v[at, 0]).mean(0)
        # weights are 1 and exact in the rows' type: fp32 sums of up to 50, a division, one rounding
        assert (abs(o - want) <= abs(want) * 2.0 ** -8 + mean * 60 * 2.0 ** -23).all()
        assert (abs(lse - math.log(len(at))) <= 4 * 2.0 ** -20).all()
