"""Queries that rows or heads have in common (strides of 0): the same in small groups and large ones."""
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import check_rows
from tests.test_gpu_attn_shared import _branches, _workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ways,hq,hkv", [(2, 4, 2), (40, 4, 2), (30, 1, 1), (9, 32, 1)])
@pytest.mark.parametrize("common", ["rows", "heads", "both"])
def test_queries_in_common(dtype, ways, hq, hkv, common):
    c, seqs, cu = _branches(dtype, hkv, 64, 16, [800], [[20] + [1] * (ways - 1)])
    one = torch.randn(1 if common != "heads" else ways, 1 if common != "rows" else hq, 64, device="cuda").to(dtype)
    q = one.expand(ways, hq, 64)
    out, lse = torch.empty(ways, hq, 64, dtype=dtype, device="cuda"), torch.empty(ways, hq, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, hq, ways), c.dev(cu), c.dev([800]), seqs=c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == 0
    kept = {s: c.tokens(0, s) for s in seqs}
    check_rows(out, lse, q, lambda i: kept[seqs[i]], 0.125, False)
