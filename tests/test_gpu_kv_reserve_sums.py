"""np_kv_reserve where the pages that are asked for add up to more than 32 bits hold (the largest pool; tables alone, no cache)."""
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild

pytestmark = pytest.mark.gpu

PAGES, P = 1 << 22, 16
ALL = PAGES * P                      # tokens that take every page of the pool


def _free(status):
    got = status.item()
    status.zero_()
    return got


def test_a_sum_of_pages_past_32_bits_is_too_many():
    nbuild.build()
    ints = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")   # noqa: E731
    desc = nb.make_kv_desc(torch.bfloat16, 1, 1, 64, P, PAGES, 1024)
    table, lens, refs, status = ints(1024, PAGES), ints(1024), ints(PAGES), ints(1)
    scratch = ints(nb.np_kv_sizes(desc).scratch_bytes // 4)
    tables = nb.make_kv_tables(table, lens, refs, scratch, status)
    nb.np_kv_reset(desc, tables)

    def reserve(n_new):
        start = torch.full((len(n_new),), 99, dtype=torch.int32, device="cuda")
        nb.np_kv_reserve(desc, tables, None, torch.tensor(n_new, dtype=torch.int32, device="cuda"), start)
        return start.tolist()

    # 512 and 513 (2^31 pages and more), 1024 (2^32): the first has room, nobody else
    for n in (512, 513, 1000, 1024):
        assert reserve([ALL] * n) == [0] + [-1] * (n - 1)
        assert lens.tolist() == [ALL] + [0] * 1023 and _free(status) == nb.NP_KV_S_FULL
        assert torch.equal(table[0], torch.arange(PAGES, dtype=torch.int32, device="cuda")) and (refs == 1).all()
        assert (table[1:n:37, :100] == -1).all() and (table[n - 1] == -1).all()
        nb.np_kv_free(desc, tables, n=1)
        assert not refs.any() and not lens.any() and _free(status) == 0
    # a few pages first, then too many, then one page (counted behind them: too many as well), then none
    assert reserve([5 * P] + [ALL] * 1020 + [1, 0, 0]) == [0] + [-1] * 1021 + [0, 0]
    assert lens.tolist() == [5 * P] + [0] * 1023 and _free(status) == nb.NP_KV_S_FULL and refs.sum().item() == 5
    # sequences that have tokens already
    assert reserve([P] + [0] * 510 + [ALL] * 512 + [3 * P]) == [5 * P] + [0] * 510 + [-1] * 513
    assert lens.tolist() == [6 * P] + [0] * 1023 and _free(status) == nb.NP_KV_S_FULL and refs.sum().item() == 6
