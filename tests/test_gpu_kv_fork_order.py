"""Forks of a sequence whose reserved tokens are appended before the fork, and after it: what include/np.h says of each order."""
import numpy as np
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, f64

pytestmark = pytest.mark.gpu


def _fork(c, a, b):
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([a]), c.dev([b]))
    c.pool.fork([a], [b])
    c.check()


@pytest.mark.parametrize("layers,P,n", [(1, 16, 40), (3, 32, 64), (2, 16, 5)])
def test_appended_and_then_forked(layers, P, n):
    c = Cache(layers=layers, hkv=2, hd=64, P=P, n_pages=20, max_seqs=3)
    c.grow([0], [n])
    _fork(c, 0, 1)
    before = [c.tokens(layer, 0) for layer in range(layers)]
    c.grow([1], [P + 3], seed=9)                     # the branch goes on
    c.check()
    for layer in range(layers):
        for got, was in zip(c.tokens(layer, 0), before[layer]):
            assert np.isfinite(was).all() and (got == was).all()
        for got, was in zip(c.tokens(layer, 1), before[layer]):
            assert (got[:n] == was).all() and np.isfinite(got).all()


@pytest.mark.parametrize("n", [16, 40, 5])
def test_forked_between_reserving_and_appending(n):
    """The source has all of its tokens; the branch those of shared pages, not those of its own last page."""
    P = 16
    c = Cache(layers=1, hkv=2, hd=64, P=P, n_pages=20, max_seqs=3)
    start, _ = c.reserve([0], [n])
    _fork(c, 0, 1)
    k, v = c.append(0, [0], start, [n])
    c.check()
    full = n // P * P
    for i, rows in enumerate((k, v)):
        assert (c.tokens(0, 0)[i] == f64(rows)).all()
        branch = c.tokens(0, 1)[i]
        assert (branch[:full] == f64(rows)[:full]).all() and np.isnan(branch[full:]).all()
    # its own tokens are appended like any other's
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k, v, c.dev([1]), c.dev([0, n]), start)
    torch.cuda.synchronize()
    for i, rows in enumerate((k, v)):
        assert (c.tokens(0, 1)[i] == f64(rows)).all() and (c.tokens(0, 0)[i] == f64(rows)).all()
