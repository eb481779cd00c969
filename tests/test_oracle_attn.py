"""The cache's and the attention's oracle against what their definitions fix."""
import numpy as np
import pytest

from oracle import attn_oracle as A


def _books(p):
    """Every page's count is the number of rows that hold it, rows hold just what their lengths need, partly filled pages have
    one owner."""
    assert (p.refs() >= 0).all()
    r = p.refs()
    for s in range(p.max_seqs):
        assert len(p.pages[s]) == -(-p.lens[s] // p.P) and len(set(p.pages[s])) == len(p.pages[s])
        if p.lens[s] % p.P:
            assert r[p.pages[s][-1]] == 1


def test_random_calls_keep_the_books():
    rng = np.random.default_rng(3)
    p = A.Pool(16, 40, 12, 20)
    for _ in range(300):
        what, n = rng.integers(4), int(rng.integers(1, 5))
        seqs = rng.permutation(12)[:n].tolist()
        before = set(p.free_pages())
        if what == 0:
            p.reserve(seqs, rng.integers(0, 60, n).tolist())
        elif what == 1:
            dst = [s for s in range(12) if p.lens[s] == 0][:n]
            copies = p.fork(rng.integers(0, 12, len(dst)).tolist(), dst)
            assert {b for _, b in copies} <= before
        elif what == 2:
            p.free(seqs)
        else:
            lens = list(p.lens)
            live, moves = p.compact()
            assert p.lens == lens and (p.refs()[:live] > 0).all() and not p.refs()[live:].any()
            assert all(a >= live > b for a, b in moves)
        _books(p)


def test_pages_come_lowest_first_and_a_short_pool_refuses_in_list_order():
    p = A.Pool(16, 6, 4, 6)
    assert p.reserve([2, 0], [17, 1]) == [0, 0] and p.pages[2] == [0, 1] and p.pages[0] == [2]
    p.free([2])
    assert p.reserve([1, 3, 0], [40, 64, 2]) == [0, -1, 1]      # three pages of five; four are not left; no page needed
    assert p.pages[1] == [0, 1, 3] and p.lens[3] == 0 and p.lens[0] == 3 and p.status == A.S_FULL


@pytest.mark.parametrize("tokens", [0, 1, 2, 33])
def test_attention_is_a_mean_and_its_sum_normalises_it(tokens):
    rng = np.random.default_rng(tokens)
    q, k, v = rng.standard_normal(64), rng.standard_normal((tokens, 64)), rng.standard_normal((tokens, 64))
    o, lse, mean, amp = A.attend(q, k, v, 0.125)
    if tokens == 0:
        assert (o == 0).all() and lse == -np.inf
        return
    w = np.exp(k @ q * 0.125 - lse)
    assert abs(w.sum() - 1) < 1e-12 and np.allclose(w @ v, o, atol=1e-12)
    assert (o <= v.max(0) + 1e-12).all() and (o >= v.min(0) - 1e-12).all() and (np.abs(o) <= mean + 1e-12).all()
    if tokens == 1:
        assert np.allclose(o, v[0]) and abs(lse - k[0] @ q * 0.125) < 1e-12
    # joining two parts by their sums gives the whole
    if tokens > 1:
        a, la, _, _ = A.attend(q, k[:1], v[:1], 0.125)
        b, lb, _, _ = A.attend(q, k[1:], v[1:], 0.125)
        t = np.logaddexp(la, lb)
        assert abs(t - lse) < 1e-12 and np.allclose(np.exp(la - t) * a + np.exp(lb - t) * b, o, atol=1e-12)
