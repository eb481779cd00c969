"""The paged cache's calls against the oracle's pool: tables bit for bit, bytes where the tables say."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, f64

pytestmark = pytest.mark.gpu


def test_reset_empties_everything():
    c = Cache(n_pages=2000, max_seqs=5, max_pages=300)
    c.check()


@pytest.mark.parametrize("P,n_pages,n", [(16, 40, 6), (64, 9000, 6), (256, 20000, 64)])
def test_reserve_and_free_follow_the_oracle(P, n_pages, n):
    """Pools of one scan round and of several; sequences that need none, one or many pages; the first free pages at the far end."""
    rng = np.random.default_rng(P)
    c = Cache(P=P, n_pages=n_pages, max_seqs=n + 3, hkv=1, max_pages=min(n_pages, 8000))
    most = c.P * c.desc.n_pages // n
    for step in range(12):
        m = int(rng.integers(1, n + 1))
        seqs = rng.permutation(n + 3)[:m].tolist()
        c.reserve(seqs, rng.integers(0, most, m).tolist())
        c.check()
        gone = rng.permutation(n + 3)[:int(rng.integers(1, n + 1))].tolist()
        nb.np_kv_free(c.desc, c.tables, c.dev(gone))
        c.pool.free(gone)
        c.check()


def test_a_pool_that_runs_short_refuses_in_list_order():
    c = Cache(P=16, n_pages=6, max_seqs=4)
    c.reserve([2, 0], [17, 1])
    nb.np_kv_free(c.desc, c.tables, c.dev([2]))
    c.pool.free([2])
    _, start = c.reserve([1, 3, 0], [40, 64, 2])
    assert start == [0, -1, 1]
    c.check()
    with pytest.raises(nb.NpError) as e:
        nb.np_attn_check(c.status)
    assert e.value.code == nb.NP_E_DEVICE and "free pages" in str(e.value)


def test_bad_entries_are_left_out_and_reported():
    """Sequence numbers outside the tables or listed twice, negative counts, lengths past a row."""
    c = Cache(P=16, n_pages=20, max_seqs=4, max_pages=3)
    c.reserve([0, -1, 4, 0], [5, 5, 5, 9])
    c.check()
    assert c.pool.status == A.S_SEQ and c.pool.lens == [5, 0, 0, 0]
    c.reserve([1, 2, 3], [-2, 49, 48])
    c.check()
    assert c.pool.status == A.S_SEQ | A.S_LENGTH and c.pool.lens == [5, 0, 0, 48]
    gone = [3, 3, 9]
    nb.np_kv_free(c.desc, c.tables, c.dev(gone))
    c.pool.free(gone)
    c.check()
    c.reserve([1], [0x7fffffff])
    c.check()


@pytest.mark.parametrize("dtype,hkv,hd,P", [(torch.bfloat16, 1, 64, 16), (torch.float16, 5, 128, 32), (torch.bfloat16, 40, 128, 256)])
def test_append_puts_rows_where_the_tables_say(dtype, hkv, hd, P):
    c = Cache(dtype=dtype, layers=2, hkv=hkv, hd=hd, P=P, n_pages=24, max_seqs=6)
    held = {s: [] for s in range(6)}
    for step, counts in enumerate([[3, 0, 40], [1, 1, 1], [P, 2 * P - 3, 17]]):
        seqs = [4, 0, 2]
        start, _ = c.reserve(seqs, counts)
        before = c.cache.clone()
        k, v = c.append(1, seqs, start, counts, seed=step)
        c.check()
        at = 0
        for s, n in zip(seqs, counts):
            held[s].append((k[at:at + n], v[at:at + n]))
            at += n
        for s in seqs:
            gk, gv = c.tokens(1, s)
            assert (gk == np.concatenate([f64(x) for x, _ in held[s]])).all() and (gv == np.concatenate([f64(x) for _, x in held[s]])).all()
        # nothing else was written: as many values changed as came in (the others still are NaN)
        assert torch.equal(before[0].view(torch.int16), c.cache[0].view(torch.int16))
        assert int((~torch.isnan(c.cache[1])).sum()) == 2 * hkv * hd * sum(c.pool.lens)


def test_append_skips_what_has_no_place():
    """A sequence that was not given room, rows behind the last sequence, positions past the length, pages that are not there."""
    c = Cache(P=16, n_pages=2, max_seqs=3, hkv=1)
    start, s = c.reserve([0, 1, 2], [10, 60, 3])
    assert s == [0, -1, 0] and c.pool.status == A.S_LENGTH
    k, v = torch.ones(80, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(80, 1, 64, dtype=torch.bfloat16, device="cuda")
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k, v, None, c.dev([0, 15, 70, 73]), start)     # five rows too many for sequence 0
    c.check()
    assert int((~torch.isnan(c.cache)).sum()) == 2 * 64 * 13
    c.table[0, 0] = 2
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k[:1], v[:1], c.dev([0]), None, c.dev([1]))
    torch.cuda.synchronize()
    assert c.status.item() == A.S_LENGTH | A.S_PAGE and int((~torch.isnan(c.cache)).sum()) == 2 * 64 * 13
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k[:2], v[:2], c.dev([7, -1]), None, c.dev([0, 0]))
    torch.cuda.synchronize()
    assert c.status.item() & A.S_SEQ and int((~torch.isnan(c.cache)).sum()) == 2 * 64 * 13


@pytest.mark.parametrize("P,layers,hkv,hd", [(16, 1, 1, 64), (64, 3, 2, 128), (32, 40, 5, 64)])
def test_fork_shares_full_pages_and_copies_the_last(P, layers, hkv, hd):
    c = Cache(layers=layers, hkv=hkv, hd=hd, P=P, n_pages=30, max_seqs=16)
    c.grow([0, 1, 2, 3], [2 * P + 5, P, 1, 0])
    src, dst = [0, 0, 1, 2, 3, 0], [9, 8, 4, 7, 5, 6]
    want = [c.tokens(layers - 1, s) for s in src]
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev(src), c.dev(dst))
    copies = c.pool.fork(src, dst)
    c.check()
    for s, (k, v) in zip(dst, want):
        gk, gv = c.tokens(layers - 1, s)
        assert (gk == k).all() and (gv == v).all()
    for layer in range(layers):
        for a, b in copies:
            assert torch.equal(c.cache[layer, a].view(torch.int16), c.cache[layer, b].view(torch.int16))
    # branches go their own ways, and the parents stay
    parents = [c.tokens(0, s) for s in range(4)]
    c.grow(dst, [3, 4, 5, 6, 7, P + 2], seed=50)
    c.check()
    for s, (k, v) in zip(range(4), parents):
        gk, gv = c.tokens(0, s)
        assert (gk == k).all() and (gv == v).all()
    nb.np_kv_free(c.desc, c.tables, n=10)
    c.pool.free(list(range(10)))
    c.check()
    assert not c.pool.refs().any()


def test_fork_refusals():
    """Targets in use, listed twice, out of range, a sequence onto itself; a pool without room for the copies."""
    c = Cache(P=16, n_pages=5, max_seqs=8, hkv=1)
    c.grow([0, 1], [17, 16])
    src, dst = [0, 0, 0, 8, 0, -1, 3, 0], [1, 2, 2, 3, 8, 4, 3, 0]
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev(src), c.dev(dst))
    c.pool.fork(src, dst)
    c.check()
    assert c.pool.status == A.S_SEQ and c.pool.lens[2] == 17
    src, dst = [0, 0, 1], [5, 6, 7]      # one free page, two wanted; a full page needs none
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev(src), c.dev(dst))
    c.pool.fork(src, dst)
    c.check()
    assert c.pool.status == A.S_SEQ | A.S_FULL and c.pool.lens[5:] == [17, 0, 16]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("P,layers,n_pages", [(16, 2, 40), (64, 5, 200), (16, 3, 257), (16, 1, 2048), (16, 1, 2049), (16, 1, 9000)])
def test_compact_moves_pages_down(P, layers, n_pages, in_place):
    c = Cache(layers=layers, hkv=2, hd=64, P=P, n_pages=n_pages, max_seqs=12)
    rng = np.random.default_rng(n_pages)
    c.grow(list(range(10)), rng.integers(0, P * n_pages // 10, 10).tolist())
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([7]), c.dev([11]))
    c.pool.fork([7], [11])
    gone = [0, 3, 4, 6]
    nb.np_kv_free(c.desc, c.tables, c.dev(gone))
    c.pool.free(gone)
    c.check()
    want = [[c.tokens(layer, s) for s in range(12)] for layer in range(layers)]
    old_table, old_cache = c.table.clone(), c.cache.clone()
    out = c.tables
    if not in_place:
        fresh = [torch.full_like(t, 55) for t in (c.table, c.lens, c.refs)]
        out = nb.make_kv_tables(*fresh, c.scratch, c.status)
    n_live = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_kv_compact(c.desc, c.cache, c.tables, out, n_live)
    live, moves = c.pool.compact()
    torch.cuda.synchronize()
    assert n_live.item() == live and len(moves) > 0
    if not in_place:
        assert torch.equal(c.table, old_table)                        # the old tables still say where the tokens were ...
        stay = torch.tensor(sorted(set(range(n_pages)) - {b for _, b in moves}), device="cuda")
        assert torch.equal(c.cache[:, stay].view(torch.int16), old_cache[:, stay].view(torch.int16))      # ... and they still are there
        c.table, c.lens, c.refs = fresh
    c.check()
    for layer in range(layers):
        for s in range(12):
            gk, gv = c.tokens(layer, s)
            assert (gk == want[layer][s][0]).all() and (gv == want[layer][s][1]).all()


def test_compact_of_empty_full_and_compact_pools():
    c = Cache(P=16, n_pages=4, max_seqs=4)
    n_live = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    nb.np_kv_compact(c.desc, c.cache, c.tables, c.tables, n_live)
    c.check()
    assert n_live.item() == 0
    c.grow([0, 1], [40, 16])
    before = c.cache.clone()
    nb.np_kv_compact(c.desc, c.cache, c.tables, c.tables, n_live)
    c.pool.compact()
    c.check()
    assert n_live.item() == 4 and torch.equal(before.view(torch.int16), c.cache.view(torch.int16))


@pytest.mark.parametrize("held", [[], [40, 16], [5]])
def test_compact_into_other_tables_of_empty_full_and_compact_pools(held):
    c = Cache(P=16, n_pages=4, max_seqs=4)
    n_live = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    if held:
        c.grow(list(range(len(held))), held)
    before = c.cache.clone()
    fresh = [torch.full_like(t, 55) for t in (c.table, c.lens, c.refs)]
    nb.np_kv_compact(c.desc, c.cache, c.tables, nb.make_kv_tables(*fresh, None, None), n_live)
    live, moves = c.pool.compact()
    c.table, c.lens, c.refs = fresh
    c.check()
    assert n_live.item() == live and not moves and torch.equal(before.view(torch.int16), c.cache.view(torch.int16))


def test_copy_pages_between_caches():
    c, d = Cache(layers=3, hkv=2, n_pages=6), Cache(layers=3, hkv=2, n_pages=6)
    c.cache.copy_(torch.randn(c.cache.shape, device="cuda"))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_kv_copy_pages(c.desc, d.cache, c.cache, c.dev([5, 0, 6, 2, -1]), c.dev([1, 3, 0, 6, 0]), status)
    torch.cuda.synchronize()
    assert torch.equal(d.cache[:, 1], c.cache[:, 5]) and torch.equal(d.cache[:, 3], c.cache[:, 0])
    assert torch.isnan(d.cache[:, [0, 2, 4, 5]]).all() and status.item() == A.S_PAGE
    nb.np_kv_copy_pages(c.desc, c.cache, c.cache, c.dev([5]), c.dev([4]), status)
    torch.cuda.synchronize()
    assert torch.equal(c.cache[:, 4], c.cache[:, 5])


def test_calls_replay_from_a_graph_on_new_contents():
    """free, reserve, append and fork captured once; each replay follows the arrays' contents of the moment."""
    c = Cache(P=16, n_pages=24, max_seqs=6, hkv=1)
    c.grow([0, 1, 2], [20, 5, 33])
    c.check()
    seqs, n_new, start = c.dev([1, 3]), c.dev([0, 0]), c.dev([0, 0])
    src, dst = c.dev([0]), c.dev([4])
    cu = c.dev([0, 0, 0])
    k, v = (torch.randn(40, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        nb.np_kv_free(c.desc, c.tables, dst, stream=s)
        nb.np_kv_reserve(c.desc, c.tables, seqs, n_new, start, stream=s)
        nb.np_kv_append(c.desc, c.cache, 0, c.tables, k, v, seqs, cu, start, stream=s)
        nb.np_kv_fork(c.desc, c.cache, c.tables, src, dst, stream=s)
    rng = np.random.default_rng(0)
    for t in range(6):
        add, a = rng.integers(0, 20, 2).tolist(), int(rng.integers(0, 4))
        n_new.copy_(torch.tensor(add))
        cu.copy_(torch.tensor([0, add[0], sum(add)]))
        src.fill_(a)
        torch.cuda.synchronize()
        g.replay()
        c.pool.free([4])
        c.pool.reserve([1, 3], add)
        c.pool.fork([a], [4])
        c.check()
        for i, s_ in enumerate([1, 3]):
            gk, _ = c.tokens(0, s_)
            if add[i]:
                at = sum(add[:i])
                assert (gk[-add[i]:] == f64(k[at:at + add[i]])).all()
        assert (c.tokens(0, 4)[0] == c.tokens(0, a)[0]).all()


def test_tensors_of_another_kind_are_refused():
    c = Cache(P=16, n_pages=4, max_seqs=4, hkv=1)
    k = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(nb.NpError):
        nb.np_kv_append(c.desc, c.cache, 0, c.tables, k.half(), k, c.dev([0, 1]), None, c.dev([0, 0]))
    with pytest.raises(nb.NpError):
        nb.np_kv_append(c.desc, c.cache[:, :3], 0, c.tables, k, k, c.dev([0, 1]), None, c.dev([0, 0]))
    with pytest.raises(nb.NpError):
        nb.np_kv_free(c.desc, c.tables, torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(nb.NpError):
        nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([0, 1]), c.dev([2]))


def test_the_most_sequences_at_once():
    """1024 sequences in one call of each kind, every one forked from the same parent but one."""
    c = Cache(P=16, n_pages=3000, max_seqs=1024, hkv=1, max_pages=4)
    c.reserve([0], [35])
    dst = list(range(1, 1024))
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([0] * 1023), c.dev(dst))
    c.pool.fork([0] * 1023, dst)
    c.check()
    c.reserve(list(range(1024)), [(7 * s) % 31 for s in range(1024)])
    c.check()
    nb.np_kv_free(c.desc, c.tables)
    c.pool.free(list(range(1024)))
    c.check()
    assert not c.refs.any()
