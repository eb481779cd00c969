"""Attention of branches that share a prefix, and what they share, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, check_rows, f64
from tests.rows_harness import Held, check_held_rows

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _workspace(c, hq, n):
    return torch.full((nb.np_attn_shared_workspace_bytes(c.desc, hq, n),), 0, dtype=torch.uint8, device="cuda")


def _shared(c, seqs, cu):
    held = torch.full((len(cu) - 1,), -7, dtype=torch.int32, device="cuda")
    nb.np_kv_shared(c.desc, c.tables, None if seqs is None else c.dev(seqs), c.dev(cu), held)
    return held


def _common(c, seqs, cu):
    """What np_kv_shared has to say, from the oracle's pool."""
    got = []
    for lo, hi in zip(cu, cu[1:]):
        rows = [(c.pool.pages[s], c.pool.lens[s] // c.P) for s in seqs[lo:hi] if s >= 0]
        n = 0
        while len(rows) > 1 and all(n < full and r[n] == rows[0][0][n] for r, full in rows):
            n += 1
        got.append(n * c.P)
    return got


def _run(c, hq, seqs, cu, held, layer=0, seed=0, ws=None, spread=1.0, check=True):
    n = len(seqs)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (torch.randn(n, hq + 3, c.hd, generator=g, device="cuda") * spread).to(c.dtype)[:, 1:hq + 1]
    room = torch.full((n + 1, hq + 1, c.hd), 7.0, dtype=c.dtype, device="cuda")
    out, lse = room[:n, :hq], torch.full((n + 1, hq), 7.0, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, layer, c.tables, q, out, _workspace(c, hq, n) if ws is None else ws, c.dev(cu), held, seqs=c.dev(seqs), lse=lse[:n])
    torch.cuda.synchronize()
    assert (room[n] == 7).all() and (room[:, hq] == 7).all() and (lse[n] == 7).all()
    if check:
        none = np.zeros((0, c.hkv, c.hd))
        kept = {s: c.tokens(layer, s) for s in set(seqs) if s >= 0}
        (check_held_rows(out, lse[:n], q, lambda i: kept.get(seqs[i], (none, none)), c.hd ** -0.5) if isinstance(c, Held) else
         check_rows(out, lse[:n], q, lambda i: kept.get(seqs[i], (none, none)), c.hd ** -0.5, True))
    return q, out, lse[:n]


def _branches(dtype, hkv, hd, P, groups, tails, layers=1, make=Cache):
    """groups: tokens of each parent; tails: for each parent the own tokens of its branches.  Parents are freed.  (cache, sequences, cu)."""
    n = sum(len(t) for t in tails)
    pages = sum(-(-x // P) for x in groups) + sum(-(-x // P) + 2 for t in tails for x in t) + 3
    c = make(dtype=dtype, layers=layers, hkv=hkv, hd=hd, P=P, n_pages=pages, max_seqs=n + len(groups))
    src, dst, own = [], [], []
    for i, (x, t) in enumerate(zip(groups, tails)):
        c.grow([n + i], [x], seed=50 + i)
        for y in t:
            src.append(n + i)
            dst.append(len(dst))
            own.append(y)
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev(src), c.dev(dst))
    c.pool.fork(src, dst)
    nb.np_kv_free(c.desc, c.tables, c.dev(range(n, n + len(groups))))
    c.pool.free(list(range(n, n + len(groups))))
    c.grow(dst, own, seed=9)
    c.check()
    return c, dst, np.concatenate([[0], np.cumsum([len(t) for t in tails])]).tolist()


CASES = [
    # dtype, query heads, key-value heads, head_dim, page, tokens of parents, own tokens of branches
    (HF, 4, 4, 64, 16, [100], [[0, 3]]),
    (BF, 4, 4, 128, 64, [640], [[1] * 7]),
    (BF, 8, 1, 128, 16, [16], [[5, 0, 40]]),
    (HF, 16, 2, 64, 32, [1000, 33, 320], [[2, 700, 0, 9], [1, 1], [3] * 20]),
    (BF, 32, 4, 128, 256, [2048, 256], [[17, 300], [0, 0, 5]]),
    (BF, 40, 8, 128, 128, [5000], [[30] * 5]),
    (HF, 48, 1, 128, 64, [700], [[9] * 11]),
    (BF, 12, 12, 64, 16, [4000], [[0] * 150]),
    (BF, 8, 8, 64, 64, [9000, 64, 128], [[100, 5], [7, 7], [0, 1]]),
    (HF, 6, 2, 128, 16, [333], [[2] * 90]),
    (BF, 128, 1, 64, 32, [512], [[3, 3, 3]]),
    (HF, 20, 10, 128, 16, [260], [[40] * 70 + [900, 0]]),
    (BF, 7, 7, 64, 32, [96, 64], [[130] * 60, [1] * 70]),
]


@pytest.mark.parametrize("dtype,hq,hkv,hd,P,groups,tails", CASES)
def test_branches(dtype, hq, hkv, hd, P, groups, tails):
    """Groups of two to a hundred and fifty branches, prefixes of a page to thousands of tokens, branches without tokens of their own; twice gives
    the same bits."""
    c, seqs, cu = _branches(dtype, hkv, hd, P, groups, tails, layers=2)
    held = _shared(c, seqs, cu)
    assert held.tolist() == _common(c, seqs, cu) == [x // P * P for x in groups]
    ws = _workspace(c, hq, len(seqs))
    _, a, la = _run(c, hq, seqs, cu, held, layer=1, ws=ws)
    _, b, lb = _run(c, hq, seqs, cu, held, layer=1, ws=ws, check=False)
    assert torch.equal(a, b) and torch.equal(la, lb)
    assert c.status.item() == 0


@pytest.mark.parametrize("dtype,hq,hkv,hd", [(BF, 4, 4, 64), (HF, 16, 2, 128)])
def test_less_than_is_shared_will_do(dtype, hq, hkv, hd):
    """Any multiple of a page up to what is shared; nothing at all; rows outside of the groups; rows of no sequence."""
    c, seqs, _ = _branches(dtype, hkv, hd, 32, [500, 300], [[20, 0, 4], [9, 8]])
    for cu, held in (([0, 3, 5], [480, 288]), ([0, 3, 5], [32, 0]), ([0, 3, 5], [0, 0]), ([1, 3], [448]), ([0, 2], [64]), ([3, 3, 5], [0, 256]), ([0, 0], [32])):
        _run(c, hq, seqs, cu, c.dev(held), seed=len(held))
    _run(c, hq, [-1, 0, 1, -3, 2, 4, 3, -1], [0, 5, 8], c.dev([480, 288]))
    _run(c, hq, [0, 0, 1, 0], [0, 4], c.dev([480]))
    assert c.status.item() == 0


def test_what_groups_cannot_share_they_do_not():
    """More than a row has, and what fills no pages: the group shares nothing, the result stands, and a bit says so."""
    for bad in (496, 17, -16):
        c, seqs, cu = _branches(BF, 2, 64, 16, [490], [[20, 0, 4]])
        _run(c, 4, seqs, cu, c.dev([bad]))
        assert c.status.item() == A.S_LENGTH


def test_a_group_that_is_longer_than_its_sequences_of_another():
    """A sequence outside the tables, a length outside its row: empty rows; the rest of the group is as it was."""
    c, seqs, cu = _branches(BF, 2, 64, 16, [160], [[20, 0, 4, 6]])
    want = _run(c, 4, seqs, cu, c.dev([160]))[1]
    q = _run(c, 4, seqs, cu, c.dev([160]))[0]
    c.lens[3] = 16 * c.desc.max_pages + 1
    out, lse = torch.empty_like(want), torch.empty(4, 4, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 4, 4), c.dev(cu), c.dev([160]), seqs=c.dev([0, 99, 2, 3]), lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == A.S_SEQ | A.S_LENGTH
    assert (out[[1, 3]] == 0).all() and (lse[[1, 3]] == -float("inf")).all()
    assert torch.equal(out[[0, 2]], want[[0, 2]])


@pytest.mark.parametrize("hq,hkv", [(4, 2), (16, 2), (64, 2), (2, 2)])
def test_rows_whose_length_their_table_does_not_hold(hq, hkv):
    """Such a row is empty, and one of a sequence that is none, in small groups and large ones; the rest of its group is as it was."""
    c, seqs, cu = _branches(BF, hkv, 64, 16, [160], [[20, 0, 4, 6] * 10])
    held = c.dev([160])
    q, want, _ = _run(c, hq, seqs, cu, held)
    for row, n in ((3, 16 * c.desc.max_pages + 1), (17, 2 ** 31 - 1)):
        c.lens[row] = n
    seqs[5], seqs[9] = c.desc.max_seqs, -2
    out, lse = torch.empty_like(want), torch.empty(40, hq, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, hq, 40), c.dev(cu), held, seqs=c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == A.S_LENGTH | A.S_SEQ
    empty = [3, 5, 9, 17]
    assert (out[empty] == 0).all() and (lse[empty] == -float("inf")).all()
    others = [i for i in range(40) if i not in empty]
    assert torch.equal(out[others], want[others])


def test_shared_pages_that_are_not_there():
    """A page number outside the pool among the shared ones: its tokens are not seen by any row."""
    for ways in (3, 40):
        _shared_pages_that_are_not_there(ways)


def _shared_pages_that_are_not_there(ways):
    c, seqs, cu = _branches(BF, 2, 64, 16, [400], [[20, 0, 4] + [1] * (ways - 3)])
    kept = {s: c.tokens(0, s) for s in seqs}
    c.table[:, 3] = c.desc.n_pages
    c.table[:, 20] = -1
    q, out, lse = _run(c, 4, seqs, cu, c.dev([400]), check=False)
    assert c.status.item() == A.S_PAGE
    seen = np.r_[0:48, 64:320, 336:10 ** 6]
    check_rows(out, lse, q, lambda i: tuple(x[seen[seen < len(x)]] for x in kept[seqs[i]]), 0.125, True)
    c.table[:, :25] = -1                                      # none of them
    q, out, lse = _run(c, 4, seqs, cu, c.dev([400]), check=False)
    check_rows(out, lse, q, lambda i: tuple(x[400:] for x in kept[seqs[i]]), 0.125, True)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_values_that_are_not_finite(dtype):
    """Infinities and NaN among shared values show in all rows of the group; scores of -inf leave nothing."""
    c, seqs, cu = _branches(dtype, 1, 64, 16, [400, 64], [[20, 0, 4], [3, 0]])
    pages = c.pool.pages[0]
    c.cache[0, pages[2], 1, 0, 5, 10] = float("inf")
    c.cache[0, pages[20], 1, 0, 5, 10] = float("inf")
    c.cache[0, pages[7], 1, 0, 1, 11] = -float("inf")
    c.cache[0, pages[7], 1, 0, 1, 12], c.cache[0, pages[9], 1, 0, 1, 12] = float("inf"), -float("inf")
    c.cache[0, pages[1], 1, 0, 1, 13] = float("nan")
    c.cache[0, c.pool.pages[3][:4], 0] = -float("inf")        # all shared keys of the second group
    c.cache[0, c.pool.pages[3][1], 1] = float("inf")          # whose values nobody sees then
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(5, 2, 64, generator=g, device="cuda").abs().to(dtype)
    out, lse = torch.empty_like(q), torch.empty(5, 2, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 2, 5), c.dev(cu), c.dev([400, 64]), seqs=c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    o = out[:3].float()
    assert (o[..., 10] == float("inf")).all() and (o[..., 11] == -float("inf")).all() and torch.isnan(o[..., 12:14]).all()
    fine = [i for i in range(64) if i not in (10, 11, 12, 13)]
    assert torch.isfinite(o[..., fine]).all() and torch.isfinite(lse[:3]).all()
    k, v = c.tokens(0, 3)
    check_rows(out[3:4], lse[3:4], q[3:4], lambda i: (k[64:], v[64:]), 0.125, True)
    assert (out[4] == 0).all() and (lse[4] == -float("inf")).all()


@pytest.mark.parametrize("ways,hq", [(3, 2), (40, 2), (6, 8)])
def test_infinities_among_shared_and_own_values(ways, hq):
    """Small groups and large ones: an infinity of either kind of token stays one however small its weight, two of different signs make a NaN."""
    c, seqs, cu = _branches(BF, 1, 64, 16, [800], [[20, 300] + [1] * (ways - 2)])
    inf = float("inf")
    pages, own = c.pool.pages[0], c.pool.pages[1][50:]
    c.cache[0, pages[2], 1, 0, 5, 10] = inf
    c.cache[0, pages[3], 1, 0, 5, 11] = -inf
    c.cache[0, own[1], 1, 0, 3, 10] = -inf
    c.cache[0, own[1], 1, 0, 3, 11] = -inf
    c.cache[0, own[2], 1, 0, 3, 12] = inf
    c.cache[0, own[0], 1, 0, 3, 13] = float("nan")
    c.cache[0, pages[2:4], 0] *= 0.01                          # small weights beside large ones
    q = (torch.randn(ways, hq, 64, device="cuda") * 12).to(BF)
    out, lse = torch.empty_like(q), torch.empty(ways, hq, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, hq, ways), c.dev(cu), c.dev([800]), seqs=c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    o = out.float()
    others = [i for i in range(ways) if i != 1]
    assert (o[others, :, 10] == inf).all() and (o[others, :, 11] == -inf).all()
    assert torch.isnan(o[1, :, 10]).all() and (o[1, :, 11] == -inf).all() and (o[1, :, 12] == inf).all() and torch.isnan(o[1, :, 13]).all()
    fine = [d for d in range(64) if d not in (10, 11, 12, 13)]
    assert torch.isfinite(o[..., fine]).all() and torch.isfinite(o[others][..., 12:14]).all() and torch.isfinite(lse).all()


def test_more_groups_than_are_kept_in_mind():
    """Large groups among hundreds of empty ones, and of groups without rows that claim what nobody has."""
    c, seqs, cu = _branches(HF, 1, 64, 16, [160, 48], [[3] * 30, [20] * 40])
    many = [0, 30] + [30] * 520 + [70]
    held = c.dev([160] + [0] * 260 + [64] * 260 + [48])
    ws = _workspace(c, 128, 70)
    _, a, la = _run(c, 128, seqs, many, held, ws=ws)
    _, b, lb = _run(c, 128, seqs, many, held, ws=ws, check=False)
    assert torch.equal(a, b) and torch.equal(la, lb) and c.status.item() == 0


def test_infinities_among_own_values_of_many_heads():
    """Rows times key-value heads fill the GPU more than once: an infinity shows in the heads that read it, and in no other."""
    c, seqs, cu = _branches(HF, 10, 64, 16, [160], [[20] * 70])
    inf = float("inf")
    c.cache[0, c.pool.pages[5][10], 1, 9, 3, 10] = inf
    c.cache[0, c.pool.pages[6][11], 1, 4, 2, 11] = -inf
    c.cache[0, c.pool.pages[6][10], 1, 5, 2, 12] = float("nan")
    held = c.dev([160])
    q = torch.randn(70, 20, 64, device="cuda").to(HF)
    out, lse = torch.empty_like(q), torch.empty(70, 20, device="cuda")
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 20, 70), c.dev(cu), held, seqs=c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    o = out.float()
    assert (o[5, 18:, 10] == inf).all() and (o[6, 8:10, 11] == -inf).all() and torch.isnan(o[6, 10:12, 12]).all()
    o[5, 18:, 10] = o[6, 8:10, 11] = o[6, 10:12, 12] = 0
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_peaked_scores():
    """Scores that differ by hundreds, within the prefix and between it and the own tokens."""
    for hq in (2, 16):
        c, seqs, cu = _branches(BF, 2, 128, 32, [1500], [[40, 300, 0, 7]])
        _run(c, hq, seqs, cu, c.dev([1472]), spread=15.0)
        c.cache[0, c.pool.pages[0][:30], 0] *= 0.01
        _run(c, hq, seqs, cu, c.dev([1472]), spread=20.0)


def test_prefix_past_32_bit_offsets():
    n_pages = (1 << 32) // (2 * 2 * 8 * 256 * 128) + 12
    c = Cache(hkv=8, hd=128, P=256, n_pages=n_pages, max_seqs=4, fill=0.0)
    c.reserve([0], [256 * (n_pages - 7)])
    c.grow([1], [1024])
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([1, 1]), c.dev([2, 3]))
    c.pool.fork([1, 1], [2, 3])
    c.grow([2, 3], [5, 0])
    seqs, cu = [1, 2, 3], [0, 3]
    held = _shared(c, seqs, cu)
    assert held.tolist() == [1024]
    _run(c, 16, seqs, cu, held)


def test_a_cache_of_8_bits():
    """Every row by itself, with the same result."""
    c, seqs, cu = _branches(BF, 2, 64, 16, [400, 64], [[20, 0, 4], [3, 0]], make=Held)
    held = _shared(c, seqs, cu)
    assert held.tolist() == [400, 64]
    q, out, lse = _run(c, 8, seqs, cu, held)
    want = torch.empty_like(out)
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, want, _workspace(c, 8, 5), seqs=c.dev(seqs))
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_captured_with_what_is_shared():
    """Captured with np_kv_shared before it and np_attn_decode behind it, replayed while the branches grow."""
    c, seqs, cu = _branches(BF, 2, 64, 16, [400, 640], [[20, 0, 4], [3, 0]])
    ws = _workspace(c, 8, 5)
    other = torch.zeros(nb.np_attn_workspace_bytes(c.desc, 8, 5), dtype=torch.uint8, device="cuda")
    q = torch.randn(5, 8, 64, device="cuda").to(BF)
    out, plain, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(5, 8, device="cuda")
    held, cu_dev, seq_dev = c.dev([0, 0]), c.dev(cu), c.dev(seqs)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        nb.np_kv_shared(c.desc, c.tables, seq_dev, cu_dev, held, stream=s)
        nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, ws, cu_dev, held, seqs=seq_dev, lse=lse, stream=s)
        nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, plain, other, seqs=seq_dev, stream=s)
    for t in range(5):
        c.grow(seqs, [t, 17, 0, 1, 2], seed=t)
        q.copy_(torch.randn(q.shape, device="cuda").to(BF))
        g.replay()
        torch.cuda.synchronize()
        kept = {x: c.tokens(0, x) for x in seqs}
        check_rows(out, lse, q, lambda i: kept[seqs[i]], 0.125, True)
        check_rows(plain, lse, q, lambda i: kept[seqs[i]], 0.125, False)


def test_streams_of_their_own():
    c, seqs, cu = _branches(BF, 4, 64, 16, [1600], [[100, 0, 30, 9]])
    q = torch.randn(4, 8, 64, device="cuda").to(BF)
    want, held, cu_dev = torch.empty_like(q), c.dev([1600]), c.dev(cu)
    nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, want, _workspace(c, 8, 4), cu_dev, held)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    spaces = [_workspace(c, 8, 4) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, ws in zip(streams, spaces):
            with torch.cuda.stream(s):
                o = torch.empty_like(q)
                nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, o, ws, cu_dev, held, stream=s)
                outs.append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_calls_one_behind_the_other():
    """Without a pause between them each call sees what the call before it has written: tokens appended between layers' calls, one workspace."""
    c, seqs, cu = _branches(BF, 2, 64, 16, [1600], [[30] * 12], layers=4)
    held, cu_dev, seq_dev, ws = c.dev([1600]), c.dev(cu), c.dev(seqs), _workspace(c, 8, 12)
    one = c.dev([1] * 12)
    outs, qs = [], []
    start = c.dev([0] * 12)
    nb.np_kv_reserve(c.desc, c.tables, seq_dev, one, start)
    c.pool.reserve(seqs, [1] * 12)
    kv = [[torch.randn(12, 2, 64, device="cuda").to(BF) for _ in range(2)] for _ in range(4)]
    for layer in range(4):
        q = torch.randn(12, 8, 64, device="cuda").to(BF)
        out = torch.empty_like(q)
        nb.np_kv_append(c.desc, c.cache, layer, c.tables, *kv[layer], seq_dev, None, start)
        nb.np_attn_decode_shared(c.desc, c.cache, layer, c.tables, q, out, ws, cu_dev, held, seqs=seq_dev)
        qs.append(q)
        outs.append(out)
    torch.cuda.synchronize()
    for layer in range(4):
        lse = torch.empty(12, 8, device="cuda")
        want = torch.empty_like(outs[layer])
        nb.np_attn_decode_shared(c.desc, c.cache, layer, c.tables, qs[layer], want, ws, cu_dev, held, seqs=seq_dev, lse=lse)
        torch.cuda.synchronize()
        assert torch.equal(want, outs[layer])
        check_rows(want, lse, qs[layer], lambda i: c.tokens(layer, seqs[i]), 0.125, True)


def test_one_workspace_serves_calls_of_all_sizes():
    """Few rows and many, small groups and large ones, both head sizes, 8 bits and nothing shared, one behind the other over one workspace."""
    small, seqs, cu = _branches(BF, 2, 64, 16, [3000, 300], [[20, 700, 4], [3, 0]])
    large, seqs2, cu2 = _branches(HF, 4, 128, 64, [2000], [[30, 5, 0] * 30])
    held, seqs3, cu3 = _branches(BF, 2, 64, 16, [4000], [[20, 0, 4]], make=Held)
    ws = torch.zeros(max(nb.np_attn_shared_workspace_bytes(small.desc, 40, 5), nb.np_attn_shared_workspace_bytes(large.desc, 16, 90)), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        _run(small, 2, seqs, cu, small.dev([2992, 288]), ws=ws)
        _run(large, 16, seqs2, cu2, large.dev([1984]), ws=ws)
        _run(held, 40, seqs3, cu3, held.dev([4000]), ws=ws)
        _run(small, 40, seqs, cu, small.dev([2992, 288]), ws=ws)
        _run(small, 4, seqs, [0], small.dev([]), ws=ws)
        _run(large, 4, seqs2, cu2, large.dev([64]), ws=ws)


# ---- what is shared ---------------------------------------------------------------------


def test_shared_tokens_follow_the_tables():
    """Forks of forks, strangers, copies that went their own way, empty rows."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=200, max_seqs=12)
    c.grow([0], [100])

    def fork(a, b):
        nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev(a), c.dev(b))
        c.pool.fork(a, b)

    fork([0, 0], [1, 2])
    c.grow([1, 2], [30, 30])
    fork([1, 1], [3, 4])
    c.grow([3, 4], [16, 40])
    c.grow([5], [100])
    c.check()
    for seqs, cu in (([0, 1, 2], [0, 3]), ([1, 3, 4], [0, 3]), ([3, 4], [0, 2]), ([0, 5], [0, 2]), ([6, 0], [0, 2]), ([3, -1, 4, 1], [0, 4]), ([3], [0, 1]),
                     ([3, -1], [0, 2]), ([4, 4], [0, 2]), ([0, 1, 2, 3, 4, 5], [0, 3, 3, 5, 6]), ([3, 4, 0], [0, 2]), ([-1, -1], [0, 2])):
        assert _shared(c, seqs, cu).tolist() == _common(c, seqs, cu), (seqs, cu)
    assert _shared(c, None, [0, 3, 5]).tolist() == _common(c, list(range(12)), [0, 3, 5])
    assert c.status.item() == 0


def test_shared_tokens_of_long_tables():
    """More pages than a block has threads, the difference at any of them."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=4000, max_seqs=40, fill=0.0)
    c.reserve([0], [16 * 1500])
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([0] * 39), c.dev(range(1, 40)))
    c.pool.fork([0] * 39, list(range(1, 40)))
    seqs = list(range(40))
    for at in (None, 1499, 1024, 1023, 512, 511, 1, 0):
        if at is not None:
            c.table[37, at] = 3999
        assert _shared(c, seqs, [0, 40]).item() == 16 * (1500 if at is None else at)
    c.table[:, 700] = 4000                                    # the same for all, and no page
    assert _shared(c, seqs[:30], [0, 30]).item() == 16 * 700


def test_shared_tokens_of_rows_outside_the_tables():
    c = Cache(hkv=1, hd=64, P=16, n_pages=20, max_seqs=4, max_pages=6)
    c.grow([0], [64])
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([0, 0]), c.dev([1, 2]))
    assert _shared(c, [0, 99, 1], [0, 3]).item() == 64 and c.status.item() == A.S_SEQ
    c.lens[2] = 97
    assert _shared(c, [0, 1, 2], [0, 3]).item() == 0 and c.status.item() == A.S_SEQ | A.S_LENGTH
