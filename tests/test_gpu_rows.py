"""Norm and rotation, rows into and out of 16-bit and 8-bit caches, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from oracle import rows_oracle as R
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, f64
from tests.rows_harness import Held, check_rotated, frequencies

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _dev(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def _cu(counts, front=0):
    return _dev(np.concatenate([[0], np.cumsum(counts)]) + front)


def _qkv(rows, hq, hkv, hd, dtype, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, hq + 2 * hkv, hd, generator=g, device="cuda") * spread).to(dtype)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _gains(hd, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [1 + 0.3 * torch.randn(hd, generator=g, device="cuda") for _ in range(2)]


def _rotation(hd, rot, norms, neighbours, base=10000.0, eps=1e-6):
    freq = frequencies(rot, base)
    qg, kg = _gains(hd)
    qg, kg = qg if "q" in norms else None, kg if "k" in norms else None
    return nb.make_rotation(freq if rot else None, qg, kg, neighbours=neighbours, eps=eps), freq, qg, kg


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd", [(1, 1, 64), (4, 4, 64), (32, 4, 64), (8, 1, 128), (40, 8, 128), (5, 3, 128)])
@pytest.mark.parametrize("rot,norms,neighbours", [(64, "qk", False), (64, "", True), (16, "q", False), (48, "k", True), (48, "qk", False), (0, "qk", False), (0, "", False)])
def test_rotate(dtype, hq, hkv, hd, rot, norms, neighbours):
    """Prompts of 0 to 40 tokens at far positions, passed-over ones among them; rows before, between and behind are left as they were."""
    counts, start = [3, 0, 40, 1, 7, 17], [0, 5, 100000, -1, 77, 2000000000]
    front, pad = 2, 3
    rows = front + sum(counts) + pad
    q, k, _ = _qkv(rows, hq, hkv, hd, dtype)
    r, freq, qg, kg = _rotation(hd, rot * hd // 64, norms, neighbours)
    wide = torch.full((rows, hq + hkv + 1, hd), 7.0, dtype=dtype, device="cuda")
    qo, ko = wide[:, :hq], wide[:, hq:hq + hkv]
    nb.np_attn_rotate(r, q, k, qo, ko, _cu(counts, front), _dev(start))
    torch.cuda.synchronize()
    assert (wide[:, -1] == 7).all()
    at, keep = front, []
    for c, s in zip(counts, start):
        if s < 0:
            assert (wide[at:at + c] == 7).all()
        else:
            keep += [(at + j, s + j) for j in range(c)]
        at += c
    assert (wide[:front] == 7).all() and (wide[at:] == 7).all()
    idx, pos = [i for i, _ in keep], [p for _, p in keep]
    check_rotated(qo[idx], q[idx], qg, 1e-6, pos, freq, neighbours)
    check_rotated(ko[idx], k[idx], kg, 1e-6, pos, freq, neighbours)


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotate_single_tokens_in_place(neighbours):
    """Without cu; the results on top of the inputs; a start of -1 leaves its row."""
    q, k, _ = _qkv(70, 8, 2, 128, BF)
    was_q, was_k = q.clone(), k.clone()
    start = list(range(0, 7000, 100))
    start[11] = -1
    r, freq, qg, kg = _rotation(128, 128, "qk", neighbours)
    nb.np_attn_rotate(r, q, k, q, k, None, _dev(start))
    torch.cuda.synchronize()
    assert torch.equal(q[11], was_q[11]) and torch.equal(k[11], was_k[11])
    idx = [i for i in range(70) if i != 11]
    check_rotated(q[idx], was_q[idx], qg, 1e-6, [start[i] for i in idx], freq, neighbours)
    check_rotated(k[idx], was_k[idx], kg, 1e-6, [start[i] for i in idx], freq, neighbours)


@pytest.mark.parametrize("spread", [1e-30, 1e-12, 1e15, 3e19, 1e37])
def test_norm_over_bf16s_range(spread):
    """Squares past fp32's range, and below it."""
    q, k, _ = _qkv(9, 4, 2, 64, BF, spread=spread)
    q[3, 1] = 0
    r, freq, qg, kg = _rotation(64, 64, "qk", False)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    nb.np_attn_rotate(r, q, k, qo, ko, _cu([9]), _dev([50]))
    check_rotated(qo, q, qg, 1e-6, range(50, 59), freq, False)
    check_rotated(ko, k, kg, 1e-6, range(50, 59), freq, False)
    assert (qo[3, 1] == 0).all()


def test_rotate_of_values_that_are_not_finite():
    """A NaN or an infinity is its row's, with a norm, or its pair's, without one; other rows do not change."""
    q, k, _ = _qkv(4, 4, 2, 64, BF)
    r, freq, qg, _ = _rotation(64, 64, "q", False)
    want_q, want_k = torch.empty_like(q), torch.empty_like(k)
    nb.np_attn_rotate(r, q, k, want_q, want_k, None, _dev([1, 2, 3, 4]))
    q[1, 2, 5], q[2, 0, 63], k[0, 1, 40] = float("nan"), float("inf"), float("inf")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    nb.np_attn_rotate(r, q, k, qo, ko, None, _dev([1, 2, 3, 4]))
    torch.cuda.synchronize()
    assert torch.isnan(qo[1, 2]).all() and torch.isnan(qo[2, 0, [31, 63]]).all() and (qo[2, 0, :31] == 0).all()
    assert not torch.isfinite(ko[0, 1, [8, 40]]).any()
    qo[1, 2], qo[2, 0], ko[0, 1] = want_q[1, 2], want_q[2, 0], want_k[0, 1]
    assert torch.equal(qo, want_q) and torch.equal(ko, want_k)


def test_rows_are_left_alone_by_empty_calls():
    q, k, _ = _qkv(5, 4, 2, 64, BF)
    r = _rotation(64, 64, "qk", False)[0]
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    nb.np_attn_rotate(r, q, k, qo, ko, _cu([0, 0]), _dev([1, 1]))
    nb.np_attn_rotate(r, q, k, qo, ko, _cu([5]), _dev([-1]))
    nb.np_attn_rotate(r, q[:0], k[:0], qo[:0], ko[:0], None, _dev([]))
    torch.cuda.synchronize()
    assert (qo == 7).all() and (ko == 7).all()


def test_rows_of_one_head_and_wide_strides():
    """One head whose stride is anything, tokens far apart."""
    base = torch.randn(6, 5, 1, 64, device="cuda").to(HF)
    q, k = base[:, 0], base[:, 3]
    r, freq, qg, kg = _rotation(64, 64, "qk", True)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    nb.np_attn_rotate(r, q, k, qo, ko, None, _dev(range(6)))
    check_rotated(qo, q, qg, 1e-6, range(6), freq, True)
    check_rotated(ko, k, kg, 1e-6, range(6), freq, True)


# ---- into the cache ---------------------------------------------------------------------


def _pool(kind, dtype, hkv, hd, P, lens, spare=2):
    make = Held if kind == "held" else Cache
    c = make(dtype=dtype, layers=2, hkv=hkv, hd=hd, P=P, n_pages=spare + sum(-(-x // P) for x in lens), max_seqs=len(lens))
    return c


@pytest.mark.parametrize("kind", ["held", "rows"])
@pytest.mark.parametrize("dtype,hq,hkv,hd,P", [(BF, 4, 4, 64, 16), (HF, 8, 1, 128, 64), (BF, 40, 8, 128, 32), (HF, 6, 3, 64, 256)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_append_rotated_is_rotate_and_append(kind, dtype, hq, hkv, hd, P, neighbours):
    """Bit for bit, in the layer concerned, for prompts and then for single tokens; the other layer and unused pages stay."""
    counts = [P + 3, 0, 1, 2 * P, 5]
    c, d = (_pool(kind, dtype, hkv, hd, P, [x + 2 for x in counts]) for _ in range(2))
    r = _rotation(hd, hd // 2 if hd == 128 else hd, "qk", neighbours)[0]
    for step, add in enumerate([counts, [1] * 5, [1] * 5]):
        start, _ = c.reserve(range(5), add)
        d.reserve(range(5), add)
        rows = sum(add)
        q, k, v = _qkv(rows + 2, hq, hkv, hd, dtype, seed=step)
        if step:
            q, k, v = q[:rows], k[:rows], v[:rows]
        cu = None if step else _cu(add)
        qo, q2 = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
        k2 = torch.full_like(k, 7.0)
        nb.np_kv_append_rotated(c.desc, c.cache, 1, c.tables, r, q, k, v, qo, c.dev(range(5)), cu, start)
        nb.np_attn_rotate(r, q, k, q2, k2, cu, start)
        nb.np_kv_append(d.desc, d.cache, 1, d.tables, k2, v, d.dev(range(5)), cu, start)
        torch.cuda.synchronize()
        assert torch.equal(qo, q2)
        assert torch.equal(c.cache.view(torch.uint8), d.cache.view(torch.uint8))
    c.check()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hkv,hd,P", [(1, 64, 16), (3, 128, 32), (8, 128, 256), (2, 64, 64)])
def test_held_rows_are_the_oracles(dtype, hkv, hd, P):
    """Values and exponents, byte for byte, over the whole range of the type; what is not written stays."""
    counts = [P - 1, 1, 0, P + 1, 3 * P]
    c = _pool("held", dtype, hkv, hd, P, counts)
    start, _ = c.reserve(range(5), counts)
    rows = sum(counts)
    _, k, v = _qkv(rows, 1, hkv, hd, dtype)
    k.mul_(torch.logspace(-5, 4, rows, device="cuda")[:, None, None].to(dtype) if dtype == HF else torch.logspace(-36, 36, rows, device="cuda")[:, None, None].to(dtype))
    v[0] = 0
    v[1, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1.0], device="cuda")
    v[2, 0] = torch.finfo(dtype).max
    v[3, 0] = torch.finfo(dtype).smallest_normal / 4
    v[4, 0, 1:] = float("nan")
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k, v, c.dev(range(5)), _cu(counts), start)
    torch.cuda.synchronize()
    c.check()
    at = 0
    for s, n in enumerate(counts):
        gk, gv = c.tokens(0, s)
        for got, x in ((gk, k), (gv, v)):
            want, e = R.hold(f64(x[at:at + n]))
            assert (np.isnan(got) == np.isnan(want)).all() and (np.nan_to_num(got) == np.nan_to_num(want)).all()
        _, e = c.parts(0, c.pool.pages[s])
        stored = e.transpose(1, 0, 3, 2).reshape(2, -1, hkv)
        assert (stored[0, :n] == R.hold(f64(k[at:at + n]))[1]).all() and (stored[1, :n] == R.hold(f64(v[at:at + n]))[1]).all()
        assert (stored[:, n:] == 0x7f).all()
        at += n
    free = c.pool.free_pages()
    assert (c.cache[0, free] == 0x7f).all() and (c.cache[1] == 0x7f).all()


@pytest.mark.parametrize("kind", ["held", "rows"])
@pytest.mark.parametrize("dtype,hkv,hd,P", [(BF, 2, 64, 16), (HF, 5, 128, 64)])
def test_read(kind, dtype, hkv, hd, P):
    """What is there comes back (rounded to the rows' type); rows past a length, of no page and of nobody are left as they were."""
    counts = [2 * P + 5, 0, P, 9, 6]
    c = _pool(kind, dtype, hkv, hd, P, counts)
    c.grow(range(5), counts)
    c.table[2, 0] = -1
    ask, start = [P + 9, 4, 6, 9, 3], [P, 0, 0, 0, -1]
    k, v = (torch.full((sum(ask) + 2, hkv + 1, hd), 7.0, dtype=dtype, device="cuda")[:, :hkv] for _ in range(2))
    nb.np_kv_read(c.desc, c.cache, 1, c.tables, k, v, c.dev(range(5)), _cu(ask), _dev(start))
    torch.cuda.synchronize()
    assert c.status.item() == A.S_PAGE
    tk, tv = c.tokens(1, 0)
    n = 2 * P + 5 - P
    for got, want in ((k, tk), (v, tv)):
        assert (f64(got[:n]) == torch.tensor(want[P:]).to(dtype).double().numpy()).all()
        assert (got[n:P + 9] == 7).all() and (got[P + 9:P + 19] == 7).all() and (got[P + 28:] == 7).all()
    tk, tv = c.tokens(1, 3)
    assert (f64(k[P + 19:P + 28]) == torch.tensor(tk).to(dtype).double().numpy()).all() and (f64(v[P + 19:P + 28]) == torch.tensor(tv).to(dtype).double().numpy()).all()


def test_finite_values_stay_finite_when_read():
    """The largest number of fp16 is held as 65536; a bf16 near the end of its range as 2^128."""
    for dtype in (HF, BF):
        c = _pool("held", dtype, 1, 64, 16, [3])
        start, _ = c.reserve([0], [3])
        x = torch.full((3, 1, 64), torch.finfo(dtype).max, dtype=dtype, device="cuda")
        x[1] *= -1
        x[2, 0, 5] = float("inf")
        k, v = torch.empty_like(x), torch.empty_like(x)
        nb.np_kv_append(c.desc, c.cache, 0, c.tables, x, x, c.dev([0]), _cu([3]), start)
        nb.np_kv_read(c.desc, c.cache, 0, c.tables, k, v, c.dev([0]), _cu([3]), start)
        torch.cuda.synchronize()
        want = x.clone()
        want[2, 0, 5] = 0
        k[2, 0, 5] = torch.where(torch.isnan(k[2, 0, 5]), torch.zeros_like(k[2, 0, 5]), k[2, 0, 5])
        assert torch.equal(k, want) and torch.isnan(v[2, 0, 5])


def test_append_rotated_leaves_out_what_has_no_place():
    """Positions past a length, pages outside the pool, sequences outside the tables: keys and values are not written, queries are rotated."""
    for kind in ("held", "rows"):
        c = _pool(kind, BF, 2, 64, 16, [20, 20, 20], spare=4)
        c.grow(range(3), [20, 20, 20])
        before = c.cache.clone()
        c.table[1, 1] = 1 << 20
        q, k, v = _qkv(4, 4, 2, 64, BF)
        r, freq, qg, _ = _rotation(64, 64, "qk", False)
        qo = torch.full_like(q, 7.0)
        nb.np_kv_append_rotated(c.desc, c.cache, 0, c.tables, r, q[:3], k[:3], v[:3], qo[:3], c.dev([0, 1, 9]), None, _dev([20, 17, 3]))
        torch.cuda.synchronize()
        assert torch.equal(c.cache.view(torch.uint8), before.view(torch.uint8))
        assert c.status.item() == A.S_PAGE | A.S_SEQ
        check_rotated(qo[:3], q[:3], qg, 1e-6, [20, 17, 3], freq, False)
        assert (qo[3] == 7).all()


def test_pages_of_8_bits_are_forked_compacted_and_copied():
    """The calls that move whole pages, over a cache of 8 bits."""
    c = Held(layers=2, hkv=2, hd=64, P=16, n_pages=40, max_seqs=6)
    c.grow([0, 1, 2], [37, 5, 64])
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([0, 2]), c.dev([3, 4]))
    c.pool.fork([0, 2], [3, 4])
    c.check()
    for layer in (0, 1):
        for a, b in ((0, 3), (2, 4)):
            for x, y in zip(c.tokens(layer, a), c.tokens(layer, b)):
                assert (x == y).all()
    want = {(layer, s): c.tokens(layer, s) for layer in (0, 1) for s in range(5)}
    nb.np_kv_free(c.desc, c.tables, c.dev([1]))
    c.pool.free([1])
    live = _dev([0])
    nb.np_kv_compact(c.desc, c.cache, c.tables, c.tables, live)
    c.pool.compact()
    c.check()
    for (layer, s), kv in want.items():
        if s != 1:
            for x, y in zip(c.tokens(layer, s), kv):
                assert (x == y).all()


def test_held_rows_past_32_bit_offsets():
    """A cache of more than 4 GB, with the sequence's pages at its end."""
    page = 2 * 8 * 256 * 129
    n_pages = (1 << 32) // page + 12
    c = Held(hkv=8, hd=128, P=256, n_pages=n_pages, max_seqs=2)
    c.reserve([0], [256 * (n_pages - 3)])
    start, _ = c.reserve([1], [500])
    k, v = c.append(0, [1], start, [500])
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    nb.np_kv_read(c.desc, c.cache, 0, c.tables, ko, vo, c.dev([1]), _cu([500]), start)
    torch.cuda.synchronize()
    assert (f64(ko) == R.hold(f64(k))[0]).all() and (f64(vo) == R.hold(f64(v))[0]).all()


def test_rows_on_a_stream_of_their_own_and_replayed():
    """Captured with a reserve before it: the replays go on where the last one left off."""
    c, d = (Held(hkv=2, hd=64, P=16, n_pages=30, max_seqs=2) for _ in range(2))
    r = _rotation(64, 64, "qk", False)[0]
    q, k, v = _qkv(2, 4, 2, 64, BF)
    qo, start, one = torch.empty_like(q), _dev([0, 0]), _dev([1, 1])
    seqs = _dev([0, 1])
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        nb.np_kv_reserve(c.desc, c.tables, seqs, one, start, stream=s)
        nb.np_kv_append_rotated(c.desc, c.cache, 0, c.tables, r, q, k, v, qo, seqs, None, start, stream=s)
    for t in range(20):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda").to(BF))
        g.replay()
        c.pool.reserve([0, 1], [1, 1])
        at, _ = d.reserve([0, 1], [1, 1])
        q2, k2 = torch.empty_like(q), torch.empty_like(k)
        nb.np_attn_rotate(r, q, k, q2, k2, None, at)
        nb.np_kv_append(d.desc, d.cache, 0, d.tables, k2, v, seqs, None, at)
        torch.cuda.synchronize()
        assert torch.equal(qo, q2)
    c.check()
    assert torch.equal(c.cache, d.cache)


@pytest.mark.parametrize("dtype,hq,hkv,hd,neighbours", [(BF, 1, 1, 64, True), (HF, 9, 3, 128, False), (BF, 64, 8, 128, False)])
def test_rotate_many_tokens_as_few(dtype, hq, hkv, hd, neighbours):
    """Calls of tens of millions of values give what pieces of them give, bit for bit."""
    rows = (1 << 25) // (hq + hkv) // hd + 1001
    q, k, _ = _qkv(rows, hq, hkv, hd, dtype)
    r = _rotation(hd, hd, "qk", neighbours)[0]
    a, b = (torch.full((rows + 1, hq + hkv, hd), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    first = 12345
    start = _dev([77, 100000])
    cu = [0, rows // 3, rows]
    nb.np_attn_rotate(r, q, k, a[:rows, :hq], a[:rows, hq:], _dev(cu), start)
    for lo in range(0, rows, first):                          # a piece: the same two spans, cut
        hi = min(rows, lo + first)
        spans = [min(max(x, lo), hi) for x in cu]
        where = _dev([77 + spans[0], 100000 + spans[1] - cu[1]])
        nb.np_attn_rotate(r, q[lo:hi], k[lo:hi], b[lo:hi, :hq], b[lo:hi, hq:], _dev([x - lo for x in spans]), where)
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and (a[rows] == 7).all()


@pytest.mark.parametrize("kind", ["held", "rows"])
@pytest.mark.parametrize("dtype,hq,hkv,hd,P", [(BF, 20, 20, 64, 16), (HF, 40, 8, 128, 64)])
def test_append_rotated_many_tokens(kind, dtype, hq, hkv, hd, P):
    """A call of tens of millions of values, into a cache: rotate and append, bit for bit."""
    n = (1 << 25) // (hq + 2 * hkv) // hd + 333
    counts = [n // 2, 0, n - n // 2]
    c, d = (_pool(kind, dtype, hkv, hd, P, counts) for _ in range(2))
    r = _rotation(hd, hd, "qk", False)[0]
    start, _ = c.reserve(range(3), counts)
    d.reserve(range(3), counts)
    q, k, v = _qkv(n, hq, hkv, hd, dtype)
    qo, q2, k2 = torch.full_like(q, 7.0), torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    nb.np_kv_append_rotated(c.desc, c.cache, 1, c.tables, r, q, k, v, qo, c.dev(range(3)), _cu(counts), start)
    nb.np_attn_rotate(r, q, k, q2, k2, _cu(counts), start)
    nb.np_kv_append(d.desc, d.cache, 1, d.tables, k2, v, d.dev(range(3)), _cu(counts), start)
    torch.cuda.synchronize()
    assert torch.equal(qo, q2) and torch.equal(c.cache.view(torch.uint8), d.cache.view(torch.uint8))
    assert c.status.item() == 0
