"""Decode attention over a cache of 8 bits against the 64-bit oracle, every element within its own bound."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import f64
from tests.rows_harness import Held, check_held_rows

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _workspace(c, hq, n):
    return torch.zeros(nb.np_attn_workspace_bytes(c.desc, hq, n), dtype=torch.uint8, device="cuda")


def _decode(c, hq, seqs=None, layer=0, seed=0, scale=None, ws=None, spread=1.0):
    """One call on random queries that are slices of a wider tensor; checked against the oracle."""
    n = len(seqs) if seqs is not None else c.desc.max_seqs
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (torch.randn(n, hq + 3, c.hd, generator=g, device="cuda") * spread).to(c.dtype)[:, 1:hq + 1]
    room = torch.full((n + 1, hq + 1, c.hd), 7.0, dtype=c.dtype, device="cuda")
    out, lse = room[:n, :hq], torch.full((n + 1, hq), 7.0, device="cuda")
    scale = c.hd ** -0.5 if scale is None else scale
    nb.np_attn_decode(c.desc, c.cache, layer, c.tables, q, out, _workspace(c, hq, n) if ws is None else ws,
                      seqs=None if seqs is None else c.dev(seqs), scale=scale, lse=lse[:n])
    torch.cuda.synchronize()
    assert (room[n] == 7).all() and (room[:, hq] == 7).all() and (lse[n] == 7).all()
    none = np.zeros((0, c.hkv, c.hd))

    def sees(i):
        s = i if seqs is None else seqs[i]
        return c.tokens(layer, s) if 0 <= s < c.desc.max_seqs else (none, none)

    check_held_rows(out, lse[:n], q, sees, scale)
    return q, out, lse[:n]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd,P", [(1, 1, 64, 16), (4, 4, 128, 64), (8, 1, 128, 32), (14, 2, 64, 256), (16, 1, 128, 16), (40, 8, 128, 128), (34, 2, 64, 64),
                                         (96, 2, 128, 16), (9, 1, 64, 16)])
def test_decode(dtype, hq, hkv, hd, P):
    """Lengths around tiles and pages; none at all; groups of one to forty-eight heads."""
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 130, 257, 700]
    c = Held(dtype=dtype, layers=2, hkv=hkv, hd=hd, P=P, n_pages=2 + sum(-(-x // P) for x in lens), max_seqs=len(lens))
    order = np.random.default_rng(1).permutation(len(lens)).tolist()
    for s in order:                           # pages of the sequences are mixed
        c.grow([s], [lens[s] // 2], seed=s)
    for s in order[::-1]:
        c.grow([s], [lens[s] - lens[s] // 2], seed=100 + s)
    c.check()
    _decode(c, hq, layer=1)
    _decode(c, hq, layer=0, seqs=[11, 3, -1, 0, 11, 1, -5], seed=2)      # any order, twice the same, padding
    c.check()


@pytest.mark.parametrize("lens,hq,hkv,hd", [([20000], 8, 1, 128), ([20000, 3, 0, 9000], 4, 2, 64), ([1] * 300, 2, 2, 64), ([5000] + [40] * 63, 16, 16, 64), ([900] * 148, 4, 4, 64),
                                            ([3000] * 7, 12, 1, 128)])
def test_decode_splits_of_all_sizes(lens, hq, hkv, hd):
    """One long sequence over all blocks, long ones among short ones, more rows than blocks; twice into the same workspace gives the
    same bits."""
    c = Held(hkv=hkv, hd=hd, P=64, n_pages=sum(-(-x // 64) for x in lens), max_seqs=len(lens))
    c.grow(list(range(len(lens))), lens)
    ws = _workspace(c, hq, len(lens))
    _, a, la = _decode(c, hq, ws=ws)
    _, b, lb = _decode(c, hq, ws=ws)
    assert torch.equal(a, b) and torch.equal(la, lb)


def _set(c, layer, s, values, exponents):
    """Writes a sequence's rows: values uint8 [2][hkv][tokens][hd], exponents [2][hkv][tokens]."""
    split = 2 * c.hkv * c.P * c.hd
    for j, p in enumerate(c.pool.pages[s]):
        n = min(c.P, c.pool.lens[s] - j * c.P)
        c.cache[layer, p, :split].view(2, c.hkv, c.P, c.hd)[:, :, :n] = values[:, :, j * c.P:j * c.P + n]
        c.cache[layer, p, split:].view(2, c.hkv, c.P)[:, :, :n] = exponents[:, :, j * c.P:j * c.P + n]


@pytest.mark.parametrize("hq,hd", [(2, 64), (8, 128), (16, 128)])
@pytest.mark.parametrize("ends", [(67, 67), (67, 90), (100, 247), (67, 247), (240, 247), (120, 134)])
def test_values_of_all_powers(hq, hd, ends):
    """Tokens whose values' powers of two differ by up to 2^180: the small ones' weights may not be lost, the large ones' may not be infinite."""
    c = Held(hkv=2, hd=hd, P=16, n_pages=40, max_seqs=2)
    c.grow([0, 1], [300, 17])
    g = torch.Generator(device="cuda").manual_seed(3)
    for s, n in ((0, 300), (1, 17)):
        x = (torch.randn(2, 2, n, hd, generator=g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        e = torch.full((2, 2, n), 120, dtype=torch.uint8, device="cuda")
        e[1] = torch.randint(ends[0], ends[1] + 1, (2, n), generator=g, device="cuda").to(torch.uint8)
        _set(c, 0, s, x, e)
    _decode(c, hq)


def test_a_large_weight_of_small_values_beside_a_small_weight_of_large_ones():
    """The first token has nearly all of the weight and values of 2^-40, the others weights of e^-60 and values of about 2^20; and the other way
    round: what counts is the product."""
    c = Held(hkv=1, hd=64, P=16, n_pages=8, max_seqs=1)
    c.grow([0], [33])
    x = torch.ones(2, 1, 33, 64, device="cuda")
    x[0, 0, 1:] = 0.0
    x[1] = torch.randn(33, 64, device="cuda") * 100
    e = torch.full((2, 1, 33), 127, dtype=torch.uint8, device="cuda")
    for first, others in ((80, 140), (140, 80), (67, 150)):
        e[1, 0, 0], e[1, 0, 1:] = first, others
        _set(c, 0, 0, x.to(torch.float8_e4m3fn).view(torch.uint8), e)
        q = torch.full((1, 1, 64), 7.5, dtype=BF, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(1, 1, device="cuda")
        nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 1, 1), lse=lse)
        check_held_rows(out, lse, q, lambda i: c.tokens(0, 0), 0.125)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_peaked_scores(dtype):
    """Scores that differ by hundreds: one token takes nearly everything, and the maximum moves late."""
    c = Held(dtype=dtype, hkv=2, hd=128, P=32, n_pages=40, max_seqs=2)
    c.grow([0, 1], [600, 333])
    _decode(c, 8, spread=12.0)
    split = 2 * 2 * 32 * 128
    c.cache[0, :, split:split + 64] = torch.linspace(100, 123, 40, device="cuda").to(torch.uint8)[:, None]
    _decode(c, 8, spread=20.0)


@pytest.mark.parametrize("size,power", [(1e-30, 200), (1e30, 70), (1e-3, 130), (3e38, 67)])
def test_queries_over_bf16s_range(size, power):
    """Large queries on small keys and the other way round."""
    c = Held(hkv=1, hd=64, P=16, n_pages=8, max_seqs=2)
    c.grow([0, 1], [40, 100])
    g = torch.Generator(device="cuda").manual_seed(3)
    for s, n in ((0, 40), (1, 100)):
        x = (torch.randn(2, 1, n, 64, generator=g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        e = torch.full((2, 1, n), 120, dtype=torch.uint8, device="cuda")
        e[0] = power
        _set(c, 0, s, x, e)
    scale = 1.0 / (size * 100 * 2.0 ** (power - 127) * 8)
    q = (torch.randn(2, 4, 64, generator=g, device="cuda").clamp(-1, 1) * size).to(BF)
    out, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 4, 2), scale=scale, lse=lse)
    check_held_rows(out, lse, q, lambda i: c.tokens(0, i), float(np.float32(scale)))


def test_nan_shows_where_it_is_seen():
    c = Held(hkv=1, hd=64, P=16, n_pages=8, max_seqs=3)
    c.grow([0, 1, 2], [20, 20, 20])
    split = 2 * 16 * 64
    page = c.cache[0, c.pool.pages[0][1], :split].view(2, 16, 64)
    page[1, 3, 7] = 0x7f                                      # a value of the last token of sequence 0
    page = c.cache[0, c.pool.pages[1][0], :split].view(2, 16, 64)
    page[0, 2, 9] = 0xff                                      # a key of sequence 1
    page = c.cache[0, c.pool.pages[2][1], :split].view(2, 16, 64)
    page[:, 4:] = 0x7f                                        # behind sequence 2
    c.cache[0, c.pool.pages[2][1], split:].view(2, 16)[:, 4:] = 255
    q = torch.ones(3, 2, 64, dtype=BF, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(3, 2, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 2, 3), lse=lse)
    torch.cuda.synchronize()
    bad = torch.isnan(out)
    assert bad[0, :, 7].all() and bad[0].sum() == 2 and torch.isfinite(lse[0]).all()
    assert bad[1].all() and torch.isnan(lse[1]).all()
    assert not bad[2].any()
    check_held_rows(out[2:], lse[2:], q[2:], lambda i: c.tokens(0, 2), 0.125)


def test_queries_that_are_not_finite():
    """A NaN among a head's queries makes its row NaN, and no other."""
    c = Held(hkv=1, hd=128, P=16, n_pages=8, max_seqs=1)
    c.grow([0], [50])
    q = torch.randn(1, 8, 128, device="cuda").to(BF)
    q[0, 3, 77] = float("nan")
    q[0, 5] = 0
    out, lse = torch.empty_like(q), torch.empty(1, 8, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 8, 1), lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(out[0, 3]).all() and torch.isnan(lse[0, 3])
    keep = [0, 1, 2, 4, 5, 6, 7]
    check_held_rows(out[:, keep], lse[:, keep], q[:, keep], lambda i: tuple(x for x in c.tokens(0, 0)), 128 ** -0.5)


def test_pages_and_rows_that_are_not_there():
    c = Held(hkv=1, hd=64, P=16, n_pages=8, max_seqs=3, max_pages=4)
    c.grow([0, 1, 2], [40, 40, 10])
    k, v = c.tokens(0, 0)
    c.table[0, 1] = 8
    q = torch.randn(4, 1, 64, device="cuda").to(BF)
    out, lse = torch.empty_like(q), torch.empty(4, 1, device="cuda")
    c.lens[2] = 65
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 1, 4), seqs=c.dev([0, 1, 3, 2]), lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == A.S_PAGE | A.S_SEQ | A.S_LENGTH
    seen = np.r_[0:16, 32:40]
    none = np.zeros((0, 1, 64))
    check_held_rows(out, lse, q, lambda i: [(k[seen], v[seen]), c.tokens(0, 1), (none, none), (none, none)][i], 0.125)


def test_past_32_bit_offsets():
    n_pages = (1 << 32) // (2 * 8 * 256 * 129) + 12
    c = Held(hkv=8, hd=128, P=256, n_pages=n_pages, max_seqs=2)
    c.reserve([0], [256 * (n_pages - 5)])
    c.grow([1], [1000])
    nb.np_kv_free(c.desc, c.tables, c.dev([0]))
    c.pool.free([0])
    _decode(c, 16, seqs=[1, 0])


def test_one_workspace_for_caches_of_both_forms_and_replays():
    """Captured calls over one workspace, replayed in turn while the sequences grow."""
    c = Held(hkv=2, hd=64, P=16, n_pages=300, max_seqs=2)
    c.grow([0, 1], [1, 700])
    ws = _workspace(c, 40, 2)
    q, out, lse = torch.randn(2, 4, 64, device="cuda").to(BF), torch.empty(2, 4, 64, dtype=BF, device="cuda"), torch.empty(2, 4, device="cuda")
    s, graphs = torch.cuda.Stream(), []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, ws, lse=lse, stream=s)
        graphs.append(g)
    for t in range(6):
        c.grow([0, 1], [600 * (t % 2), 33], seed=t)
        torch.cuda.synchronize()
        out.fill_(float("nan"))
        graphs[t & 1].replay()
        torch.cuda.synchronize()
        check_held_rows(out, lse, q, lambda i: c.tokens(0, i), 0.125)
        _decode(c, 40, ws=ws)


def test_streams_of_their_own():
    c = Held(hkv=4, hd=64, P=16, n_pages=400, max_seqs=4)
    c.grow([0, 1, 2, 3], [1500, 900, 1, 2000])
    q = torch.randn(4, 8, 64, device="cuda").to(BF)
    want = torch.empty_like(q)
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, want, _workspace(c, 8, 4))
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    spaces = [_workspace(c, 8, 4) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, ws in zip(streams, spaces):
            with torch.cuda.stream(s):
                o = torch.empty_like(q)
                nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, o, ws, stream=s)
                outs.append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_held_decode_is_near_the_rows_it_stands_for(dtype):
    """What the 8 bits cost: the result over the rows themselves is as far as half a step of every key and value lets it be."""
    c = Held(dtype=dtype, hkv=2, hd=64, P=16, n_pages=20, max_seqs=1)
    start, _ = c.reserve([0], [200])
    k, v = c.append(0, [0], start, [200])
    q, out, _ = _decode(c, 4)
    kn, vn, qn, on = f64(k), f64(v), f64(q), f64(out)
    for h in range(4):
        want, _, mean, _ = A.attend(qn[0, h], kn[:, h // 2], vn[:, h // 2], 0.125)
        ds = 0.125 * 2.0 ** -4 * np.abs(kn[:, h // 2]) @ np.abs(qn[0, h])       # how far a score may move
        bound = mean * (2.0 ** -4 + np.expm1(2 * ds.max())) + 0.01 * np.abs(vn).max()
        assert (np.abs(on[0, h] - want) <= bound).all()


def test_logs_of_sums_without_scores():
    """Queries of 0: the log of the sum is that of the number of tokens, whatever the values' exponents.

    A weight is the square of a power of two that is off by 2^-22 at most, so it is off by 2^-21; up to four of them add up with 2^-22 more; the log of
    a number between a half and one is off by 2^-21.4 and the maximum's product, of numbers below 2, by 2^-23.  Together below 2^-20 + 2^-21."""
    lens = [1, 2, 3, 4, 1, 2]
    c = Held(dtype=BF, hkv=2, hd=64, P=16, n_pages=8, max_seqs=len(lens))
    for s, n in enumerate(lens):
        c.grow([s], [n], seed=s)
    c.cache[0, c.pool.pages[4][0], 2 * 2 * 16 * 64 + 2 * 16:] += 100     # values far larger, far smaller
    c.cache[0, c.pool.pages[5][0], 2 * 2 * 16 * 64 + 2 * 16:] -= 50
    q = torch.zeros(len(lens), 4, 64, dtype=BF, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(len(lens), 4, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 4, len(lens)), lse=lse)
    off = (lse.double().cpu() - torch.tensor(lens, dtype=torch.float64).log()[:, None]).abs().max().item()
    assert off < 2.0 ** -20 + 2.0 ** -21


def test_queries_at_the_end_of_their_range():
    """The largest queries against keys of the least exponent: the products are far from fp32's end, and the largest score takes all of the weight."""
    c = Held(dtype=BF, hkv=1, hd=64, P=16, n_pages=2, max_seqs=1)
    c.grow([0], [3], seed=4)
    k = torch.zeros(3, 1, 64, dtype=BF, device="cuda")
    k[:, 0, 0] = torch.tensor([224.0, 448.0, -448.0]) * 2.0 ** -60
    v = torch.randn(3, 1, 64, device="cuda").to(BF)
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k, v, c.dev([0]), cu=c.dev([0, 3]), start=c.dev([0]))
    q = torch.zeros(1, 2, 64, dtype=BF, device="cuda")
    q[0, 0, 0], q[0, 1, 0] = 1.5 * 2.0 ** 127, -1.5 * 2.0 ** 127
    out, lse = torch.empty_like(q), torch.empty(1, 2, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 2, 1), scale=1.0, lse=lse)
    want = c.tokens(0, 0)[1][[1, 2], 0]
    assert (np.abs(f64(out[0]) - want) <= np.abs(want) * 2.0 ** -8).all()
    # the scale times log2(e), the score, the maximum times ln 2: a rounding each, and twice that of the constants
    assert (lse.double() / (1.5 * 448 * 2.0 ** 67) - 1).abs().max() <= 6 * 2.0 ** -24
    assert c.status.item() == 0
