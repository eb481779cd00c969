"""Attention over the paged cache and over packed prompts against the 64-bit oracle, every element within its own bound."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, check_rows, f64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _workspace(c, hq, n):
    return torch.zeros(nb.np_attn_workspace_bytes(c.desc, hq, n), dtype=torch.uint8, device="cuda")


def _decode(c, hq, seqs=None, layer=0, seed=0, scale=None, ws=None, spread=1.0):
    """One call on random queries that are slices of a wider tensor; checked against the oracle."""
    n = len(seqs) if seqs is not None else c.desc.max_seqs
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = (torch.randn(n, hq + 3, c.hd, generator=g, device="cuda") * spread).to(c.dtype)
    q = wide[:, 1:hq + 1]
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

    check_rows(out, lse[:n], q, sees, scale, False)
    return q, out, lse[:n]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd,P", [(1, 1, 64, 16), (4, 4, 128, 64), (8, 1, 128, 32), (14, 2, 64, 256), (16, 1, 128, 16), (40, 8, 128, 128), (34, 2, 64, 64),
                                         (96, 2, 128, 16)])
def test_decode(dtype, hq, hkv, hd, P):
    """Lengths around tiles and pages; none at all; groups of one to forty-eight heads."""
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 130, 257, 700]
    c = Cache(dtype=dtype, layers=2, hkv=hkv, hd=hd, P=P, n_pages=2 + sum(-(-x // P) for x in lens), max_seqs=len(lens))
    order = np.random.default_rng(1).permutation(len(lens)).tolist()
    for s in order:                           # pages of the sequences are mixed
        c.grow([s], [lens[s] // 2], seed=s)
    for s in order[::-1]:
        c.grow([s], [lens[s] - lens[s] // 2], seed=100 + s)
    c.check()
    _decode(c, hq, layer=1)
    _decode(c, hq, layer=0, seqs=[11, 3, -1, 0, 11, 1, -5], seed=2)      # any order, twice the same, padding
    c.check()


@pytest.mark.parametrize("lens,hq,hkv,hd", [([20000], 8, 1, 128), ([20000, 3, 0, 9000], 4, 2, 64), ([1] * 300, 2, 2, 64), ([5000] + [40] * 63, 16, 16, 64), ([900] * 148, 4, 4, 64)])
def test_decode_splits_of_all_sizes(lens, hq, hkv, hd):
    """One long sequence over all blocks, long ones among short ones, more rows than blocks; twice into the same workspace gives the
    same bits."""
    P = 64
    c = Cache(hkv=hkv, hd=hd, P=P, n_pages=sum(-(-x // P) for x in lens), max_seqs=len(lens))
    c.grow(list(range(len(lens))), lens)
    ws = _workspace(c, hq, len(lens))
    _, a, la = _decode(c, hq, ws=ws)
    _, b, lb = _decode(c, hq, ws=ws)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_one_workspace_serves_calls_of_different_sizes():
    c = Cache(hkv=2, hd=64, P=16, n_pages=600, max_seqs=6)
    c.grow(list(range(6)), [3000, 10, 900, 2000, 0, 77])
    d = Cache(dtype=HF, hkv=1, hd=128, P=64, n_pages=40, max_seqs=3)
    d.grow([0, 1, 2], [1700, 5, 300])
    ws = torch.zeros(max(nb.np_attn_workspace_bytes(c.desc, 40, 6), nb.np_attn_workspace_bytes(d.desc, 12, 3)), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        _decode(c, 40, ws=ws)
        _decode(c, 4, seqs=[3], ws=ws)
        _decode(d, 12, ws=ws)
        _decode(c, 2, seqs=[2, 0], ws=ws)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_decode_of_peaked_scores(dtype):
    """Scores that differ by hundreds: one token takes nearly everything, and the maximum moves late."""
    c = Cache(dtype=dtype, hkv=2, hd=128, P=32, n_pages=40, max_seqs=2)
    c.grow([0, 1], [600, 333])
    _decode(c, 8, spread=12.0)
    c.cache[:, :, 0] *= torch.linspace(0.0, 1.0, 40, device="cuda").to(dtype)[:, None, None, None]
    _decode(c, 8, spread=20.0)


def test_decode_of_infinite_and_missing_values():
    """-inf scores leave a row empty; a NaN or an infinity that is seen shows, one that is not seen does not."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=8, max_seqs=3)
    c.grow([0, 1, 2], [20, 20, 20])
    q = torch.ones(3, 2, 64, dtype=BF, device="cuda")
    c.cache[0, c.pool.pages[0], 0] = -float("inf")                       # every key of sequence 0: scores of -inf
    c.cache[0, c.pool.pages[1][1], 1, 0, 3] = float("nan")               # the last token's value of sequence 1
    c.cache[0, c.pool.pages[2][1], :, 0, 4:] = float("inf")              # behind sequence 2
    out, lse = torch.empty_like(q), torch.empty(3, 2, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 2, 3), lse=lse)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and (lse[0] == -float("inf")).all()
    assert torch.isnan(out[1]).all() and torch.isfinite(lse[1]).all()
    assert torch.isfinite(out[2]).all() and torch.isfinite(lse[2]).all()


def test_decode_leaves_out_pages_and_rows_that_are_not_there():
    """A page number outside the pool: its tokens are not seen.  A sequence outside the tables or a length outside its row: an empty row."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=8, max_seqs=3, max_pages=4)
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
    check_rows(out, lse, q, lambda i: [(k[seen], v[seen]), c.tokens(0, 1), (none, none), (none, none)][i], 0.125, False)


def test_decode_past_32_bit_offsets():
    """A cache of more than 4 GB, with the sequence's pages at its end."""
    n_pages = (1 << 32) // (2 * 2 * 8 * 256 * 128) + 12
    c = Cache(hkv=8, hd=128, P=256, n_pages=n_pages, max_seqs=2, fill=0.0)
    c.reserve([0], [256 * (n_pages - 5)])
    c.grow([1], [1000])
    nb.np_kv_free(c.desc, c.tables, c.dev([0]))
    c.pool.free([0])
    _decode(c, 16, seqs=[1, 0])
    c.check()


def test_decode_on_streams_of_their_own():
    """Two calls at once, each with its workspace, on streams that wait for nothing but their own inputs."""
    c = Cache(hkv=4, hd=64, P=16, n_pages=400, max_seqs=4)
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


def test_decode_replays_from_graphs_that_share_a_workspace():
    """Two captured calls over one workspace, replayed in turn while the sequences grow."""
    c = Cache(hkv=2, hd=64, P=16, n_pages=300, max_seqs=2)
    c.grow([0, 1], [1, 700])
    ws = _workspace(c, 4, 2)
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
        check_rows(out, lse, q, lambda i: c.tokens(0, i), 0.125, False)


def _prompt(dtype, lens, hq, hkv, hd, pad=0, front=0, seed=0, scale=None, spread=1.0, change=None, only=None):
    """One call on slices of one projection's output whose rows outside the prompts are NaN; checked row by row (`only`: some rows)."""
    rows = front + sum(lens) + pad
    cu = np.concatenate([[0], np.cumsum(lens)]) + front
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(rows, hq + 2 * hkv, hd, generator=g, device="cuda")
    qkv[:, :hq] *= spread
    qkv = qkv.to(dtype)
    qkv[:front] = float("nan")
    qkv[cu[-1]:] = float("nan")
    if change is not None:
        change(qkv)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    out, lse = torch.full((rows, hq, hd), 7.0, dtype=dtype, device="cuda"), torch.full((rows, hq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = hd ** -0.5 if scale is None else scale
    nb.np_attn_prompt(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), out, status, scale=scale, lse=lse)
    assert nb.np_attn_check(status) == nb.NP_OK
    assert (out[:front] == 7).all() and (out[cu[-1]:] == 7).all() and (lse[:front] == 7).all() and (lse[cu[-1]:] == 7).all()
    kn, vn = f64(k), f64(v)
    want = [r for r in range(front, cu[-1]) if only is None or r - front in only]
    first = {r: cu[np.searchsorted(cu, r, side="right") - 1] for r in want}
    at = torch.tensor(want, dtype=torch.long, device="cuda")
    check_rows(out[at], lse[at], q[at], lambda i: (kn[first[want[i]]:want[i] + 1], vn[first[want[i]]:want[i] + 1]), scale, True)
    return out, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd", [(1, 1, 64), (2, 2, 128), (8, 1, 128), (5, 1, 64), (14, 2, 128), (64, 1, 64), (128, 1, 128), (65, 1, 128)])
def test_prompt_head_layouts(dtype, hq, hkv, hd):
    """Groups that divide a tile's rows and groups that do not; prompts of no token, one token and odd lengths."""
    _prompt(dtype, [0, 1, 77, 0, 140, 2], hq, hkv, hd, pad=3, front=2)


@pytest.mark.parametrize("n", [1, 2, 31, 127, 128, 129, 255, 256, 257, 383, 385, 511, 513])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 128), (4, 1, 64)])
def test_prompt_lengths_around_tiles(n, hq, hkv, hd):
    _prompt(BF, [n], hq, hkv, hd, pad=1, seed=n)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [(BF, 2, 1, 128), (HF, 1, 1, 64), (BF, 3, 1, 128)])
def test_prompt_of_many_tiles(dtype, hq, hkv, hd):
    n = 2600
    rng = np.random.default_rng(0)
    only = set(rng.integers(0, n, 250).tolist()) | set(range(40)) | set(range(n - 40, n)) | set(range(1015, 1035))
    _prompt(dtype, [n], hq, hkv, hd, only=only)


def test_prompt_many_prompts():
    rng = np.random.default_rng(5)
    _prompt(BF, rng.integers(0, 9, 700).tolist(), 2, 1, 64, pad=5)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_prompt_of_peaked_scores(dtype):
    """Maxima that grow by hundreds from tile to tile: the accumulators are rescaled; and scores that shrink again."""
    def ramp(qkv):
        n = len(qkv)
        qkv[:, 2:3] *= torch.cat([torch.linspace(0, 1, n // 2, device="cuda"), torch.linspace(1, 0, n - n // 2, device="cuda")])[:, None, None].to(dtype)
    _prompt(dtype, [700], 2, 1, 128, spread=20.0, change=ramp, seed=3)


def test_prompt_later_tokens_do_not_reach_earlier_rows():
    """Infinities and NaN in keys and values show in the rows that see them, and in no other."""
    hq = 2
    bad = [(100, 2, float("nan")), (120, 3, float("inf")), (340, 3, float("nan")), (345, 2, -float("inf"))]    # (row, key or value head, what)
    g = torch.Generator(device="cuda").manual_seed(0)
    qkv = torch.randn(350, hq + 2, 128, generator=g, device="cuda").to(BF)
    for r, h, x in bad:
        qkv[r, h] = x
    out, l2 = torch.empty(350, hq, 128, dtype=BF, device="cuda"), torch.empty(350, hq, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(qkv[:, :2], qkv[:, 2:3], qkv[:, 3:], torch.tensor([0, 150, 350], dtype=torch.int32, device="cuda"), out, status, lse=l2)
    assert nb.np_attn_check(status) == nb.NP_OK
    fine = list(range(100)) + list(range(150, 340))
    at = torch.tensor(fine, device="cuda")
    kn, vn = f64(qkv[:, 2:3]), f64(qkv[:, 3:])
    check_rows(out[at], l2[at], qkv[at, :2], lambda i: (kn[(0 if fine[i] < 150 else 150):fine[i] + 1], vn[(0 if fine[i] < 150 else 150):fine[i] + 1]),
               128 ** -0.5, True)
    assert torch.isnan(out[100:150].float()).all() and torch.isnan(out[340:].float()).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd", [(1, 1, 64), (4, 2, 128), (5, 1, 128), (8, 1, 64)])
def test_prompt_infinite_values_reach_the_rows_that_see_them(dtype, hq, hkv, hd):
    """Values that are not finite, in single places of tokens of every part of a prompt: each row's result is what the weighted sum
    over the tokens that it sees is, infinities with their signs, and finite everywhere else."""
    lens = [400, 3, 150]
    rows, cu = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    g = torch.Generator(device="cuda").manual_seed(hq)
    qkv = torch.randn(rows, hq + 2 * hkv, hd, generator=g, device="cuda").to(dtype)
    rng = np.random.default_rng(hd)
    places = [(t, int(rng.integers(0, hkv)), int(rng.integers(0, hd)), x) for t, x in zip(
        [0, 30, 127, 128, 129, 255, 256, 300, 399, 401, 403, 540, 552], [np.inf, -np.inf, np.nan, np.inf, np.inf, -np.inf, np.inf, np.nan, np.inf, np.inf,
                                                                         -np.inf, np.nan, np.inf])]
    for t, h, d, x in places:
        qkv[t, hq + hkv + h, d] = x
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    out, lse = torch.empty(rows, hq, hd, dtype=dtype, device="cuda"), torch.empty(rows, hq, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), out, status, lse=lse)
    assert nb.np_attn_check(status) == nb.NP_OK
    on, kn, vn, qn, scale = f64(out), f64(k), f64(v), f64(q), hd ** -0.5
    fine = np.nan_to_num(vn, nan=0.0, posinf=0.0, neginf=0.0)
    for r in range(rows):
        a = cu[np.searchsorted(cu, r, side="right") - 1]
        for h in range(hq):
            c = h // (hq // hkv)
            seen = vn[a:r + 1, c]
            add = np.where(np.isfinite(seen), 0.0, seen)
            with np.errstate(invalid="ignore"):
                want_odd = add.sum(0)                      # weights are above 0: what is not finite stays that, signs and all
            want, wl, mean, amp = A.attend(qn[r, h], kn[a:r + 1, c], fine[a:r + 1, c], scale)
            tol, _ = A.tolerances(want, wl, mean, amp, r + 1 - a, hd, dtype == HF, True, np.abs(fine).max())
            odd = ~np.isfinite(want_odd)
            assert np.array_equal(on[r, h][odd], want_odd[odd], equal_nan=True), (r, h)
            assert (np.abs(on[r, h][~odd] - want[~odd]) <= tol[~odd]).all(), (r, h)


def test_prompt_of_nothing_but_nan_values_ends_like_any_other():
    n, hq = 6000, 4
    qkv = torch.randn(n, hq + 2, 128, device="cuda").to(BF)
    qkv[:, hq + 1] = float("nan")
    out, status = torch.zeros(n, hq, 128, dtype=BF, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(qkv[:, :hq], qkv[:, hq:hq + 1], qkv[:, hq + 1:], torch.tensor([0, n], dtype=torch.int32, device="cuda"), out, status)
    assert nb.np_attn_check(status) == nb.NP_OK and torch.isnan(out).all()
    qkv[:] = float("nan")
    out.zero_()
    nb.np_attn_prompt(qkv[:, :hq], qkv[:, hq:hq + 1], qkv[:, hq + 1:], torch.tensor([0, n], dtype=torch.int32, device="cuda"), out, status)
    assert nb.np_attn_check(status) == nb.NP_OK and torch.isnan(out).all()


def test_prompt_rows_with_nothing_but_minus_infinity():
    """Keys of -inf make every score -inf as long as they are all there is: zeros, as for an empty sequence."""
    rows = 140
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn(rows, 3, 64, generator=g, device="cuda").to(BF)
    qkv[:, :1] = qkv[:, :1].abs() + 0.1
    qkv[:5, 1:2] = -float("inf")
    out, lse = torch.empty(rows, 1, 64, dtype=BF, device="cuda"), torch.empty(rows, 1, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], torch.tensor([0, rows], dtype=torch.int32, device="cuda"), out, status, lse=lse)
    assert nb.np_attn_check(status) == nb.NP_OK
    assert (out[:5] == 0).all() and (lse[:5] == -float("inf")).all()
    qkv[3, 2] = float("nan")                   # seen with a weight that is no number: zeros as long as there is no other
    nb.np_attn_prompt(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], torch.tensor([0, 5], dtype=torch.int32, device="cuda"), out, status, lse=lse)
    assert nb.np_attn_check(status) == nb.NP_OK and (out[:5] == 0).all()
    qkv[3, 2] = 0.5
    nb.np_attn_prompt(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], torch.tensor([0, rows], dtype=torch.int32, device="cuda"), out, status, lse=lse)
    torch.cuda.synchronize()
    kn, vn = f64(qkv[:, 1:2]), f64(qkv[:, 2:])
    check_rows(out[5:], lse[5:], qkv[5:, :1], lambda i: (kn[5:i + 6], vn[5:i + 6]), 0.125, True)


def test_prompt_orders_of_strides():
    """Heads outermost, rows with gaps, one token, one head."""
    for shape in [(90, 4, 2), (1, 4, 2), (90, 1, 1)]:
        n, hq, hkv = shape
        q = torch.randn(hq, n, 64, device="cuda").to(BF).transpose(0, 1)
        k = torch.randn(n, 3, hkv, 64, device="cuda").to(BF)[:, 1]
        v = torch.randn(hkv, n + 5, 64, device="cuda").to(BF)[:, 2:n + 2].transpose(0, 1)
        out, lse = torch.empty(hq, n, 64, dtype=BF, device="cuda").transpose(0, 1), torch.empty(n, hq, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        nb.np_attn_prompt(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), out, status, lse=lse)
        assert nb.np_attn_check(status) == nb.NP_OK
        kn, vn = f64(k), f64(v)
        check_rows(out, lse, q, lambda i: (kn[:i + 1], vn[:i + 1]), 0.125, True)
    with pytest.raises(nb.NpError):
        nb.np_attn_prompt(q, torch.randn(90, 1, 128, device="cuda").to(BF)[:, :, ::2], v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), out, status)


def test_prompt_bounds_that_make_no_sense_touch_nothing_else():
    """cu that runs past the rows or backwards: such a prompt is cut or empty, no row outside the buffers is touched."""
    n = 60
    qkv = torch.randn(n, 3, 64, device="cuda").to(BF)
    out = torch.full((n, 1, 64), 7.0, dtype=BF, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.np_attn_prompt(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], torch.tensor([0, 20, 10, 99], dtype=torch.int32, device="cuda"), out, status)
    assert nb.np_attn_check(status) == nb.NP_OK
    assert torch.isfinite(out.float()).all()
    nb.np_attn_prompt(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], torch.tensor([-7, -3], dtype=torch.int32, device="cuda"), out.fill_(7.0), status)
    torch.cuda.synchronize()
    assert (out == 7).all()


def test_prompt_replays_on_new_prompts():
    n, hq, hkv, hd = 300, 4, 2, 128
    qkv = torch.randn(n, hq + 2 * hkv, hd, device="cuda").to(HF)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    out, lse = torch.empty(n, hq, hd, dtype=HF, device="cuda"), torch.empty(n, hq, device="cuda")
    status, cu = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        nb.np_attn_prompt(q, k, v, cu, out, status, lse=lse, stream=s)
    for bounds in ([0, 100, 300], [0, 0, 300], [0, 299, 300]):
        cu.copy_(torch.tensor(bounds))
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert nb.np_attn_check(status) == nb.NP_OK
        kn, vn = f64(k), f64(v)
        check_rows(out, lse, q, lambda i: (kn[(bounds[1] if i >= bounds[1] else 0):i + 1], vn[(bounds[1] if i >= bounds[1] else 0):i + 1]), hd ** -0.5, True)


def test_a_run_of_them_together():
    """Two prompts are read and kept, one is forked, both branches decode beside the other prompt, the pool is closed up between
    steps; every step's attention is the oracle's over the tokens that the host has kept."""
    hq, hkv, hd, P = 8, 2, 64, 16
    c = Cache(hkv=hkv, hd=hd, P=P, n_pages=60, max_seqs=5, dtype=BF)
    lens = [37, 100]
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn(sum(lens), hq + 2 * hkv, hd, generator=g, device="cuda").to(BF)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    cu = c.dev([0, 37, 137])
    out, lse = torch.empty(137, hq, hd, dtype=BF, device="cuda"), torch.empty(137, hq, device="cuda")
    start, _ = c.reserve([3, 0], lens)
    nb.np_kv_append(c.desc, c.cache, 0, c.tables, k, v, c.dev([3, 0]), cu, start)
    nb.np_attn_prompt(q, k, v, cu, out, c.status, lse=lse)
    hist = {3: [(f64(k[:37]), f64(v[:37]))], 0: [(f64(k[37:]), f64(v[37:]))]}

    def kept(s):
        return tuple(np.concatenate([x[i] for x in hist[s]]) for i in (0, 1))

    kn, vn = f64(k), f64(v)
    check_rows(out, lse, q, lambda i: (kn[(37 if i >= 37 else 0):i + 1], vn[(37 if i >= 37 else 0):i + 1]), 0.125, True)
    # the last row of a prompt is what a decode call for it gives
    o1, l1 = torch.empty(1, hq, hd, dtype=BF, device="cuda"), torch.empty(1, hq, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q[36:37], o1, _workspace(c, hq, 1), seqs=c.dev([3]), lse=l1)
    torch.cuda.synchronize()
    check_rows(o1, l1, q[36:37], lambda i: kept(3), 0.125, False)
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev([3]), c.dev([1]))
    c.pool.fork([3], [1])
    hist[1] = list(hist[3])
    seqs, ws = [0, 1, 3], _workspace(c, hq, 3)
    for t in range(20):
        step = torch.randn(3, hq + 2 * hkv, hd, generator=g, device="cuda").to(BF)
        start, _ = c.reserve(seqs, [1, 1, 1])
        nb.np_kv_append(c.desc, c.cache, 0, c.tables, step[:, hq:hq + hkv], step[:, hq + hkv:], c.dev(seqs), None, start)
        for i, s in enumerate(seqs):
            hist[s].append((f64(step[i:i + 1, hq:hq + hkv]), f64(step[i:i + 1, hq + hkv:])))
        o, l = torch.empty(3, hq, hd, dtype=BF, device="cuda"), torch.empty(3, hq, device="cuda")
        nb.np_attn_decode(c.desc, c.cache, 0, c.tables, step[:, :hq], o, ws, seqs=c.dev(seqs), lse=l)
        c.check()
        check_rows(o, l, step[:, :hq], lambda i: kept(seqs[i]), 0.125, False)
        if t == 8:
            nb.np_kv_free(c.desc, c.tables, c.dev([0]))
            c.pool.free([0])
            nb.np_kv_compact(c.desc, c.cache, c.tables, c.tables)
            c.pool.compact()
            hist[0] = []
    assert nb.np_attn_check(c.status) == nb.NP_OK


def test_prompts_on_streams_of_their_own():
    """Long and short prompts at once, eager and replayed, one and two tiles to a block: each call as if it were alone."""
    jobs = []
    for seed, (lens, hq, hkv, hd) in enumerate([([700, 3, 0, 900], 8, 2, 128), ([64] * 30, 4, 4, 64), ([1], 2, 1, 128)]):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows = sum(lens)
        q, k, v = (torch.randn(rows, h, hd, generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv))
        cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        status, want = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty_like(q)
        nb.np_attn_prompt(q, k, v, cu, want, status)
        jobs.append((q, k, v, cu, status, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs, graphs = [], []
    for q, k, v, cu, status, want, s in jobs:
        held, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            nb.np_attn_prompt(q, k, v, cu, held, status, stream=s)
        graphs.append((graph, s, held, want))
    for _ in range(20):
        for (q, k, v, cu, status, want, s), (graph, *_r) in zip(jobs, graphs):
            with torch.cuda.stream(s):
                o = torch.empty_like(q)
                nb.np_attn_prompt(q, k, v, cu, o, status, stream=s)
                outs.append((o, want))
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o, want in outs) and all(torch.equal(h, want) for _, _, h, want in graphs)
    assert all(job[4].item() == 0 for job in jobs)


def test_decode_of_the_most_rows():
    """1024 rows of a call, most of them the same sequences again or padding; the largest table."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=600, max_seqs=1024, max_pages=40)
    seqs = list(range(0, 1024, 7))
    c.grow(seqs, [1 + (5 * s) % 43 for s in seqs])
    rows = [[seqs[i % len(seqs)], -1, 1][0 if i % 3 == 0 else i % 3] for i in range(1024)]
    _decode(c, 4, seqs=rows)
    c.check()


# ---- groups of more than eight heads: keys and values come another way --------------------------------------------------
@pytest.mark.parametrize("lens,hq,hkv,hd", [([20000], 16, 1, 128), ([20000, 3, 0, 9000], 24, 2, 64), ([1] * 300, 18, 2, 64), ([5000] + [40] * 63, 64, 4, 128),
                                            ([31, 16, 17, 15, 33], 12, 1, 128)])
def test_decode_of_large_groups_splits_of_all_sizes(lens, hq, hkv, hd):
    """Chunks that end inside a page and at its end, few and many pieces; twice into the same workspace gives the same bits."""
    P = 32
    c = Cache(hkv=hkv, hd=hd, P=P, n_pages=sum(-(-x // P) for x in lens), max_seqs=len(lens))
    c.grow(list(range(len(lens))), lens)
    ws = _workspace(c, hq, len(lens))
    _, a, la = _decode(c, hq, ws=ws)
    _, b, lb = _decode(c, hq, ws=ws)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_decode_of_large_groups_infinite_and_missing_values():
    """As for small groups: -inf scores leave a row empty, what is seen shows, what is not seen does not."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=8, max_seqs=3)
    c.grow([0, 1, 2], [20, 20, 20])
    q = torch.ones(3, 11, 64, dtype=BF, device="cuda")
    c.cache[0, c.pool.pages[0], 0] = -float("inf")
    c.cache[0, c.pool.pages[1][1], 1, 0, 3] = float("nan")
    c.cache[0, c.pool.pages[2][1], :, 0, 4:] = float("inf")
    out, lse = torch.empty_like(q), torch.empty(3, 11, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 11, 3), lse=lse)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and (lse[0] == -float("inf")).all()
    assert torch.isnan(out[1]).all() and torch.isfinite(lse[1]).all()
    assert torch.isfinite(out[2]).all() and torch.isfinite(lse[2]).all()


def test_decode_of_large_groups_leaves_out_pages_and_rows_that_are_not_there():
    c = Cache(hkv=1, hd=128, P=16, n_pages=40, max_seqs=3, max_pages=30)
    c.grow([0, 1, 2], [300, 40, 10])
    k, v = c.tokens(0, 0)
    for page in (0, 5, 6, 7, 18):
        c.table[0, page] = -1 if page & 1 else 40
    q = torch.randn(4, 16, 128, device="cuda").to(BF)
    out, lse = torch.empty_like(q), torch.empty(4, 16, device="cuda")
    c.lens[2] = 16 * 30 + 1
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, _workspace(c, 16, 4), seqs=c.dev([0, 1, 3, 2]), lse=lse)
    torch.cuda.synchronize()
    assert c.status.item() == A.S_PAGE | A.S_SEQ | A.S_LENGTH
    seen = np.r_[16:80, 128:288]
    none = np.zeros((0, 1, 128))
    check_rows(out, lse, q, lambda i: [(k[seen], v[seen]), c.tokens(0, 1), (none, none), (none, none)][i], 128 ** -0.5, False)


def test_decode_of_large_groups_past_32_bit_offsets():
    n_pages = (1 << 32) // (2 * 2 * 8 * 256 * 128) + 12
    c = Cache(hkv=8, hd=128, P=256, n_pages=n_pages, max_seqs=2, fill=0.0)
    c.reserve([0], [256 * (n_pages - 5)])
    c.grow([1], [1000])
    nb.np_kv_free(c.desc, c.tables, c.dev([0]))
    c.pool.free([0])
    _decode(c, 80, seqs=[1, 0])
    c.check()


def test_decode_of_large_groups_at_once_and_replayed():
    """Calls of two streams at once, each with its workspace, eager and from a graph, beside calls of small groups."""
    c = Cache(hkv=2, hd=128, P=16, n_pages=400, max_seqs=4)
    c.grow([0, 1, 2, 3], [1500, 900, 1, 2000])
    jobs = []
    for hq in (32, 26, 8):
        q = torch.randn(4, hq, 128, device="cuda").to(BF)
        want, out, s, ws = torch.empty_like(q), torch.empty_like(q), torch.cuda.Stream(), _workspace(c, hq, 4)
        nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, want, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, ws, stream=s)
        jobs.append((q, want, out, s, ws, g))
    eager = []
    for _ in range(15):
        for q, want, out, s, ws, g in jobs:
            with torch.cuda.stream(s):
                o = torch.empty_like(q)
                nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, o, ws, stream=s)
                eager.append((o, want))
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o, want in eager) and all(torch.equal(j[2], j[1]) for j in jobs)
    assert nb.np_attn_check(c.status) == nb.NP_OK
