"""Values of V that are not finite, in tokens that are seen, through np_attn_decode: the result is what the weighted sum is, infinities
with their signs, as np_attn_prompt gives them."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, f64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")


def _call(c, hq, q, seqs=None):
    n = q.shape[0]
    out, lse = torch.empty_like(q), torch.empty(n, hq, device="cuda")
    ws = torch.zeros(nb.np_attn_workspace_bytes(c.desc, hq, n), dtype=torch.uint8, device="cuda")
    nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, out, ws, seqs=None if seqs is None else c.dev(seqs), lse=lse)
    torch.cuda.synchronize()
    assert not ws[-4 * n:].any()              # counts are zero again
    return f64(out), f64(lse)


def _put(c, s, token, head, d, x):
    c.cache[0, c.pool.pages[s][token // c.P], 1, head, token % c.P, d] = x


def _check(c, hq, q, out, lse, seqs=None):
    """Every element: not finite where the values that the row sees make it so, else within its bound."""
    qn, scale = f64(q), c.hd ** -0.5
    for i in range(len(qn)):
        k, v = c.tokens(0, i if seqs is None else seqs[i])
        for h in range(hq):
            kk, vv = k[:, h * c.hkv // hq], v[:, h * c.hkv // hq]
            with np.errstate(invalid="ignore"):
                want_odd = np.where(np.isfinite(vv), 0.0, vv).sum(0)        # weights are above 0: what is not finite stays that
            fine = np.nan_to_num(vv, nan=0.0, posinf=0.0, neginf=0.0)
            want, wl, mean, amp = A.attend(qn[i, h], kk, fine, scale)
            tol, tl = A.tolerances(want, wl, mean, amp, len(kk), c.hd, c.dtype == HF, False, np.abs(fine).max() if len(kk) else 0.0)
            odd = ~np.isfinite(want_odd)
            assert np.array_equal(out[i, h][odd], want_odd[odd], equal_nan=True), (i, h, out[i, h][odd], want_odd[odd])
            assert (np.abs(out[i, h][~odd] - want[~odd]) <= tol[~odd]).all(), (i, h)
            assert lse[i, h] == wl if len(kk) == 0 else abs(lse[i, h] - wl) <= tl


# heads of a group: one, eight (one form of the kernel), nine, sixteen, twenty-four (the other, with one block of heads and two)
LAYOUTS = [(1, 1, 64), (8, 1, 128), (8, 4, 64), (9, 1, 128), (32, 2, 64), (24, 1, 128)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,hd", LAYOUTS)
@pytest.mark.parametrize("spread", [1.0, 40.0])
def test_infinite_values_show_with_their_signs(dtype, hq, hkv, hd, spread):
    """Lengths of one to a few tiles, pieces whole and split.  `spread` 40: most weights underflow, the same infinities are there."""
    lens = [1, 1, 1, 2, 17, 64, 65, 130, 700, 0, 40]
    c = Cache(dtype=dtype, hkv=hkv, hd=hd, P=32, n_pages=60, max_seqs=len(lens))
    c.grow(list(range(len(lens))), lens)
    rng = np.random.default_rng(hq)
    for s, token, x in [(0, 0, INF), (1, 0, -INF), (2, 0, NAN), (3, 1, INF), (4, 0, -INF), (4, 16, INF), (5, 63, INF), (6, 64, -INF), (7, 31, INF),
                        (7, 32, NAN), (7, 129, -INF), (8, 0, INF), (8, 350, -INF), (8, 699, INF)]:
        _put(c, s, token, int(rng.integers(0, hkv)), int(rng.integers(0, hd)), x)
    # both signs in one place make a NaN
    _put(c, 10, 3, 0, 5, INF)
    _put(c, 10, 39, 0, 5, -INF)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = (torch.randn(len(lens), hq, hd, generator=g, device="cuda") * spread).to(dtype)
    _check(c, hq, q, *_call(c, hq, q))


@pytest.mark.parametrize("hq,hkv,hd", [(8, 1, 128), (4, 4, 64), (16, 1, 128), (12, 1, 64)])
def test_infinite_values_of_sequences_that_many_blocks_share(hq, hkv, hd):
    """Long sequences, whose partial results are joined in one step and in two; the first token, the last, one that a row takes nearly
    all of its result from, and one whose weight underflows."""
    lens = [20000, 3, 9000]
    c = Cache(hkv=hkv, hd=hd, P=64, n_pages=460, max_seqs=3)
    c.grow([0, 1, 2], lens)
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(3, hq, hd, generator=g, device="cuda").to(BF)
    k, _ = c.tokens(0, 0)
    score = k[:, 0] @ f64(q)[0, 0]
    for token, d, x in [(0, 1, INF), (19999, 2, -INF), (int(score.argmax()), 3, INF), (int(score.argmin()), 4, -INF), (10000, 5, NAN)]:
        _put(c, 0, token, 0, d, x)
    _put(c, 2, 4000, hkv - 1, 7, INF)
    _put(c, 2, 8999, hkv - 1, 7, -INF)
    _check(c, hq, q, *_call(c, hq, q))
    q *= 50                                                             # all but a few weights underflow
    _check(c, hq, q, *_call(c, hq, q))


@pytest.mark.parametrize("hq", [6, 15])
def test_infinite_values_beside_rows_that_are_no_number_or_empty(hq):
    """A head whose scores are NaN stays NaN, one whose scores all are -inf stays zero; values of pages that are not there have no say."""
    c = Cache(hkv=1, hd=64, P=16, n_pages=12, max_seqs=3)
    c.grow([0, 1, 2], [40, 40, 40])
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(3, hq, 64, generator=g, device="cuda").to(BF)
    for s in range(3):
        _put(c, s, 20, 0, 9, INF)
    q[0, 1, 0] = NAN
    c.cache[0, c.pool.pages[1], 0, 0, :, :] = -INF                      # sequence 1: every score -inf for queries above 0
    q[1] = q[1].abs() + 0.1
    c.table[2, 1] = -1                                                  # tokens 16 to 31 of sequence 2
    out, lse = _call(c, hq, q)
    assert np.isnan(out[0, 1]).all() and np.isnan(lse[0, 1])
    others = [h for h in range(hq) if h != 1]
    assert (out[0, others, 9] == np.inf).all() and np.isfinite(np.delete(out[0, others], 9, axis=1)).all()
    assert (out[1] == 0).all() and (lse[1] == -np.inf).all()
    assert np.isfinite(out[2]).all() and np.isfinite(lse[2]).all()


def test_infinite_values_from_a_graph_and_into_strided_rows():
    """Replayed on contents that change, results in the middle of wider rows; what lies beside them stays."""
    c = Cache(hkv=2, hd=64, P=16, n_pages=200, max_seqs=2)
    c.grow([0, 1], [1500, 30])
    q = torch.randn(2, 4, 64, device="cuda").to(BF)
    room = torch.full((2, 6, 64), 7.0, dtype=BF, device="cuda")
    ws = torch.zeros(nb.np_attn_workspace_bytes(c.desc, 4, 2), dtype=torch.uint8, device="cuda")
    lse = torch.empty(2, 4, device="cuda")
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        nb.np_attn_decode(c.desc, c.cache, 0, c.tables, q, room[:, 1:5], ws, lse=lse, stream=s)
    for x in (INF, 0.25, -INF, NAN):
        _put(c, 0, 700, 1, 33, x)
        _put(c, 1, 29, 0, 0, x)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        _check(c, 4, q, f64(room[:, 1:5]), f64(lse))
        assert (room[:, 0] == 7).all() and (room[:, 5] == 7).all() and not ws[-8:].any()
