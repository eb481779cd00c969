"""Shared set-up of the tests of rows on their way and of caches held in 8 bits."""
import numpy as np
import torch

from oracle import attn_oracle as A
from oracle import rows_oracle as R
from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild
from tests.attn_harness import Cache, f64

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}     # half a step below the normal numbers


class Held(Cache):
    """A cache of 8 bits and the oracle's pool.  It starts as NaN with exponents of 2^0: what must not be read shows."""

    def __init__(self, dtype=torch.bfloat16, layers=1, hkv=2, hd=64, P=16, n_pages=32, max_seqs=8, max_pages=None, fill=0x7f):
        nbuild.build()
        self.dtype, self.hkv, self.hd, self.P = dtype, hkv, hd, P
        max_pages = n_pages if max_pages is None else max_pages
        self.desc = nb.make_kv_desc(dtype, layers, hkv, hd, P, n_pages, max_seqs, max_pages, e4m3=True)
        self.page = nb.np_kv_sizes(self.desc).page_bytes
        assert self.page == 2 * hkv * P * (hd + 1)
        self.cache = torch.full((layers, n_pages, self.page), fill, dtype=torch.uint8, device="cuda")
        ints = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.lens, self.refs, self.status = ints(max_seqs, max_pages), ints(max_seqs), ints(n_pages), ints(1)
        self.scratch = ints(nb.np_kv_sizes(self.desc).scratch_bytes // 4)
        self.tables = nb.make_kv_tables(self.table, self.lens, self.refs, self.scratch, self.status)
        self.pool = A.Pool(P, n_pages, max_seqs, max_pages)
        nb.np_kv_reset(self.desc, self.tables)

    def parts(self, layer, pages):
        """Bytes of some pages: values [pages][2][hkv][P][hd], exponents [pages][2][hkv][P]."""
        b = self.cache[layer, torch.as_tensor(pages, dtype=torch.long, device="cuda")].cpu().numpy()
        split = 2 * self.hkv * self.P * self.hd
        shape = (len(pages), 2, self.hkv, self.P)
        return b[:, :split].reshape(*shape, self.hd), b[:, split:].reshape(shape)

    def tokens(self, layer, s):
        n, pages = self.pool.lens[s], self.pool.pages[s]
        values, e = self.parts(layer, pages)
        got = R.e4m3_values()[values] * 2.0 ** (e.astype(np.float64) - 127)[..., None]
        got = got.transpose(1, 0, 3, 2, 4).reshape(2, -1, self.hkv, self.hd)[:, :n]
        return got[0], got[1]


def frequencies(rot, base=10000.0):
    return base ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") / max(1, rot // 2))


def check_rotated(out, x, gain, eps, pos, freq, neighbours):
    """Rows [tokens][heads][head_dim], every element within its bound.

    The norm's factor: a sum of head_dim squares in fp32, a root and two products, off by at most (head_dim / 2 + 8) 2^-24 + 2^-21 of itself.
    A rotated value is two products and a sum of values of size |a| + |b| at most: cosine and sine are off by at most 2^-21 (their own
    rounding and the fraction of a turn, 2^-26 of one, in fp32) and by what the fp64 product leaves of the angle, 4 * 2^-53 of it.  Then the
    result's rounding, half a step of its type."""
    xn, on, fr = f64(x), f64(out), f64(freq)
    g = None if gain is None else f64(gain)
    half, tiny = HALF[x.dtype], TINY[x.dtype]
    n, hd = len(fr), x.shape[-1]
    for t, p in enumerate(pos):
        want = R.rotate(xn[t], g, eps, p, fr, neighbours)
        y = np.abs(R.rotate(xn[t], g, eps, 0, np.zeros(0), neighbours))
        size, angle = y.copy(), np.zeros(hd)
        turn = np.abs(float(p) * fr) * 4 * 2.0 ** -53
        if neighbours:
            size[:, 0:2 * n] = np.repeat(y[:, 0:2 * n:2] + y[:, 1:2 * n:2], 2, -1)
            angle[0:2 * n] = np.repeat(turn, 2)
        else:
            size[:, :2 * n] = np.tile(y[:, :n] + y[:, n:2 * n], 2)
            angle[:2 * n] = np.tile(turn, 2)
        off = size * ((hd / 2 + 8) * 2.0 ** -24 + 2.0 ** -20 + angle)
        tol = half * (np.abs(want) + off) + off + tiny
        assert (np.abs(on[t] - want) <= tol).all(), (t, p, np.abs(on[t] - want).max())


def check_held_rows(out, lse, q, per_row, scale):
    """Attention over a cache of 8 bits; ``per_row`` as for check_rows.

    Beyond attn_oracle.tolerances with weights in two terms (of fp16): queries are exact in fp16 but for what is 2^-28 of a head's largest, where
    they are off by 2^-39 of that (nothing beside the fp32 sums' own bound); a weight is off by 2^-25 of the largest where it is below
    fp16's normal numbers, for every token, times values of up to 448 * 2^e, at most twice the largest value.  The log of the sum carries an
    offset of 30 through fp32: 2^-19."""
    fp16 = q.dtype == torch.float16
    qn, on, ln = f64(q), f64(out), f64(lse)
    n, hq, hd = qn.shape
    for i in range(n):
        k, v = per_row(i)
        g = hq // k.shape[1]
        for h in range(hq):
            kk, vv = k[:, h // g], v[:, h // g]
            want, wl, mean, amp = A.attend(qn[i, h], kk, vv, scale)
            most = np.abs(vv).max() if len(kk) else 0.0
            tol, tl = A.tolerances(want, wl, mean, amp, len(kk), hd, fp16, False, most)
            tol = tol + len(kk) * 2.0 ** -24 * most
            assert (np.abs(on[i, h] - want) <= tol).all(), (i, h, np.abs(on[i, h] - want).max(), tol.min())
            if len(kk) == 0:
                assert ln[i, h] == -np.inf and (on[i, h] == 0).all()
            else:
                assert abs(ln[i, h] - wl) <= tl + 2.0 ** -18, (i, h, ln[i, h], wl, tl)
