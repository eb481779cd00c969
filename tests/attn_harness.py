"""Shared set-up of the cache and attention tests: a cache on the GPU with its tables beside the oracle's pool."""
import numpy as np
import torch

from oracle import attn_oracle as A
from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Cache:
    """A pool of pages on the device and the oracle's, moved by the same calls.  The cache starts as NaN: what a call must not
    read shows in its results."""

    def __init__(self, dtype=torch.bfloat16, layers=1, hkv=2, hd=64, P=16, n_pages=32, max_seqs=8, max_pages=None, fill=float("nan")):
        nbuild.build()
        self.dtype, self.hkv, self.hd, self.P = dtype, hkv, hd, P
        max_pages = n_pages if max_pages is None else max_pages
        self.desc = nb.make_kv_desc(dtype, layers, hkv, hd, P, n_pages, max_seqs, max_pages)
        self.cache = torch.full((layers, n_pages, 2, hkv, P, hd), fill, dtype=dtype, device="cuda")
        ints = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.lens, self.refs, self.status = ints(max_seqs, max_pages), ints(max_seqs), ints(n_pages), ints(1)
        self.scratch = ints(nb.np_kv_sizes(self.desc).scratch_bytes // 4)
        self.tables = nb.make_kv_tables(self.table, self.lens, self.refs, self.scratch, self.status)
        self.pool = A.Pool(P, n_pages, max_seqs, max_pages)
        nb.np_kv_reset(self.desc, self.tables)

    def dev(self, v):
        return torch.tensor(list(v), dtype=torch.int32, device="cuda")

    def check(self):
        """Tables and status are the oracle's."""
        torch.cuda.synchronize()
        assert self.lens.tolist() == self.pool.lens
        assert (self.table.cpu().numpy() == self.pool.table()).all()
        assert (self.refs.cpu().numpy() == self.pool.refs()).all()
        assert self.status.item() == self.pool.status

    def reserve(self, seqs, n_new):
        start = torch.full((len(seqs),), 99, dtype=torch.int32, device="cuda")
        nb.np_kv_reserve(self.desc, self.tables, self.dev(seqs), self.dev(n_new), start)
        want = self.pool.reserve(list(seqs), list(n_new))
        assert start.tolist() == want
        return start, want

    def append(self, layer, seqs, start, counts, seed=0):
        """Random tokens, handed over as slices of one projection's output; returns them as (k, v) of the call."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows = sum(counts)
        kv = torch.randn(rows, 2 * self.hkv, self.hd, generator=g, device="cuda").to(self.dtype)
        k, v = kv[:, :self.hkv], kv[:, self.hkv:]
        cu = self.dev(np.concatenate([[0], np.cumsum(counts)]))
        nb.np_kv_append(self.desc, self.cache, layer, self.tables, k, v, self.dev(seqs), cu, start)
        return k, v

    def grow(self, seqs, counts, seed=0):
        start, _ = self.reserve(seqs, counts)
        for layer in range(self.desc.n_layers):
            self.append(layer, seqs, start, counts, seed + layer)

    def tokens(self, layer, s):
        """Keys and values of a sequence as the oracle's pages say, [tokens][hkv][hd] float64 (copied to the host once)."""
        n = self.pool.lens[s]
        pages = torch.tensor(self.pool.pages[s], dtype=torch.long, device="cuda")
        got = f64(self.cache[layer, pages])                    # [pages][2][hkv][P][hd]
        got = got.transpose(1, 0, 3, 2, 4).reshape(2, -1, self.hkv, self.hd)[:, :n]
        return got[0], got[1]


def check_rows(out, lse, q, per_row, scale, p_rounded):
    """``per_row``: for row i the (k, v) [tokens][hkv][hd] that it sees.  Every element within its own bound."""
    fp16 = q.dtype == torch.float16
    qn, on, ln = f64(q), f64(out), f64(lse)
    n, hq, hd = qn.shape
    for i in range(n):
        k, v = per_row(i)
        g = hq // k.shape[1]
        for h in range(hq):
            kk, vv = k[:, h // g], v[:, h // g]
            want, wl, mean, amp = A.attend(qn[i, h], kk, vv, scale)
            tol, tl = A.tolerances(want, wl, mean, amp, len(kk), hd, fp16, p_rounded, np.abs(vv).max() if len(kk) else 0.0)
            assert (np.abs(on[i, h] - want) <= tol).all(), (i, h, np.abs(on[i, h] - want).max(), tol.min())
            if len(kk) == 0:
                assert ln[i, h] == -np.inf and (on[i, h] == 0).all()
            else:
                assert abs(ln[i, h] - wl) <= tl, (i, h, ln[i, h], wl, tl)
