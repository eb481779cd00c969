"""Plain oracle of the paged key-value cache and its attention (64-bit numpy, no code shared with the GPU path).

``Pool`` keeps lists of page numbers per sequence and a count per page; the rules are those of ``include/np.h``: pages are taken
in list order, the lowest free number first; forks share full pages and copy a partly filled one; a compaction moves the i-th
live page behind the live count to the i-th hole before it.
"""
import numpy as np

S_PAGE, S_SEQ, S_LENGTH, S_TIMEOUT, S_FULL = 1, 2, 4, 8, 32


class Pool:
    def __init__(self, page_tokens, n_pages, max_seqs, max_pages):
        self.P, self.n_pages, self.max_seqs, self.max_pages = page_tokens, n_pages, max_seqs, max_pages
        self.pages = [[] for _ in range(max_seqs)]
        self.lens = [0] * max_seqs
        self.status = 0

    # ---- the tables as the device holds them
    def refs(self):
        r = np.zeros(self.n_pages, np.int32)
        for row in self.pages:
            for p in row:
                r[p] += 1
        return r

    def table(self):
        t = np.full((self.max_seqs, self.max_pages), -1, np.int32)
        for s, row in enumerate(self.pages):
            t[s, :len(row)] = row
        return t

    def free_pages(self):
        return np.flatnonzero(self.refs() == 0).tolist()

    def _known(self, s, earlier):
        if not 0 <= s < self.max_seqs or s in earlier:
            self.status |= S_SEQ
            return False
        return True

    # ---- calls; each returns what np.h says
    def reserve(self, seqs, n_new):
        free, start, counted = self.free_pages(), [], 0
        for i, (s, add) in enumerate(zip(seqs, n_new)):
            start.append(-1)
            if not self._known(s, seqs[:i]):
                continue
            to = self.lens[s] + add
            now = -(-to // self.P)
            if add < 0 or now > self.max_pages or to > 0x7fffffff:
                self.status |= S_LENGTH
                continue
            need = now - len(self.pages[s])
            counted += need
            if need > 0 and counted > len(free):
                self.status |= S_FULL
                continue
            start[-1] = self.lens[s]
            self.pages[s] = self.pages[s] + free[counted - need:counted]
            self.lens[s] = to
        return start

    def fork(self, src, dst):
        """Pairs (from, to) of pages that are copied."""
        free, counted, copies = self.free_pages(), 0, []
        was_len, was = list(self.lens), [list(r) for r in self.pages]
        for i, (a, b) in enumerate(zip(src, dst)):
            if not self._known(b, dst[:i]):
                continue
            if not 0 <= a < self.max_seqs or was_len[b] != 0:
                self.status |= S_SEQ
                continue
            full, part = divmod(was_len[a], self.P)
            need = 1 if part else 0
            counted += need
            if need and counted > len(free):
                self.status |= S_FULL
                continue
            self.pages[b] = was[a][:full]
            if need:
                self.pages[b].append(free[counted - 1])
                copies.append((was[a][full], free[counted - 1]))
            self.lens[b] = was_len[a]
        return copies

    def free(self, seqs):
        for i, s in enumerate(seqs):
            if self._known(s, seqs[:i]):
                self.pages[s], self.lens[s] = [], 0

    def compact(self):
        """(live count, pairs (from, to) of pages that move)."""
        r = self.refs()
        live = int((r > 0).sum())
        moves = list(zip([p for p in range(live, self.n_pages) if r[p] > 0], [p for p in range(live) if r[p] == 0]))
        new = dict(moves)
        self.pages = [[new.get(p, p) for p in row] for row in self.pages]
        return live, moves


def attend(q, k, v, scale):
    """One row: q [d], k and v [tokens][d], all float64.  (out [d], log of the sum, the weighted mean of |v|, the largest
    scale * sum |q||k|): the last two are what error bounds are made of."""
    if len(k) == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
    z = (k @ q) * scale
    top = z.max()
    e = np.exp(z - top)
    w = e / e.sum()
    return w @ v, top + np.log(e.sum()), w @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * scale)


def tolerances(want, lse, mean_abs, amp, tokens, head_dim, fp16, p_rounded, vmax):
    """Bounds of |out - want| (per element) and of |lse - want|.

    Scores: fp32 sums of head_dim products and a scaling, off by at most (head_dim + 8) 2^-24 amp, which moves a weight by as
    much relative to itself and the sum by no more, so the mean by twice that times mean_abs.  Exponentials are good to 2^-21, the
    sums over the tokens to tokens * 2^-24.  Probabilities that are rounded to the rows' type are off by half a step, 2^-8 (bf16)
    or 2^-11 (fp16) relative to themselves / 2^-25 of the largest below fp16's normal range; two terms square that.  The
    result's own rounding is half a step of it, 2^-25 below fp16's normal range."""
    half = 2.0 ** -11 if fp16 else 2.0 ** -8
    tiny = 2.0 ** -25 if fp16 else 0.0
    ds = (head_dim + 8) * 2.0 ** -24 * amp
    rel = 2 * ds + 2.0 ** -20 + 2 * tokens * 2.0 ** -24 + (half if p_rounded else half * half)
    exact_part = mean_abs * rel + tokens * tiny * vmax
    out = half * (np.abs(want) + exact_part) + exact_part + tiny
    return out, ds + 2.0 ** -20 + tokens * 2.0 ** -24 + (abs(lse) * 2.0 ** -22 if np.isfinite(lse) else 0.0)
