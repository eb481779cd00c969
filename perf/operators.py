"""Workloads of the attention half of a decode step: the paged key-value cache and the attention that reads it.

A case is one call, or the few calls that belong together, of a program that serves with this package:

* ``prompt``   causal attention over packed prompts of different lengths, heads in groups that share keys and values
* ``decode``   attention of one new token per sequence over the paged cache
* ``append``   keys and values of new tokens go into the cache's pages; with ``fresh`` the sequences are freed and get
               their pages anew before that (a prompt that arrives in a slot)
* ``fork``     branches of sequences are dropped and begun again from their parents: full pages are shared, the partly
               filled last page of each is copied in every layer
* ``compact``  live pages move to the lowest page numbers, in every layer; the tables are rewritten into a second set
               (steps that still run read the first)

Shapes are those of the stacks in ``synth.CONFIGS`` (model width = heads * head size: 4 x 64, 32 x 128, 40 x 128,
64 x 128) with all heads' own or eight shared key-value heads.
"""
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}

# (query heads, key-value heads, head size)
LAYOUTS = [(4, 4, 64), (32, 32, 128), (40, 40, 128), (64, 8, 128), (40, 8, 128), (32, 4, 64), (64, 64, 64), (8, 1, 128), (64, 2, 128)]


def _lens(case):
    """Tokens of each sequence: all ``len``, or spread between nothing and ``len`` with both ends among them."""
    n, most = case["n"], case["len"]
    if not case["ragged"]:
        return [most] * n
    r = random.Random(1000 * n + most)
    got = [min(most, int(math.exp(r.uniform(0.0, math.log(most + 1))))) if r.random() < 0.5 else r.randint(0, most) for _ in range(n)]
    got[0] = most
    if n > 2:
        got[n // 2] = 0
        got[-1] = min(1, most)
    return got


def _case(op, heads, **kw):
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "hd": heads[2], "dtype": "bf16", "n": 1, "len": 1, "ragged": False,
         "pad": 0, "page": 64, "layers": 1, "ways": 1, "fresh": False, "past": 0, "live": 50}
    c.update(kw)
    return c


def listed():
    tiny, s7, s70 = (4, 4, 64), (32, 32, 128), (64, 8, 128)
    return [
        # one short prompt with the tiny stack's heads: launches and latency
        _case("prompt", tiny, name="prompt tiny 77", dtype="fp16", len=77),
        # prompts of twelve users in one batch, an empty one and one of a single token among them; rows behind them unused
        _case("prompt", s7, name="prompt 7b packed", n=12, len=1500, ragged=True, pad=13),
        # one long prompt with shared key-value heads: bound by the matrix products
        _case("prompt", s70, name="prompt 70b 8192", len=8192),
        # the next token of one short sequence
        _case("decode", tiny, name="decode tiny 100", dtype="fp16", len=100, page=16),
        # the next token of sixteen sequences of all lengths: the ordinary serving step
        _case("decode", s7, name="decode 7b x16", n=16, len=4095, ragged=True),
        # one sequence with a long history and shared heads: few rows, a long axis
        _case("decode", s70, name="decode 70b 131071", len=131071),
        # one token for each of sixteen sequences goes into the cache (once per layer and step)
        _case("append", s7, name="append 7b x16", n=16, len=1, past=700),
        # a long prompt's keys and values go into a slot's fresh pages
        _case("append", s70, name="append 70b 8192", len=8192, fresh=True),
        # one branch begins from one short parent
        _case("fork", tiny, name="fork tiny", len=75, page=16, layers=2),
        # four parents with four branches each, all layers of the 7B-shaped stack
        _case("fork", s7, name="fork 7b 4x4", n=4, len=500, page=16, layers=32, ways=4),
        # a small pool is closed up
        _case("compact", tiny, name="compact tiny", n=3, len=200, ragged=True, page=16, layers=2),
        # half of the pages of the 70B-shaped stack's pool are live
        _case("compact", s70, name="compact 70b", n=6, len=500, page=64, layers=80),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["prompt", "decode", "append", "fork", "compact"])
    hq, hkv, hd = rng.choice(LAYOUTS)
    heads, dtype, page = (hq, hkv, hd), rng.choice(["bf16", "fp16"]), rng.choice([16, 32, 64, 128, 256])
    token = 4 * hkv * hd                                  # bytes of one token's keys and values in one layer
    if op == "prompt":
        n, total = log(1, 32), log(16, 8000)
        n = min(n, total)
        return _case(op, heads, dtype=dtype, n=n, len=max(1, total // n), ragged=rng.random() < 0.6, pad=rng.choice([0, 5]))
    if op == "decode":
        n = log(1, 128)
        most = max(2, min(131072, 400_000_000 // (token * n)))
        return _case(op, heads, dtype=dtype, n=n, len=log(1, most), ragged=rng.random() < 0.6, page=page)
    if op == "append":
        fresh = rng.random() < 0.5
        n = log(1, 64)
        if fresh:
            return _case(op, heads, dtype=dtype, n=n, len=log(1, max(2, min(16384, 60_000_000 // (token * n)))), ragged=rng.random() < 0.5, fresh=True, page=page)
        return _case(op, heads, dtype=dtype, n=n, len=rng.choice([1, 1, 3, 17]), past=log(1, 2000), page=page)
    layers = rng.choice([2, 32, 40])
    if layers * page * token > 40_000_000:
        page = 16
    pages = max(16, min(256, 800_000_000 // (layers * page * token)))   # pages of the pool, about
    n = log(1, 6)
    if op == "fork":
        # a parent holds its own pages, and each branch one
        ways = rng.randint(1, max(1, min(4, pages // (2 * n))))
        most = max(1, (pages - n * ways) // n) * page
        return _case(op, heads, dtype=dtype, n=n, len=log(1, max(2, most - 1)), ragged=rng.random() < 0.5, page=page, layers=layers, ways=ways)
    return _case(op, heads, dtype=dtype, n=n, len=log(1, max(2, pages // (2 * n) * page)), ragged=rng.random() < 0.5, page=page, layers=layers,
                 live=rng.choice([30, 50, 80]))


def _pages(case):
    """Pages that each sequence of a case holds (``past`` tokens were there before an append)."""
    return [-(-(x + case["past"]) // case["page"]) for x in _lens(case)]


def _partial(case):
    return sum(1 for x in _lens(case) if x % case["page"])


def work(case):
    hq, hkv, hd, lens = case["hq"], case["hkv"], case["hd"], _lens(case)
    t = sum(lens)
    token = 4 * hkv * hd
    if case["op"] == "prompt":
        return {"bytes": t * (4 * hq * hd + token + 4 * hq), "flops": 4 * hd * hq * sum(x * (x + 1) // 2 for x in lens)}
    if case["op"] == "decode":
        return {"bytes": t * token + len(lens) * (4 * hq * hd + 4 * hq), "flops": 4 * hd * hq * t}
    if case["op"] == "append":
        return {"bytes": 2 * t * token, "flops": 0}
    page = case["layers"] * case["page"] * token
    if case["op"] == "fork":
        return {"bytes": 2 * _partial(case) * case["ways"] * page + 8 * sum(_pages(case)) * case["ways"], "flops": 0}
    live, total = sum(_pages(case)), _pool(case)
    return {"bytes": 2 * _moves(case) * page + 8 * (live + total), "flops": 0}


def _pool(case):
    """Pages of a case's pool."""
    used = sum(_pages(case))
    if case["op"] == "fork":
        return used + _partial(case) * case["ways"] + 3
    if case["op"] == "compact":
        return max(used + 1, 100 * used // case["live"])
    return used + 3


def _placed(case, seed):
    """Page numbers of a case's sequences, in token order: scattered over the pool.  The seed decides which, and how many lie where is
    the same for all seeds (what a compaction moves is work of the case)."""
    used, total = sum(_pages(case)), _pool(case)
    r = random.Random(77 * total + used)
    if case["op"] == "append" and case["fresh"]:
        got = list(range(used))                           # taken in order from an empty pool
    else:
        got = r.sample(range(total), used)
        random.Random(seed).shuffle(got)
    return got


def _moves(case):
    used = sum(_pages(case))
    return sum(1 for p in _placed(case, 0) if p >= used)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, hq, hkv, hd, n = DTYPE[case["dtype"]], case["hq"], case["hkv"], case["hd"], case["n"]
    lens = _lens(case)
    s = {"case": case, "scale": 1.0 / math.sqrt(hd)}

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    if case["op"] in ("prompt", "append"):
        rows = cu[-1] + case["pad"]
        # one projection's output holds a token's queries, keys and values side by side
        qkv = randn(rows, hq + 2 * hkv, hd)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["cu"] = ints(cu)
    if case["op"] == "prompt":
        s["out"] = torch.full((rows, hq, hd), 2.0, dtype=dt, device="cuda")
        s["lse"] = torch.full((rows, hq), 2.0, dtype=torch.float32, device="cuda")
        return _handles(s)

    # the paged cache: [layers][pages][keys, values][key-value heads][tokens of a page][head size]
    P, L, per, total = case["page"], case["layers"], _pages(case), _pool(case)
    slots = n * (1 + case["ways"]) if case["op"] == "fork" else n
    s["max_pages"] = max(per) + 1
    s["cache"] = torch.empty((L, total, 2, hkv, P, hd), dtype=dt, device="cuda")
    for layer in s["cache"]:
        layer.copy_(randn(*layer.shape))
    placed, table, refs, at = _placed(case, seed), [[-1] * s["max_pages"] for _ in range(slots)], [0] * total, 0
    for i, m in enumerate(per):
        table[i][:m] = placed[at:at + m]
        for p in placed[at:at + m]:
            refs[p] = 1
        at += m
    s["table"], s["lens"], s["refs"] = ints(table), ints([x + case["past"] for x in lens] + [0] * (slots - n)), ints(refs)
    s["scratch"] = torch.zeros(4 * total + 4096, dtype=torch.int32, device="cuda")
    if case["op"] == "decode":
        s["q"], s["out"] = randn(n, hq, hd), torch.empty((n, hq, hd), dtype=dt, device="cuda")
        s["lse"] = torch.empty((n, hq), dtype=torch.float32, device="cuda")
    elif case["op"] == "append":
        s["seqs"], s["start"], s["new"] = ints(range(n)), ints([case["past"]] * n), ints(lens)
    elif case["op"] == "fork":
        s["src"] = ints([i for i in range(n) for _ in range(case["ways"])])
        s["dst"] = ints(range(n, slots))
    else:
        s["table2"], s["lens2"], s["refs2"] = torch.full_like(s["table"], -1), torch.zeros_like(s["lens"]), torch.zeros_like(s["refs"])
        s["n_live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return _handles(s)


def _handles(s):
    """What a program keeps beside its tensors: the cache's description, its tables by address, the decode call's workspace."""
    if own and "cache" in s:
        from paper_2608_22643_b200 import binding as nb
        L, total, _, hkv, P, hd = s["cache"].shape
        slots, most = s["table"].shape
        s["desc"] = nb.make_kv_desc(s["cache"].dtype, L, hkv, hd, P, total, slots, most)
        s["tables"] = nb.make_kv_tables(s["table"], s["lens"], s["refs"], s["scratch"], s["status"])
        if "table2" in s:
            s["tables2"] = nb.make_kv_tables(s["table2"], s["lens2"], s["refs2"], s["scratch"], s["status"])
        if s["case"]["op"] == "decode":
            s["workspace"] = torch.zeros(nb.np_attn_workspace_bytes(s["desc"], s["q"].shape[1], s["q"].shape[0]), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"prompt": _prompt, "decode": _decode, "append": _append, "fork": _fork, "compact": _compact}[op](s)


def _own(s, op):
    from paper_2608_22643_b200 import binding as nb
    stream = torch.cuda.current_stream()
    if op == "prompt":
        nb.np_attn_prompt(s["q"], s["k"], s["v"], s["cu"], s["out"], s["status"], scale=s["scale"], lse=s["lse"], stream=stream)
        return {"out": s["out"], "lse": s["lse"]}
    if op == "decode":
        nb.np_attn_decode(s["desc"], s["cache"], 0, s["tables"], s["q"], s["out"], s["workspace"], scale=s["scale"], lse=s["lse"], stream=stream)
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        if s["case"]["fresh"]:
            nb.np_kv_free(s["desc"], s["tables"], s["seqs"], stream=stream)
            nb.np_kv_reserve(s["desc"], s["tables"], s["seqs"], s["new"], s["start"], stream=stream)
        nb.np_kv_append(s["desc"], s["cache"], 0, s["tables"], s["k"], s["v"], s["seqs"], s["cu"], s["start"], stream=stream)
    elif op == "fork":
        nb.np_kv_free(s["desc"], s["tables"], s["dst"], stream=stream)
        nb.np_kv_fork(s["desc"], s["cache"], s["tables"], s["src"], s["dst"], stream=stream)
    else:
        nb.np_kv_compact(s["desc"], s["cache"], s["tables"], s["tables2"], s["n_live"], stream=stream)
        return {"cache": s["cache"], "table": s["table2"], "lens": s["lens2"], "refs": s["refs2"], "live": s["n_live"]}
    return {"cache": s["cache"], "table": s["table"], "lens": s["lens"], "refs": s["refs"]}


# ---- plain forms ------------------------------------------------------------------------


def _softmax_sum(scores, v):
    """Softmax of each row of fp32 scores (-inf: not seen; overwritten) times the values, and the log of the sum; an empty row gives
    zeros and -inf."""
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = scores.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (top + total.log()).squeeze(-1)


def _prompt(s):
    q, k, v, cu = s["q"], s["k"], s["v"], s["cu"]
    rows, hq, hd = q.shape
    hkv = k.shape[1]
    g = hq // hkv
    i = torch.arange(rows, device=q.device, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:], i, right=True)          # the sequence of each row; its count: behind the last
    inside = seq < len(cu) - 1
    seen = (seq[:, None] == seq[None, :]) & (i[None, :] <= i[:, None]) & inside[:, None]
    kf = k.float().permute(1, 2, 0)
    vf = torch.where(inside[:, None, None], v.float(), 0.0).permute(1, 0, 2)
    qf = q.float().view(rows, hkv, g, hd).permute(1, 2, 0, 3).reshape(hkv, g * rows, hd)
    scores = torch.matmul(qf, kf).mul_(s["scale"])
    scores.view(hkv, g, rows, rows).masked_fill_(~seen, -math.inf)
    o, lse = _softmax_sum(scores, vf)
    o = o.view(hkv, g, rows, hd).permute(2, 0, 1, 3).reshape(rows, hq, hd)
    lse = lse.view(hkv, g, rows).permute(2, 0, 1).reshape(rows, hq)
    s["out"].copy_(torch.where(inside[:, None, None], o.to(q.dtype), s["out"]))
    s["lse"].copy_(torch.where(inside[:, None], lse, s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _decode(s):
    q, cache, table, lens = s["q"], s["cache"], s["table"], s["lens"]
    n, hq, hd = q.shape
    _, _, _, hkv, P, _ = cache.shape
    g, width = hq // hkv, table.shape[1] * P
    kv = cache[0][table.clamp(min=0)]                         # [n][pages][2][hkv][P][hd]
    kf = kv[:, :, 0].transpose(1, 2).reshape(n, hkv, width, hd).float()
    vf = kv[:, :, 1].transpose(1, 2).reshape(n, hkv, width, hd).float()
    seen = torch.arange(width, device=q.device) < lens[:, None]
    scores = torch.matmul(q.float().view(n, hkv, g, hd), kf.transpose(2, 3)).mul_(s["scale"])
    scores.masked_fill_(~seen[:, None, None, :], -math.inf)
    o, lse = _softmax_sum(scores, vf)
    s["out"].copy_(o.reshape(n, hq, hd))
    s["lse"].copy_(lse.reshape(n, hq))
    return {"out": s["out"], "lse": s["lse"]}


def _release(s, seqs):
    """The listed sequences give their pages back."""
    P, most = s["cache"].shape[4], s["table"].shape[1]
    seqs = seqs.long()
    used = torch.arange(most, device=seqs.device) < (s["lens"][seqs, None] + P - 1) // P
    rows = s["table"][seqs]
    s["refs"].index_add_(0, rows.clamp(min=0).reshape(-1), -used.to(torch.int32).reshape(-1))
    s["table"][seqs] = torch.where(used, torch.full_like(rows, -1), rows)
    s["lens"][seqs] = 0


def _free_pages(s):
    """Page numbers, free ones first, each kind ascending."""
    return torch.sort((s["refs"] > 0).to(torch.int32), stable=True).indices.to(torch.int32)


def _append(s):
    cache, table, cu = s["cache"], s["table"], s["cu"]
    P, most = cache.shape[4], table.shape[1]
    seqs = s["seqs"].long()
    if s["case"]["fresh"]:
        _release(s, seqs)
        free = _free_pages(s)
        need = (s["new"] + P - 1) // P                        # the sequences are empty
        first = need.cumsum(0) - need
        j = torch.arange(most, device=cu.device)
        takes = j < need[:, None]
        page = free[(first[:, None] + j).clamp(max=len(free) - 1)]
        table[seqs] = torch.where(takes, page, table[seqs])
        s["refs"].index_add_(0, page.reshape(-1), takes.to(torch.int32).reshape(-1))
        s["start"].copy_(s["lens"][seqs])
        s["lens"][seqs] = s["start"] + s["new"]
    t = torch.arange(s["k"].shape[0], device=cu.device, dtype=torch.int32)
    i = torch.searchsorted(cu[1:], t, right=True)
    at = (s["start"][i] + t - cu[i]).long()
    page = table[seqs[i], at // P].long()
    cache[0, page, 0, :, at % P] = s["k"]
    cache[0, page, 1, :, at % P] = s["v"]
    return {"cache": cache, "table": table, "lens": s["lens"], "refs": s["refs"]}


def _fork(s):
    cache, table, lens, refs = s["cache"], s["table"], s["lens"], s["refs"]
    src, dst = s["src"].long(), s["dst"].long()
    _release(s, dst)
    P, most = cache.shape[4], table.shape[1]
    full, part = lens[src] // P, lens[src] % P > 0
    j = torch.arange(most, device=src.device)
    shared, last = j < full[:, None], (j == full[:, None]) & part[:, None]
    free = _free_pages(s)
    took = free[(part.cumsum(0) - 1).clamp(min=0)]            # the i-th branch with a partly filled page takes the i-th free page
    rows = table[src]
    refs.index_add_(0, rows.clamp(min=0).reshape(-1), shared.to(torch.int32).reshape(-1))
    refs.index_add_(0, took, part.to(torch.int32))
    of = rows.gather(1, full.clamp(max=most - 1).long()[:, None])[:, 0]
    nobody = free[-1:].expand_as(of)                          # a page that is copied onto itself where there is nothing to copy
    cache[:, torch.where(part, took, nobody).long()] = cache[:, torch.where(part, of, nobody).long()]
    table[dst] = torch.where(shared, rows, torch.where(last, took[:, None], table[dst]))
    lens[dst] = lens[src]
    return {"cache": cache, "table": table, "lens": lens, "refs": refs}


def _compact(s):
    cache, table, lens, refs = s["cache"], s["table"], s["lens"], s["refs"]
    P, total, most = cache.shape[4], refs.shape[0], table.shape[1]
    p = torch.arange(total, device=refs.device, dtype=torch.int32)
    live = refs > 0
    count = live.sum(dtype=torch.int32)
    moves, hole = live & (p >= count), ~live & (p < count)
    # the i-th live page behind the count goes to the i-th hole before it
    holes = torch.sort(hole.to(torch.int32), stable=True, descending=True).indices.to(torch.int32)
    movers = torch.sort(moves.to(torch.int32), stable=True, descending=True).indices.to(torch.int32)
    new = torch.where(moves, holes[(moves.cumsum(0) - 1).clamp(min=0)], p)
    old = torch.where(hole, movers[(hole.cumsum(0) - 1).clamp(min=0)], p)
    cache.copy_(cache[:, old.long()])
    used = torch.arange(most, device=refs.device) < (lens[:, None] + P - 1) // P
    s["table2"].copy_(torch.where(used, new[table.clamp(min=0).long()], -1))
    s["lens2"].copy_(lens)
    s["refs2"].copy_(torch.where(p < count, refs[old.long()], 0))
    s["n_live"].copy_(count)
    return {"cache": cache, "table": s["table2"], "lens": s["lens2"], "refs": s["refs2"], "live": s["n_live"]}


# ---- from the definition, in 64 bits ----------------------------------------------------


def exact(case, seed):
    if case["op"] not in ("prompt", "decode"):
        return None                                           # nothing is computed: bytes are moved and whole numbers kept
    s = prepare(case, seed)
    lens, hq, hkv = _lens(case), case["hq"], case["hkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    if case["op"] == "prompt":
        out[sum(lens):], lse[sum(lens):] = s["out"][sum(lens):].double(), s["lse"][sum(lens):].double()
    at = 0
    for b, x in enumerate(lens):
        if case["op"] == "decode":
            pages = s["table"][b, :-(-x // case["page"])].long()
            k = s["cache"][0, pages, 0].transpose(0, 1).flatten(1, 2)[:, :x]
            v = s["cache"][0, pages, 1].transpose(0, 1).flatten(1, 2)[:, :x]
        for h in range(hq if x else 0):
            c = h // (hq // hkv)
            if case["op"] == "decode":
                z = (k[c].double() @ s["q"][b, h].double()) * s["scale"]
                w = torch.softmax(z, 0)
                out[b, h], lse[b, h] = w @ v[c].double(), torch.logsumexp(z, 0)
            else:
                kk, vv = s["k"][at:at + x, c].double(), s["v"][at:at + x, c].double()
                z = (s["q"][at:at + x, h].double() @ kk.T) * s["scale"]
                z += torch.full((x, x), -math.inf, dtype=torch.float64, device="cuda").triu(1)
                out[at:at + x, h], lse[at:at + x, h] = torch.softmax(z, 1) @ vv, torch.logsumexp(z, 1)
        at += x
    return {"out": out, "lse": lse}
