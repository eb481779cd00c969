"""Workloads of what a decode step does to queries, keys and values between their projection and the attention's result: norm and
rotation, a cache held in 8 bits, and attention of branches that share a prefix.

A case is one call, or the few calls that belong together, of a program that serves with this package:

* ``rotate``   norms of queries and keys per head and their rotation by position, in one pass
* ``enter``    the same, the keys (and the values) going straight into the cache's pages
* ``keep``     keys and values go into a cache that holds them in 8 bits, and are read back as rows
* ``decode``   attention of one new token per sequence over a cache held in 8 bits
* ``shared``   attention of one new token for each branch of groups whose sequences begin with the same pages; how many tokens a
               group shares is found from the page tables

Shapes are those of the stacks in ``synth.CONFIGS`` (model width = heads * head size: 4 x 64, 32 x 128, 40 x 128,
64 x 128) with all heads' own or a few shared key-value heads.
"""
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}

# (query heads, key-value heads, head size)
LAYOUTS = [(4, 4, 64), (32, 32, 128), (40, 40, 128), (64, 8, 128), (40, 8, 128), (32, 4, 64), (64, 64, 64), (8, 1, 128), (64, 4, 128)]


def _spread(case, most, least=0):
    """One number for each sequence: all ``most``, or (ragged) spread from ``least`` to ``most`` with both ends among them."""
    n = case["n"]
    if not case["ragged"]:
        return [most] * n
    r = random.Random(1000 * n + most)
    got = [min(most, max(least, int(math.exp(r.uniform(0.0, math.log(most + 1)))))) if r.random() < 0.5 else r.randint(min(least, most), most) for _ in range(n)]
    got[0] = most
    if n > 2:
        got[n // 2] = min(least, most)
        got[-1] = min(1, most)
    return got


def _case(op, heads, **kw):
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "hd": heads[2], "dtype": "bf16", "n": 1, "len": 1, "ragged": False, "page": 64, "past": 0,
         "norm": True, "turned": heads[2], "neighbours": False, "base": 10000.0, "ways": 1, "held": 0}
    c.update(kw)
    return c


def listed():
    tiny, s7, s70 = (4, 4, 64), (32, 32, 128), (64, 8, 128)
    return [
        # the next token of one sequence with the tiny stack's heads: launch and latency
        _case("rotate", tiny, name="rotate tiny 1", dtype="fp16", past=500, neighbours=True),
        # a batch of prompts of different lengths far into their sequences, half of each head turned
        _case("rotate", s70, name="rotate 70b 9 prompts", n=9, len=2000, ragged=True, past=1000000, turned=64, base=500000.0),
        # the next token of sixteen sequences goes through and into the cache: once per layer and step
        _case("enter", s7, name="enter 7b x16", n=16, past=700),
        # a long prompt, without norms
        _case("enter", s70, name="enter 70b 8192", len=8192, norm=False, base=500000.0),
        # the next token of sixteen sequences into 8 bits and out again
        _case("keep", s7, name="keep 7b x16", n=16, past=700),
        # prompts of different lengths into 8 bits and out again
        _case("keep", s70, name="keep 70b 5 prompts", dtype="fp16", n=5, len=4000, ragged=True),
        # the next token of one short sequence
        _case("decode", tiny, name="decode tiny 100", dtype="fp16", len=100, page=16),
        # the next token of sixteen sequences of all lengths: the ordinary serving step
        _case("decode", s7, name="decode 7b x16", n=16, len=4095, ragged=True),
        # one sequence with a long history and shared heads: few rows, a long axis
        _case("decode", s70, name="decode 70b 131071", len=131071),
        # two branches of one short sequence
        _case("shared", tiny, name="shared tiny 2", dtype="fp16", n=2, ways=2, held=96, len=20, page=16),
        # four parents with four branches each
        _case("shared", s7, name="shared 7b 4x4", n=16, ways=4, held=2048, len=300, ragged=True, page=16),
        # sixty-four users behind one long instruction
        _case("shared", s70, name="shared 70b 64", n=64, ways=64, held=8192, len=200, ragged=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotate", "enter", "keep", "decode", "shared"])
    heads = rng.choice(LAYOUTS)
    hq, hkv, hd = heads
    kw = {"dtype": rng.choice(["bf16", "fp16"]), "page": rng.choice([16, 32, 64, 128, 256]), "ragged": rng.random() < 0.6}
    if op in ("rotate", "enter"):
        kw.update(norm=rng.random() < 0.6, turned=rng.choice([hd, hd, hd // 2, 32]), neighbours=rng.random() < 0.4, base=rng.choice([10000.0, 500000.0]))
    if op in ("rotate", "enter", "keep"):
        tokens = min(8000, 60_000_000 // ((hq + 2 * hkv) * hd))
        if rng.random() < 0.4:                                # a decode step
            n = log(1, 128)
            return _case(op, heads, n=n, past=log(1, 500 if op != "rotate" else 1000000), **dict(kw, ragged=False))
        n = log(1, 16)
        return _case(op, heads, n=n, len=log(2, max(4, tokens // n)), past=rng.choice([0, 0, log(1, 300)]), **kw)
    if op == "decode":
        n = log(1, 128)
        return _case(op, heads, n=n, len=log(1, max(2, min(131072, 250_000_000 // (2 * hkv * hd * n)))), **kw)
    ways, groups = log(2, 64), log(1, 8)
    ways = max(2, min(ways, 96 // groups))
    n, most = ways * groups, 400_000_000 // (ways * groups * hkv * hd)   # tokens of a sequence
    tail = log(1, max(2, min(600, most // 4)))
    held = max(1, log(1, max(2, (most - tail) // kw["page"]))) * kw["page"]
    return _case(op, heads, n=n, ways=ways, held=held, len=tail, **kw)


def _new(case):
    """Tokens of each sequence that a case is about; a decode's are the sequence, a shared one's those behind the prefix."""
    return _spread(case, case["len"], 1 if case["op"] == "shared" else 0)


def _lens(case):
    return [x + case["past"] + case["held"] for x in _new(case)]


def work(case):
    hq, hkv, hd, new = case["hq"], case["hkv"], case["hd"], _new(case)
    t = sum(new)
    if case["op"] == "rotate":
        return {"bytes": 4 * t * (hq + hkv) * hd, "flops": 0}
    if case["op"] == "enter":
        return {"bytes": 4 * t * (hq + 2 * hkv) * hd, "flops": 0}
    if case["op"] == "keep":                                  # rows in, 8 bits out; 8 bits in, rows out
        return {"bytes": t * 2 * hkv * (2 * hd + 2 * (hd + 1) + 2 * hd), "flops": 0}
    rows = len(new) * (4 * hq * hd + 4 * hq)
    if case["op"] == "decode":
        return {"bytes": t * 2 * hkv * (hd + 1) + rows, "flops": 4 * hd * hq * t}
    groups = len(new) // case["ways"]
    return {"bytes": (groups * case["held"] + t) * 4 * hkv * hd + rows, "flops": 4 * hd * hq * (t + len(new) * case["held"])}


def _tables(case, seed):
    """Rows of page numbers, scattered over the pool; the branches of a group begin with the same pages.  And the pool's size."""
    P, n, ways = case["page"], case["n"], case["ways"]
    first = case["held"] // P
    per = [-(-x // P) for x in _lens(case)]
    used = sum(m - first for m in per) + (n // ways) * first
    total = used + 3
    placed = list(range(total))
    random.Random(seed).shuffle(placed)
    rows, at = [], 0
    for i, m in enumerate(per):
        if i % ways == 0:
            shared, at = placed[at:at + first], at + first
        rows.append(shared + placed[at:at + m - first])
        at += m - first
    return rows, total


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, op = DTYPE[case["dtype"]], case["op"]
    hq, hkv, hd, n, P = case["hq"], case["hkv"], case["hd"], case["n"], case["page"]
    s = {"case": case, "scale": 1.0 / math.sqrt(hd)}

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    new = _new(case)
    if op in ("rotate", "enter", "keep"):
        # one projection's output holds a token's queries, keys and values side by side
        qkv = randn(sum(new), hq + 2 * hkv, hd)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["cu"] = None if new == [1] * n else ints([sum(new[:i]) for i in range(n + 1)])
        r = random.Random(seed)
        s["start"] = ints([r.randint(0, case["past"]) for _ in new] if op == "rotate" else [case["past"]] * n)
    if op in ("rotate", "enter"):
        half = case["turned"] // 2
        s["freq"] = case["base"] ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        s["q_gain"] = s["k_gain"] = None
        if case["norm"]:
            s["q_gain"], s["k_gain"] = (1.0 + 0.1 * torch.randn(hd, generator=g, device="cuda") for _ in range(2))
        s["q_out"] = torch.empty((sum(new), hq, hd), dtype=dt, device="cuda")
    if op in ("rotate", "keep"):
        s["k_out"], s["v_out"] = (torch.empty((sum(new), hkv, hd), dtype=dt, device="cuda") for _ in range(2))
    if op == "rotate":
        return _handles(s)

    rows, total = _tables(case, seed)
    width = max(len(r) for r in rows) + 1
    s["table"], s["lens"] = ints([r + [-1] * (width - len(r)) for r in rows]), ints(_lens(case))
    refs = [0] * total
    for row in rows:
        for p in row:
            refs[p] += 1
    s["refs"], s["status"] = ints(refs), ints([0])
    s["scratch"] = torch.zeros(4 * total + 4096, dtype=torch.int32, device="cuda")
    s["seqs"] = ints(range(n))
    if op in ("keep", "decode"):
        # [layers][pages][bytes of a page]: e4m3 [keys, values][key-value heads][tokens of a page][head size], then a power of two for each
        # of these rows, as its biased exponent
        s["cache"] = torch.empty((1, total, 2 * hkv * P * (hd + 1)), dtype=torch.uint8, device="cuda")
        values = s["cache"][0, :, :2 * hkv * P * hd]
        for at in range(0, total, 64):
            part = values[at:at + 64]
            part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 100.0).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8))
        s["cache"][0, :, 2 * hkv * P * hd:] = torch.randint(118, 122, (total, 2 * hkv * P), generator=g, device="cuda", dtype=torch.uint8)
    else:
        s["cache"] = torch.empty((1, total, 2, hkv, P, hd), dtype=dt, device="cuda")
        for at in range(0, total, 64):
            s["cache"][0, at:at + 64] = randn(*s["cache"][0, at:at + 64].shape)
    if op in ("decode", "shared"):
        s["q"], s["out"] = randn(n, hq, hd), torch.empty((n, hq, hd), dtype=dt, device="cuda")
        s["lse"] = torch.empty((n, hq), dtype=torch.float32, device="cuda")
    if op == "shared":
        s["cu"] = ints(range(0, n + 1, case["ways"]))
        s["held"] = torch.zeros(n // case["ways"], dtype=torch.int32, device="cuda")
    return _handles(s)


def _handles(s):
    """What a program keeps beside its tensors: the cache's description, its tables by address, the rotation, a workspace."""
    if not own:
        return s
    from paper_2608_22643_b200 import binding as nb
    c = s["case"]
    if "freq" in s:
        s["rotation"] = nb.make_rotation(s["freq"], s["q_gain"], s["k_gain"], neighbours=c["neighbours"], eps=1e-6)
    if "cache" in s:
        slots, width = s["table"].shape
        s["desc"] = nb.make_kv_desc(DTYPE[c["dtype"]], 1, c["hkv"], c["hd"], c["page"], s["cache"].shape[1], slots, width, e4m3=c["op"] in ("keep", "decode"))
        s["tables"] = nb.make_kv_tables(s["table"], s["lens"], s["refs"], s["scratch"], s["status"])
    if c["op"] == "decode":
        s["workspace"] = torch.zeros(nb.np_attn_workspace_bytes(s["desc"], c["hq"], c["n"]), dtype=torch.uint8, device="cuda")
    if c["op"] == "shared":
        s["workspace"] = torch.zeros(nb.np_attn_shared_workspace_bytes(s["desc"], c["hq"], c["n"]), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"rotate": _rotate, "enter": _enter, "keep": _keep, "decode": _decode, "shared": _shared}[op](s)


def _own(s, op):
    from paper_2608_22643_b200 import binding as nb
    stream = torch.cuda.current_stream()
    if op == "rotate":
        nb.np_attn_rotate(s["rotation"], s["q"], s["k"], s["q_out"], s["k_out"], s["cu"], s["start"], stream=stream)
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "enter":
        nb.np_kv_append_rotated(s["desc"], s["cache"], 0, s["tables"], s["rotation"], s["q"], s["k"], s["v"], s["q_out"], s["seqs"], s["cu"], s["start"],
                                stream=stream)
        return {"q": s["q_out"], "cache": s["cache"]}
    if op == "keep":
        nb.np_kv_append(s["desc"], s["cache"], 0, s["tables"], s["k"], s["v"], s["seqs"], s["cu"], s["start"], stream=stream)
        nb.np_kv_read(s["desc"], s["cache"], 0, s["tables"], s["k_out"], s["v_out"], s["seqs"], s["cu"], s["start"], stream=stream)
        return {"k": s["k_out"], "v": s["v_out"]}
    if op == "decode":
        nb.np_attn_decode(s["desc"], s["cache"], 0, s["tables"], s["q"], s["out"], s["workspace"], scale=s["scale"], lse=s["lse"], stream=stream)
        return {"out": s["out"], "lse": s["lse"]}
    nb.np_kv_shared(s["desc"], s["tables"], s["seqs"], s["cu"], s["held"], stream=stream)
    nb.np_attn_decode_shared(s["desc"], s["cache"], 0, s["tables"], s["q"], s["out"], s["workspace"], s["cu"], s["held"], scale=s["scale"], lse=s["lse"],
                             stream=stream)
    return {"held": s["held"], "out": s["out"], "lse": s["lse"]}


# ---- plain forms ------------------------------------------------------------------------


def _where(s):
    """The sequence of each row of a call, and the row's position."""
    t = torch.arange(s["k"].shape[0], device="cuda", dtype=torch.int32)
    if s["cu"] is None:
        return t, s["start"]
    i = torch.searchsorted(s["cu"][1:], t, right=True)
    return i, s["start"][i] + t - s["cu"][i]


def _turn(s, x, gain, angles):
    """Norm and rotation of fp32 rows [tokens][heads][head size]."""
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain
    turned = s["case"]["turned"]
    half = turned // 2
    cos, sin = angles.cos().float()[:, None], angles.sin().float()[:, None]
    if s["case"]["neighbours"]:
        a, b = x[..., 0:turned:2], x[..., 1:turned:2]
        pairs = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:turned]
        pairs = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((pairs, x[..., turned:]), -1)


def _rotate(s):
    angles = _where(s)[1].double()[:, None] * s["freq"]       # far positions: 32 bits would lose the angle
    s["q_out"].copy_(_turn(s, s["q"].float(), s["q_gain"], angles))
    s["k_out"].copy_(_turn(s, s["k"].float(), s["k_gain"], angles))
    return {"q": s["q_out"], "k": s["k_out"]}


def _places(s):
    """Page and place in it of each row of a call."""
    i, at = _where(s)
    P = s["case"]["page"]
    return s["table"][s["seqs"][i].long(), (at // P).long()].long(), (at % P).long()


def _enter(s):
    angles = _where(s)[1].double()[:, None] * s["freq"]
    s["q_out"].copy_(_turn(s, s["q"].float(), s["q_gain"], angles))
    page, at = _places(s)
    s["cache"][0, page, 0, :, at] = _turn(s, s["k"].float(), s["k_gain"], angles).to(s["k"].dtype)
    s["cache"][0, page, 1, :, at] = s["v"]
    return {"q": s["q_out"], "cache": s["cache"]}


def _parts(s, layer=0):
    """A layer's values [pages][2][heads][tokens][head size] and exponents [pages][2][heads][tokens], as bytes."""
    c = s["case"]
    pages, split = s["cache"].shape[1], 2 * c["hkv"] * c["page"] * c["hd"]
    shape = (pages, 2, c["hkv"], c["page"])
    return s["cache"][layer, :, :split].view(*shape, c["hd"]), s["cache"][layer, :, split:].view(shape)


def _power(e):
    """2^(e - 127) for bytes e of 1 to 254."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _keep(s):
    values, exponents = _parts(s)
    page, at = _places(s)
    x = torch.stack((s["k"], s["v"]), 1).float()              # [tokens][2][heads][head size]
    top = x.abs().amax(-1).view(torch.int32)
    e = ((top >> 23) - 8 + ((top & 0x7fffff) > 0x600000).int()).clamp(67, 247)   # the least 2^(e - 127) with top <= 448 * 2^(e - 127)
    q = (x * _power(254 - e)[..., None]).to(torch.float8_e4m3fn)
    values[page, :, :, at] = q.view(torch.uint8)
    exponents[page, :, :, at] = e.to(torch.uint8)
    back = values[page, :, :, at].view(torch.float8_e4m3fn).float() * _power(exponents[page, :, :, at])[..., None]
    s["k_out"].copy_(back[:, 0])
    s["v_out"].copy_(back[:, 1])
    return {"k": s["k_out"], "v": s["v_out"]}


def _attend(s, kv):
    """Attention of one token per sequence over gathered pages, fp32 [sequences][pages][2][heads][tokens][head size]."""
    q = s["q"]
    n, hq, hd = q.shape
    hkv, width = kv.shape[3], kv.shape[1] * kv.shape[4]
    kf = kv[:, :, 0].transpose(1, 2).reshape(n, hkv, width, hd)
    vf = kv[:, :, 1].transpose(1, 2).reshape(n, hkv, width, hd)
    seen = torch.arange(width, device=q.device) < s["lens"][:, None]
    scores = torch.matmul(q.float().view(n, hkv, hq // hkv, hd), kf.transpose(2, 3)).mul_(s["scale"])
    scores.masked_fill_(~seen[:, None, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = scores.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    s["out"].copy_((torch.matmul(e, vf) / torch.where(total > 0, total, torch.ones_like(total))).view(n, hq, hd))
    s["lse"].copy_((top + total.log()).view(n, hq))
    return {"out": s["out"], "lse": s["lse"]}


def _decode(s):
    values, exponents = _parts(s)
    pages = s["table"].clamp(min=0).long()
    return _attend(s, values[pages].view(torch.float8_e4m3fn).float() * _power(exponents[pages])[..., None])


def _shared(s):
    P, ways = s["case"]["page"], s["case"]["ways"]
    rows = s["table"][s["seqs"].long()]
    full = (s["lens"][s["seqs"].long()] // P)[:, None]
    first = rows[::ways].repeat_interleave(ways, 0)
    same = (rows == first) & (torch.arange(rows.shape[1], device=rows.device) < full)
    count = same.int().cumprod(1).sum(1)                      # pages that a row has in common with its group's first
    s["held"].copy_(count.view(-1, ways).amin(1) * P)
    return {"held": s["held"], **_attend(s, s["cache"][0][s["table"].clamp(min=0).long()].float())}


# ---- from the definition, in 64 bits ----------------------------------------------------


def _turned(case, x, gain, at, freq):
    x = x.double()
    if gain is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * gain.double()
    turned = case["turned"]
    z = torch.polar(torch.ones_like(at[:, None] * freq), at[:, None] * freq)[:, None]
    out = x.clone()
    if case["neighbours"]:
        w = torch.view_as_complex(x[..., :turned].reshape(*x.shape[:-1], turned // 2, 2).contiguous()) * z
        out[..., 0:turned:2], out[..., 1:turned:2] = w.real, w.imag
    else:
        w = torch.complex(x[..., :turned // 2].contiguous(), x[..., turned // 2:turned].contiguous()) * z
        out[..., :turned // 2], out[..., turned // 2:turned] = w.real, w.imag
    return out


def _e4m3(x):
    """Rows of 64-bit values as e4m3 times a power of two for each holds them."""
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                                   # top = m * 2^e, m in [1/2, 1); 448 = 0.875 * 2^9
    scale = torch.ldexp(torch.ones_like(top), (e - 9 + (m > 0.875).int()).clamp(-60, 120))
    y = x / scale
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step * scale


def exact(case, seed):
    s = prepare(case, seed)
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    starts = s["start"].tolist() if "start" in s else []
    at = [p + j for p, x in zip(starts, _new(case)) for j in range(x)]
    if op in ("rotate", "enter"):
        pos = torch.tensor(at, dtype=torch.float64, device="cuda")
        q, k = _turned(case, s["q"], s["q_gain"], pos, s["freq"]), _turned(case, s["k"], s["k_gain"], pos, s["freq"])
        if op == "rotate":
            return {"q": q, "k": k}
        cache, P = s["cache"].double(), case["page"]
        page = torch.tensor([int(b) for row, p, x in zip(s["table"].tolist(), starts, _new(case)) for b in (row[(p + j) // P] for j in range(x))], device="cuda")
        place = torch.tensor([p % P for p in at], device="cuda")
        cache[0, page, 0, :, place], cache[0, page, 1, :, place] = k, s["v"].double()
        return {"q": q, "cache": cache}
    if op == "keep":
        return {"k": _e4m3(s["k"].double()), "v": _e4m3(s["v"].double())}
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for b, x in enumerate(_lens(case)):
        pages = s["table"][b, :-(-x // case["page"])].long()
        if op == "decode":
            values, exponents = _parts(s)
            kv = torch.ldexp(values[pages].view(torch.float8_e4m3fn).double(), (exponents[pages].int() - 127)[..., None])
        else:
            kv = s["cache"][0, pages].double()
        k, v = (kv[:, i].transpose(0, 1).flatten(1, 2)[:, :x] for i in (0, 1))
        for h in range(hq if x else 0):
            c = h // (hq // hkv)
            z = (k[c] @ s["q"][b, h].double()) * s["scale"]
            out[b, h], lse[b, h] = torch.softmax(z, 0) @ v[c], torch.logsumexp(z, 0)
    return {"out": out, "lse": lse} if op == "decode" else {"held": None, "out": out, "lse": lse}
