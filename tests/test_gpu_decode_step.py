"""The attention half of a decode step as a program runs it: prompts through norm, rotation, cache and attention, then steps of branches over
the prefix that they share, in a 16-bit cache and in one of 8 bits; each call's result against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from tests.attn_harness import Cache, check_rows
from tests.rows_harness import Held, check_held_rows, check_rotated, frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("make", [Cache, Held])
@pytest.mark.parametrize("dtype,hq,hkv,hd,P", [(torch.float16, 4, 4, 64, 16), (torch.bfloat16, 16, 2, 128, 32)])
def test_prompts_branches_and_steps(make, dtype, hq, hkv, hd, P):
    layers, lens, ways, steps = 2, [5 * P + 3, 2 * P, 1], 3, 4
    c = make(dtype=dtype, layers=layers, hkv=hkv, hd=hd, P=P, n_pages=80, max_seqs=16)
    held = make is Held
    gen = torch.Generator(device="cuda").manual_seed(0)
    freq = frequencies(hd)
    gain = 1 + 0.1 * torch.randn(hd, generator=gen, device="cuda")
    rotation = nb.make_rotation(freq, gain, gain)
    scale = hd ** -0.5

    def project(rows):
        x = torch.randn(rows, hq + 2 * hkv, hd, generator=gen, device="cuda").to(dtype)
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    def enter(layer, seqs, cu, start, positions):
        """Rotated queries; the cache's keys are what rotation alone gives."""
        q, k, v = project(len(positions))
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        nb.np_kv_append_rotated(c.desc, c.cache, layer, c.tables, rotation, q, k, v, qo, seqs, cu, start)
        check_rotated(qo, q, gain, 1e-6, positions, freq, False)
        nb.np_attn_rotate(rotation, q, k, torch.empty_like(q), ko, cu, start)
        kr, vr = torch.empty_like(k), torch.empty_like(v)
        nb.np_kv_read(c.desc, c.cache, layer, c.tables, kr, vr, seqs, cu, start)
        torch.cuda.synchronize()
        if held:
            assert ((kr.float() - ko.float()).abs() <= ko.float().abs() * 2.0 ** -4 + ko.float().abs().amax(-1, keepdim=True) * 2.0 ** -17).all()
        else:
            assert torch.equal(kr, ko) and torch.equal(vr, v)
        return qo, ko, v

    # ---- prompts
    parents = c.dev(range(3))
    start, _ = c.reserve(range(3), lens)
    cu = np.concatenate([[0], np.cumsum(lens)])
    positions = [j for n in lens for j in range(n)]
    for layer in range(layers):
        q, k, v = enter(layer, parents, c.dev(cu), start, positions)
        out, lse = torch.empty_like(q), torch.empty(len(positions), hq, device="cuda")
        nb.np_attn_prompt(q, k, v, c.dev(cu), out, c.status, lse=lse)
        kn, vn = k.double().cpu().numpy(), v.double().cpu().numpy()
        row = [(int(cu[i]), int(cu[i]) + j + 1) for i, n in enumerate(lens) for j in range(n)]
        check_rows(out, lse, q, lambda i: (kn[row[i][0]:row[i][1]], vn[row[i][0]:row[i][1]]), scale, True)

    # ---- branches of the prompts, which go their own ways
    src, dst = [i for i in range(3) for _ in range(ways)], list(range(3, 3 + 3 * ways))
    nb.np_kv_fork(c.desc, c.cache, c.tables, c.dev(src), c.dev(dst))
    c.pool.fork(src, dst)
    c.check()
    n = len(dst)
    seqs, groups, shared = c.dev(dst), c.dev(range(0, n + 1, ways)), c.dev([0] * 3)
    ws = torch.zeros(nb.np_attn_shared_workspace_bytes(c.desc, hq, n), dtype=torch.uint8, device="cuda")
    other = torch.zeros(nb.np_attn_workspace_bytes(c.desc, hq, n), dtype=torch.uint8, device="cuda")
    for _ in range(steps):
        start, at = c.reserve(dst, [1] * n)
        nb.np_kv_shared(c.desc, c.tables, seqs, groups, shared)
        for layer in range(layers):
            q, _, _ = enter(layer, seqs, None, start, at)
            out, lse, plain = torch.empty_like(q), torch.empty(n, hq, device="cuda"), torch.empty_like(q)
            nb.np_attn_decode_shared(c.desc, c.cache, layer, c.tables, q, out, ws, groups, shared, seqs=seqs, lse=lse)
            nb.np_attn_decode(c.desc, c.cache, layer, c.tables, q, plain, other, seqs=seqs)
            torch.cuda.synchronize()
            kept = [c.tokens(layer, s) for s in dst]
            if held:
                check_held_rows(out, lse, q, lambda i: kept[i], scale)
                assert torch.equal(out, plain)
            else:
                check_rows(out, lse, q, lambda i: kept[i], scale, True)
                check_rows(plain, lse, q, lambda i: kept[i], scale, False)
        assert shared.tolist() == [5 * P, 2 * P, 0]
    c.check()
