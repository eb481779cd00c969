"""np_attn_decode_shared's workspace at any 16-byte aligned address."""
import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild

BF = torch.bfloat16


@pytest.mark.parametrize("heads,n", [(4, 1), (8, 4), (512, 1024)])
def test_there_is_room_for_a_beginning_that_is_aligned(heads, n):
    """What the kernels keep there is a multiple of 32 bytes long and begins at one (they store 32 bytes at a time); the caller's address is a multiple of 16."""
    nbuild.build()
    size = nb.np_attn_shared_workspace_bytes(nb.make_kv_desc(BF, 2, 4, 128, 64, 100, 8, 50), heads, n)
    assert size % 32 == 16


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, torch.float16])
@pytest.mark.parametrize("ways,hq,hd", [(3, 2, 64), (40, 2, 64), (70, 8, 128), (6, 16, 128)])
def test_a_workspace_between_multiples_of_32(dtype, ways, hq, hd):
    """Small groups and large ones: the results of an aligned workspace, twice, and nothing written around it."""
    from tests.test_gpu_attn_shared import _branches
    c, seqs, cu = _branches(dtype, 2, hd, 16, [1600], [[20, 300] + [1] * (ways - 2)])
    q = torch.randn(ways, hq, hd, device="cuda").to(dtype)
    size = nb.np_attn_shared_workspace_bytes(c.desc, hq, ways)
    got = []
    for at in (0, 16, 48, 240):
        room = torch.full((at + size + 512,), 0x5a, dtype=torch.uint8, device="cuda")
        assert room.data_ptr() % 32 == 0
        ws = room[at:at + size]
        ws.zero_()
        for _ in range(2):
            out, lse = torch.full_like(q, 7.0), torch.full((ways, hq), 7.0, device="cuda")
            nb.np_attn_decode_shared(c.desc, c.cache, 0, c.tables, q, out, ws, c.dev(cu), c.dev([1600]), seqs=c.dev(seqs), lse=lse)
            got.append((out, lse))
        torch.cuda.synchronize()
        assert (room[:at] == 0x5a).all() and (room[at + size:] == 0x5a).all()
    assert all(torch.equal(o, got[0][0]) and torch.equal(x, got[0][1]) for o, x in got[1:])
    assert not (got[0][0] == 7).any() and c.status.item() == 0
