"""A prompt of two million tokens with a NaN in its last value: the rows of the last tile that do not see it are computed again, for longer than
any wait of the kernel lasts by itself, and nothing is given up for that."""
import pytest
import torch

from paper_2608_22643_b200 import binding as nb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,hd", [((1 << 21) - 37, 128), ((1 << 20) + (1 << 19), 64)])
def test_rows_that_take_seconds(n, hd):
    BF = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k = (torch.randn(n, 1, hd, generator=g, device="cuda", dtype=BF) for _ in range(2))
    # every token has the same values: a row's result is that value, whatever its weights are
    v = (torch.arange(hd, device="cuda") / 64 - 0.5).to(BF).expand(n, 1, hd).contiguous()
    cu, status = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n, 1, device="cuda")
    clean, clean_lse = torch.empty_like(q), torch.empty(n, 1, device="cuda")
    nb.np_attn_prompt(q, k, v, cu, clean, status, lse=clean_lse)
    v[-1] = float("nan")
    nb.np_attn_prompt(q, k, v, cu, out, status, lse=lse)
    assert nb.np_attn_check(status) == nb.NP_OK
    assert torch.isnan(out[-1]).all() and torch.equal(lse, clean_lse)
    first = (n - 1) // 128 * 128                      # of the last tile of keys
    assert torch.equal(out[:first], clean[:first])
    # the rows that were computed again: fp32 sums of n weights and of the same weights times one value, a lane's 8 tokens at a time: n / 8 steps of
    # the sum, n of the product's, each off by half a step of 2^-23 at most; a division of 2^-22, one rounding
    want = v[0, 0].double()
    tol = want.abs() * (2.0 ** -8 + (1 + 2.0 ** -8) * (n / 8 + n + 64) * 2.0 ** -24)
    assert ((out[first:-1, 0].double() - want).abs() <= tol).all()
