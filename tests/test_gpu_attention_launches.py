"""An attention call of more work-groups than one launch takes."""
import pytest
import torch

from tests._cache import U

pytestmark = pytest.mark.gpu


def test_more_work_groups_than_a_launch_takes():
    """2^20 requests of one token, 8 heads of their own: 2^23 items and more.  Bound: a
    score of 8 exact-product terms is off by 24 roundings of 2^-24 of sum |q k| (4 at most
    here: values below 1), twice that a weight's, the weight rounded (u), sums of at most 16
    terms, the output u."""
    from paper_2511_19457_amd import abi
    n, heads, dim, pages = 1 << 20, 8, 8, 64
    g = torch.Generator("cuda").manual_seed(1)
    q = (2 * torch.rand(n + 3, heads, dim, generator=g, device="cuda") - 1).bfloat16()
    k, v = ((2 * torch.rand(pages, heads, 16, dim, generator=g, device="cuda") - 1).bfloat16()
            for _ in range(2))
    r = torch.arange(n, device="cuda")
    lens, table = (1 + r % 16).int(), (r * 7 % pages).int()
    starts = torch.arange(n + 1, device="cuda").int()
    d = abi.kv_desc(n + 3, n, heads, heads, dim, pages, 16, 1, torch.bfloat16, max_queries=1)
    ws = torch.empty(max(16, abi.sparoa_attention_workspace_size(d)), dtype=torch.uint8,
                     device="cuda")
    out = torch.full_like(q, 7.0)
    abi.sparoa_paged_attention(d, abi.attention_opts(1.0), q, k, v, starts, lens, table, None, None,
                               None, out, ws)
    torch.cuda.synchronize()
    assert (out[n:] == 7.0).all()
    seen = torch.arange(16, device="cuda")
    for a in range(0, n, 1 << 16):
        mine = slice(a, a + (1 << 16))
        keys, values = k[table[mine].long()].double(), v[table[mine].long()].double()
        x = (q[mine].double()[:, :, None] * keys).sum(3)
        x = torch.where(seen < lens[mine, None, None], x, -torch.inf)
        w = torch.softmax(x, 2)[..., None]
        want, size = (w * values).sum(2), (w * values.abs()).sum(2)
        tol = (2 * U["bf16"] + 2 * 24 * 8 * 2.0 ** -24 + 2.0 ** -18) * size + 1e-30
        assert ((out[mine].double() - want).abs() <= tol).all(), a
