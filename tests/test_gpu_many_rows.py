"""An adapted FC of more rows than one launch of its first product has threads for:
its rows are those of the same call over a part of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_adapted_of_2_to_the_27_rows_and_some():
    from paper_2511_19457_amd import abi
    dev, (m, k, n, adapters, rank) = torch.device("cuda"), ((1 << 27) + 37, 8, 8, 2, 16)
    g = torch.Generator(device=dev).manual_seed(1)
    rand = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)
    x, w, a, b = rand(m, k), rand(n, k), rand(adapters, rank, k), rand(adapters, n, rank)
    ids = torch.arange(m, device=dev, dtype=torch.int32) % 3 - 1
    scale = torch.ones(adapters, device=dev)

    def run(rows):
        d = abi.fc_adapted_desc(len(rows), k, n, adapters, rank, x.dtype)
        ws = torch.empty(abi.sparoa_fc_adapted_workspace_size(d), dtype=torch.uint8, device=dev)
        y = torch.full((len(rows), n), float("nan"), dtype=x.dtype, device=dev)
        abi.sparoa_fc_adapted(d, 0, x[rows.start:rows.stop], w, None, a, b, scale,
                              ids[rows.start:rows.stop], None, y, ws)
        return y

    y = run(range(m))
    part = 1 << 24
    for r0 in [0, part - 64, m // 2 // 64 * 64, (m - 40000) // 64 * 64]:
        rows = range(r0, min(r0 + 100000, m))
        assert torch.equal(y[rows.start:rows.stop], run(rows)), r0
    # and every row by the formula: one rounding of h (2^-8) and of y, sums of 8 and 16
    for r0 in range(0, m, part):
        r1 = min(r0 + part, m)
        xs, mine = x[r0:r1].float(), ids[r0:r1]
        want = xs @ w.float().t()
        slack = xs.abs() @ w.float().abs().t()
        for i in range(adapters):
            h = xs @ a[i].float().t()
            on = (mine == i).float()[:, None]
            want += on * (h @ b[i].float().t())
            slack += 512 * on * (h.abs() * 2.0 ** -8 @ b[i].float().abs().t())
        bad = ~((y[r0:r1].float() - want).abs() <= 2.0 ** -8 * want.abs() + slack / 512 + 1e-4)
        assert not bad.any(), (r0, int(bad.sum()))
