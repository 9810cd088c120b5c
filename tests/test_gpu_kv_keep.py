"""sparoa_kv_keep against indexing: any order and repeats of kept drafts, entries that
move nothing, several layers, pages of every size, requests left out.  It copies, so
bits are equal."""
import pytest
import torch

from tests._cache import DT, Batch

pytestmark = pytest.mark.gpu


def _abi():
    from paper_2511_19457_amd import abi
    return abi


def case(b, keep, layers=1, table=None, kept=None, left_out=(), **desc):
    abi = _abi()
    most = max(1, max(len(k) for k in keep))
    g = torch.Generator().manual_seed(3)
    kc = torch.randn(layers, *b.k.shape, generator=g).to(DT[b.dt])
    vc = torch.randn(layers, *b.k.shape, generator=g).to(DT[b.dt])
    kc[0, 0, 0, 0, 0] = float("nan")
    starts, lens, own = b.gpu()
    table = b.table if table is None else table
    idx = b.ints([k + [-5] * (most - len(k)) for k in keep])
    n_kept = b.ints([len(k) for k in keep] if kept is None else kept)
    on_k, on_v = kc.cuda(), vc.cuda()
    abi.sparoa_kv_keep(b.desc(abi, **desc), layers, starts, lens, table.cuda(), idx, n_kept, on_k,
                       on_v)
    torch.cuda.synchronize()
    for got, cache in ((on_k, kc), (on_v, vc)):
        want = cache.clone()
        for r, k in enumerate(keep):
            base = b.keys[r] - b.rows[r]
            if r in left_out or len(k) > b.rows[r]:
                continue
            for j, i in enumerate(k):
                if not 0 <= i < b.rows[r]:
                    continue
                src, dst = base + i, base + j
                ps, pd = int(table[r, src // b.page]), int(table[r, dst // b.page])
                if 0 <= ps < b.pages and 0 <= pd < b.pages:
                    want[:, pd, :, dst % b.page] = cache[:, ps, :, src % b.page]
        bits = torch.int16 if b.dt != "f32" else torch.int32
        assert torch.equal(got.cpu().view(bits), want.view(bits))


TYPES = ["bf16", "f16", "f32"]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("dim,page,layers", [(128, 16, 1), (64, 1, 3), (80, 25, 2), (8, 7, 1),
                                             (256, 64, 5)])
def test_shapes(dim, page, layers, dt):
    b = Batch([26, 1, 60, 0], [126, 1, 70, 33], 4, 2, dim, page, dt, seed=dim)
    case(b, [[0, 2, 5, 25], [0], [0, 1, 2, 3, 40, 59], []], layers)


def test_any_order():
    """Everything is read before anything is written."""
    b = Batch([8, 200, 256], [20, 333, 256], 2, 2, 128, 16, "bf16", seed=1)
    case(b, [[3, 2, 1, 0, 0, 7], list(range(199, -1, -1)), list(range(1, 256)) + [0]])
    case(Batch([256], [300], 1, 1, 256, 16, "f32", seed=2), [list(range(255, -1, -1))], 2)


def test_entries_that_move_nothing():
    b = Batch([8, 8], [20, 10], 2, 2, 64, 16, "f16", seed=3)
    case(b, [[-1, 8, 2 ** 31 - 1, 7], [-2 ** 31, 0]])


def test_requests_left_out():
    b = Batch([4, 5, 6], [40, 50, 60], 2, 1, 64, 16, "bf16", seed=4)
    keep = [[1, 3], [1, 4], [2, 5]]
    case(b, keep, left_out=(2,), max_queries=5)
    case(b, keep, left_out=(1, 2), max_keys=49)
    case(b, keep, kept=[3, 2, 2], left_out=(0,))        # above `most`
    case(b, keep, kept=[-1, 2, 0], left_out=(0, 2))
    case(b, [[0, 1, 2, 3, 0, 1], [4], [5]])             # more than its nodes


def test_pages_that_are_none():
    b = Batch([40], [60], 2, 2, 64, 16, "bf16", seed=5)
    t = b.table.clone()
    t[0, 2] = -1
    case(b, [[0, 30, 31, 5, 6, 7, 8, 9, 10, 11, 12, 13, 39]], table=t)


def test_many_requests():
    b = Batch([3] * 300, [3 + r % 9 for r in range(300)], 2, 2, 16, 4, "f32", seed=6)
    case(b, [[0, 2] if r % 3 else [2] for r in range(300)], 2)
