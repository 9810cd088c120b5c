"""sparoa_kv_append with entries of q_start that break their bounds, among up to 5000
requests: the requests that the entry begins or ends are left out, every other one
is appended, whatever a search over the entries meets on its way."""
import pytest
import torch

from tests._cache import Batch
from tests.test_gpu_kv_append import case

pytestmark = pytest.mark.gpu


class Broken(Batch):
    """q_start with other entries than the rows' sums."""
    entries = {}

    def gpu(self):
        start = list(self.start)
        for i, v in self.entries.items():
            start[i] = v
        return self.ints(start), self.ints(self.keys), self.table.cuda()


def batch(rows, seed, **kw):
    g = torch.Generator().manual_seed(seed)
    keys = [n + int(e) for n, e in zip(rows, torch.randint(0, 5, (len(rows),), generator=g))]
    return Broken(rows, keys, 2, 1, 8, 4, "f32", seed=seed, spare=5, fill=3.0, **kw)


@pytest.mark.parametrize("requests", [64, 65, 300, 5000])
@pytest.mark.parametrize("live", [1, 3, 40])
def test_unused_entries_are_zero(live, requests):
    """Requests in front, the entries of the others never filled in."""
    b = batch([1 + i % 3 for i in range(live)] + [0] * (requests - live), requests + live)
    b.entries = {i: 0 for i in range(live + 1, requests + 1)}
    case(b, 8, False)


@pytest.mark.parametrize("requests", [64, 65, 300, 5000])
@pytest.mark.parametrize("value", [-3, 0, 2 ** 31 - 1, -2 ** 31])
def test_one_entry(value, requests):
    """An entry in the middle: below 0, back to 0 (a request of more rows than any may
    have), past the end."""
    for i in sorted({requests // 64 * 13, requests // 64 * 63, requests // 2 + 1, requests - 1}):
        g = torch.Generator().manual_seed(requests + i)
        rows = torch.randint(0, 3, (requests,), generator=g).tolist()
        rows[0], rows[i - 1], rows[i] = 1, 1, 1
        b = batch(rows, requests + i)
        b.entries = {i: value}
        case(b, 8, False, left_out=(i - 1, i))


@pytest.mark.parametrize("requests", [64, 65, 300])
def test_requests_that_break_other_bounds(requests):
    """More rows than max_queries, more keys than max_keys, fewer keys than rows, beside
    others that hold them."""
    rows = [4 if i in (7, 50) else 1 for i in range(requests)]
    b = batch(rows, requests)
    case(b, 8, False, left_out=(7, 50), max_queries=3)
    long = batch([1] * requests, requests)
    out = tuple(r for r in range(requests) if long.keys[r] > 4)
    assert 0 < len(out) < requests
    case(long, 8, False, left_out=out, max_keys=4)
