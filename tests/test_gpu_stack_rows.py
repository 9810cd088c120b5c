"""The expert stack's rows of no request: what a pass gives for them follows from its own
inputs, not from the batches that were served before."""
import pytest
import torch

import synth
from tests.test_gpu_attention_stack import HIDDEN, _stack

pytestmark = pytest.mark.gpu


def _batch(rows, keys, table):
    i = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    return i(starts), i(keys), table.cuda()


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("how", ["forward", "blocks", "attend"])
def test_short_batch_after_a_full_one(how, dt):
    table = torch.arange(40, dtype=torch.int32).reshape(2, 20).contiguous()
    used, fresh = (_stack(60, 2, 20, 41, dt) for _ in range(2))
    ids = torch.randint(-1, 5, (60,), generator=torch.Generator().manual_seed(3)).int().cuda()
    x = synth.normal((60, HIDDEN), dt, 9800).cuda()
    used.forward(synth.normal((60, HIDDEN), dt, 9801).cuda(), ids,
                 batch=_batch([30, 30], [40, 30], table))
    assert used.o.any(2).any(1).all()
    fresh.k_cache.copy_(used.k_cache)
    fresh.v_cache.copy_(used.v_cache)
    short = _batch([1, 6], [100, 70], table)
    got = []
    for s in (used, fresh):
        if how == "forward":
            s.forward(x, ids, batch=short)
        else:
            s.n.copy_(x)
            s.r.copy_(x)
            for b in range(2):
                (s.run_block if how == "blocks" else s.attend)(b, ids, batch=short)
        got.append([t.clone() for t in (s.o, s.r, s.n, s.k_cache, s.v_cache)])
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert not got[0][0][7:].any()


def test_on_another_stream():
    """The rows are cleared in the stream that the pass was given."""
    table = torch.arange(40, dtype=torch.int32).reshape(2, 20).contiguous()
    s = _stack(60, 2, 20, 41, "bf16")
    ids = torch.zeros(60, dtype=torch.int32).cuda()
    x = synth.normal((60, HIDDEN), "bf16", 9802).cuda()
    full, short = _batch([30, 30], [40, 30], table), _batch([1, 6], [100, 70], table)
    s.forward(x, ids, batch=full)      # (its keys are in the cache of every short pass)
    s.forward(x, ids, batch=short)
    want = s.n.clone()
    other = torch.cuda.Stream()
    for stream in (other, other.cuda_stream):
        torch.cuda.synchronize()
        for _ in range(3):
            s.forward(x, ids, stream=stream, batch=full)
        s.forward(x, ids, stream=stream, batch=short)
        torch.cuda.synchronize()
        assert not s.o[7:].any() and torch.equal(s.n, want)


def test_the_default_stream_by_its_handle():
    """Handle 0, with another stream current that is busy: the rows are cleared in order."""
    s = _stack(60, 2, 20, 41, "bf16")
    s.o.fill_(1.0)
    busy = torch.zeros(1 << 27, device="cuda")
    before = torch.empty_like(s.o)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        busy.add_(1.0)
    before.copy_(s.o)                  # (behind the busy kernels of the default stream)
    with torch.cuda.stream(other):
        s._clear(0)
    torch.cuda.synchronize()
    assert not s.o.any() and (before == 1.0).all()


def test_captured():
    table = torch.arange(40, dtype=torch.int32).reshape(2, 20).contiguous()
    s = _stack(60, 2, 20, 41, "bf16")
    ids = torch.zeros(60, dtype=torch.int32).cuda()
    x = synth.normal((60, HIDDEN), "bf16", 9803).cuda()
    starts, lens, pages = _batch([30, 30], [40, 30], table)
    s.forward(x, ids, batch=(starts, lens, pages))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.forward(x, ids, batch=(starts, lens, pages))
    for rows, keys in (([30, 30], [40, 30]), ([1, 6], [100, 70]), ([20, 0], [140, 3]),
                       ([0, 2], [9, 9])):
        b = _batch(rows, keys, table)
        starts.copy_(b[0])
        lens.copy_(b[1])
        caches = s.k_cache.clone(), s.v_cache.clone()
        g.replay()
        torch.cuda.synchronize()
        replayed = s.n.clone()
        assert not s.o[sum(rows):].any()
        s.k_cache.copy_(caches[0])
        s.v_cache.copy_(caches[1])
        assert torch.equal(replayed, s.forward(x, ids, batch=(starts, lens, pages)))
        torch.cuda.synchronize()
