"""An adapter whose matrices hold infinities or NaN spoils the rows that name
it and no others, whatever rows share its tile (sparoa_fc_adapted)."""
import numpy as np
import pytest
import torch

import synth
from tests.test_gpu_fc_adapted import DT, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("where", ["a", "b", "both"])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,k,n,rank", [(3, 96, 40, 8), (40, 256, 136, 16), (90, 101, 72, 8),
                                        (300, 512, 520, 4), (700, 256, 384, 40),
                                        (2500, 128, 2104, 24)])
def test_other_rows_keep_their_results(dt, where, m, k, n, rank):
    from paper_2511_19457_amd import abi
    dev, adapters = torch.device("cuda"), 4
    x, w = synth.normal((m, k), dt, 9800), synth.normal((n, k), dt, 9801, std=k ** -0.5)
    a = synth.normal((adapters, rank, k), dt, 9802, std=k ** -0.5)
    b = synth.normal((adapters, n, rank), dt, 9803, std=0.7)
    scale = np.ones(adapters, np.float32)
    ids = (np.arange(m) % 5 - 1).astype(np.int32)       # -1: no adapter
    bad = ids == 2
    ref, err = reference(x, w, None, a, b, scale, np.where(bad, -1, ids), None, 0, dt)
    if where != "b":
        a[2, 0, 1], a[2, rank - 1, k - 1] = float("inf"), float("nan")
    if where != "a":
        b[2, n - 1, rank - 1], b[2, 0, 0], b[2, :, rank // 2] = float("-inf"), float("nan"), \
            float("inf")
    x[m - 1, 0] = float("nan")                          # and a row of its own
    keep = ~bad
    keep[m - 1] = False
    d = abi.fc_adapted_desc(m, k, n, adapters, rank, DT[dt])
    ws = torch.full((abi.sparoa_fc_adapted_workspace_size(d),), 255, dtype=torch.uint8, device=dev)
    y = torch.zeros(m, n, dtype=DT[dt], device=dev)
    abi.sparoa_fc_adapted(d, abi.ACT_NONE, x.to(dev), w.to(dev), None, a.to(dev), b.to(dev),
                          torch.from_numpy(scale).to(dev), torch.from_numpy(ids).to(dev), None, y,
                          ws)
    got = y.double().cpu().numpy()
    off = ~(np.abs(got[keep] - ref[keep]) <= err[keep])
    assert not off.any(), (int(off.sum()), np.argwhere(off)[:4].tolist())
    assert not np.isfinite(got[m - 1]).any()
    if where != "a":
        assert not np.isfinite(got[bad][:, [0, n - 1]]).any()
    else:
        assert not np.isfinite(got[bad]).any()
