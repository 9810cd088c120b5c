"""The stack of expert blocks, block by block: every operator's output against
its formula in 64 bits on the bytes that the operator read (the choice of
experts is not continuous, so blocks are not compared end to end), then a
captured pass against a launched one."""
import numpy as np
import pytest
import torch

import oracle
import synth
from tests import test_gpu_block_norm as norm_test
from tests import test_gpu_expert_ffn as ffn_test
from tests import test_gpu_expert_route as route_test
from tests import test_gpu_fc_adapted as fc_test
from tests._util import RTOL, assert_close

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _stack(tokens, dt, blocks=2):
    from paper_2511_19457_amd.experts import ExpertStack
    return ExpertStack(tokens, 192, 96, 12, 3, blocks, 5, 8, DT[dt], seed=40, eps=norm_test.EPS)


def _inputs(tokens, dt, seed=0):
    g = np.random.default_rng(seed)
    x = synth.normal((tokens, 192), dt, 9900 + seed).cuda()
    ids = torch.from_numpy(g.integers(-1, 5, tokens).astype(np.int32)).cuda()
    mask = torch.from_numpy((g.random(tokens) < 0.8).astype(np.uint8)).cuda()
    return x, ids, mask


def _within(got, ref, err, what):
    bad = ~(np.abs(got.double().cpu().numpy() - ref) <= err)
    assert not bad.any(), (what, int(bad.sum()))


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens", [1, 37, 600])
def test_blocks(tokens, dt):
    s = _stack(tokens, dt)
    x, ids, mask = _inputs(tokens, dt)
    s.forward(x, ids, mask)
    total = s.n.clone()
    from paper_2511_19457_amd import abi
    abi.sparoa_block_norm(s.first, None, None, None, None, x, s.first_norm, None, s.r, s.n)
    for b, w in enumerate(s.blocks):
        r0, n0 = s.r.clone(), s.n.clone()
        s.run_block(b, ids, mask)
        ref, err = fc_test.reference(n0.cpu(), w["proj"].cpu(), None, w["lora_a"].cpu(),
                                     w["lora_b"].cpu(), np.ones(5, np.float32), ids.cpu().numpy(),
                                     None, 0, dt)
        _within(s.p, ref, err, "projection")
        # the first norm again, from p: r and n between the halves
        r1, n1 = torch.empty_like(r0), torch.empty_like(r0)
        abi.sparoa_block_norm(s.norm, s.p, w["norms"][0], None, w["gates"][0], r0, w["norms"][1],
                              None, r1, n1)
        ref, err, (nref, nerr) = norm_test._reference(
            s.p, w["norms"][0], None, w["gates"][0][None], tokens, r0, w["norms"][1], None, 1, 1, 1.0,
            tokens, 192)
        norm_test._check(r1, ref, err, dt, "r between the halves")
        norm_test._check(n1, nref, nerr, dt, "n between the halves")
        y, size = oracle.fc(n1.cpu(), w["router"].cpu(), tokens, 192, 12)
        assert_close(s.logits.cpu(), y, size, RTOL[DT[dt]], "router")
        # (equal logits aside, choices follow the logits' own order)
        ri, rw = route_test.reference(s.logits.double().cpu().numpy(), 3, 0, 1, 1, 1, None, True,
                                      1.0, mask.cpu().numpy())
        idx, weights = s.idx.cpu().numpy(), s.weights.cpu().numpy()
        assert np.array_equal(idx, ri)
        assert np.all(np.abs(weights - rw) <= route_test.RTOL * rw + 1e-37)
        route_test.check_plan(s.plan, idx, tokens, 3, 12)
        ref, err = ffn_test.reference(n1.cpu(), w["w_up"].cpu(), None, w["w_down"].cpu(), None,
                                      idx, weights, None, True, "silu", dt)
        _within(s.f, ref, err, "experts")
        assert not s.f[mask == 0].any()
        ref, err, (nref, nerr) = norm_test._reference(
            s.f, w["norms"][2], None, w["gates"][1][None], tokens, r1, w["norms"][3], None, 1, 1, 1.0,
            tokens, 192)
        norm_test._check(s.r, ref, err, dt, "r")
        norm_test._check(s.n, nref, nerr, dt, "n")
    assert torch.equal(total, s.n)


def test_captured_passes():
    s = _stack(48, "bf16", blocks=3)
    x, ids, mask = _inputs(48, "bf16")
    s.forward(x, ids, mask)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.forward(x, ids, mask)
    for rep in range(4):
        for t, new in zip((x, ids, mask), _inputs(48, "bf16", 1 + rep)):
            t.copy_(new)
        g.replay()
        torch.cuda.synchronize()
        replayed = s.n.clone()
        assert torch.equal(replayed, s.forward(x, ids, mask)) and torch.isfinite(replayed).all()
        torch.cuda.synchronize()


def test_refuses_other_inputs():
    s = _stack(8, "bf16", blocks=1)
    x, ids, mask = _inputs(8, "bf16")
    from paper_2511_19457_amd.abi import SparoaError
    with pytest.raises(ValueError):
        s.forward(x[:4], ids)
    with pytest.raises(ValueError):
        s.forward(x.float(), ids)
    with pytest.raises(SparoaError):
        s.forward(x, ids.long())
    with pytest.raises(SparoaError):
        s.forward(x, ids, mask.bool())
