"""What the transformer-block calls refuse, before any device work (no GPU
needed: the pointers here are never read)."""
import ctypes

import pytest
import torch

from paper_2511_19457_amd import abi

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P, ODD = 0x10000, 0x10008            # aligned to 16 bytes, and not
BIG = 1 << 40


def test_status_codes():
    assert "invalid" in abi.sparoa_status_string(INVALID)
    assert "unsupported" in abi.sparoa_status_string(UNSUPPORTED)


def _route(ptrs=None, ws=BIG, **kw):
    d = dict(tokens=8, experts=16, top_k=4, groups=1, top_groups=1, group_best=1, dtype=abi.BF16,
             score=abi.SCORE_SOFTMAX, renormalise=1, scale=1.0)
    d.update(kw)
    p = dict(logits=P, bias=None, mask=None, idx=P, weights=P, plan=P, ws=P)
    p.update(ptrs or {})
    return abi._L.sparoa_expert_route(ctypes.byref(abi.ExpertRouteDesc(**d)), *p.values(), ws, None)


@pytest.mark.parametrize("status,args", [
    (INVALID, dict(tokens=0)), (INVALID, dict(experts=0)), (INVALID, dict(top_k=0)),
    (INVALID, dict(tokens=-1)), (INVALID, dict(top_k=17)), (INVALID, dict(groups=3)),
    (INVALID, dict(groups=0)), (INVALID, dict(groups=4, top_groups=5)),
    (INVALID, dict(groups=4, top_groups=0)), (INVALID, dict(groups=4, top_groups=1, top_k=5)),
    (INVALID, dict(group_best=3)), (INVALID, dict(score=2)), (INVALID, dict(dtype=9)),
    (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))),
    (UNSUPPORTED, dict(experts=513)), (UNSUPPORTED, dict(experts=64, top_k=33)),
    (UNSUPPORTED, dict(experts=130, groups=65, top_groups=65)),
    (UNSUPPORTED, dict(tokens=(1 << 28) + 1)),
    (INVALID, dict(ptrs=dict(logits=None))), (INVALID, dict(ptrs=dict(idx=None))),
    (INVALID, dict(ptrs=dict(weights=None))), (UNSUPPORTED, dict(ptrs=dict(logits=ODD))),
    (UNSUPPORTED, dict(ptrs=dict(plan=ODD))), (WORKSPACE, dict(ws=16)),
    (WORKSPACE, dict(ptrs=dict(ws=None)))])
def test_route(status, args):
    assert _route(**args) == status and abi.sparoa_last_error()


@pytest.mark.parametrize("status,args", [
    (INVALID, (0, 4, 16, P, P, P, BIG)), (INVALID, (8, 0, 16, P, P, P, BIG)),
    (INVALID, (8, 4, 0, P, P, P, BIG)), (UNSUPPORTED, (8, 4, 600, P, P, P, BIG)),
    (INVALID, (8, 4, 16, None, P, P, BIG)), (INVALID, (8, 4, 16, P, None, P, BIG)),
    (UNSUPPORTED, (8, 4, 16, ODD, P, P, BIG)), (WORKSPACE, (8, 4, 16, P, P, P, 8)),
    (WORKSPACE, (8, 4, 16, P, P, None, BIG))])
def test_plan(status, args):
    assert abi._L.sparoa_expert_plan(*args, None) == status


def _ffn(ptrs=None, ws=BIG, act=abi.ACT_SILU, **kw):
    d = dict(tokens=8, top_k=2, experts=4, hidden=64, inner=32, dtype=abi.BF16, gated=1, has_bias=0)
    d.update(kw)
    p = dict(x=P, w_up=P, b_up=None, w_down=P, b_down=None, weights=P, plan=P, residual=None, y=P,
             ws=P)
    p.update(ptrs or {})
    return abi._L.sparoa_expert_ffn(ctypes.byref(abi.ExpertFfnDesc(**d)), act, *p.values(), ws,
                                    None)


@pytest.mark.parametrize("status,args", [
    (INVALID, dict(tokens=0)), (INVALID, dict(hidden=0)), (INVALID, dict(inner=-4)),
    (INVALID, dict(dtype=3)), (INVALID, dict(act=5)), (INVALID, dict(act=-1)),
    (INVALID, dict(has_bias=1)), (INVALID, dict(ptrs=dict(b_up=P))),
    (INVALID, dict(ptrs=dict(x=None))), (INVALID, dict(ptrs=dict(plan=None))),
    (INVALID, dict(ptrs=dict(y=None))), (INVALID, dict(ptrs=dict(weights=None))),
    (UNSUPPORTED, dict(ptrs=dict(w_down=ODD))), (UNSUPPORTED, dict(ptrs=dict(residual=ODD))),
    (UNSUPPORTED, dict(experts=513)), (UNSUPPORTED, dict(tokens=1 << 24)),
    (UNSUPPORTED, dict(inner=1 << 24)), (UNSUPPORTED, dict(hidden=1 << 40)),
    (WORKSPACE, dict(ws=64)), (WORKSPACE, dict(ptrs=dict(ws=None)))])
def test_ffn(status, args):
    assert _ffn(**args) == status


def _adapted(ptrs=None, ws=BIG, act=abi.ACT_NONE, **kw):
    d = dict(m=8, k=64, n=32, adapters=3, rank=8, dtype=abi.BF16, has_bias=0)
    d.update(kw)
    p = dict(x=P, w=P, bias=None, a=P, b=P, scale=P, ids=P, residual=None, y=P, ws=P)
    p.update(ptrs or {})
    return abi._L.sparoa_fc_adapted(ctypes.byref(abi.FcAdaptedDesc(**d)), act, *p.values(), ws,
                                    None)


@pytest.mark.parametrize("status,args", [
    (INVALID, dict(m=0)), (INVALID, dict(k=0)), (INVALID, dict(n=-1)), (INVALID, dict(adapters=0)),
    (INVALID, dict(rank=0)), (INVALID, dict(dtype=7)), (INVALID, dict(act=abi.ACT_SILU)),
    (INVALID, dict(has_bias=1)), (INVALID, dict(ptrs=dict(bias=P))),
    (INVALID, dict(ptrs=dict(ids=None))), (INVALID, dict(ptrs=dict(scale=None))),
    (INVALID, dict(ptrs=dict(a=None))), (UNSUPPORTED, dict(rank=513)),
    (UNSUPPORTED, dict(ptrs=dict(x=ODD))), (UNSUPPORTED, dict(n=1 << 26)),
    (UNSUPPORTED, dict(k=1 << 45)), (INVALID, dict(m=1 << 60)),
    (WORKSPACE, dict(ws=64)), (WORKSPACE, dict(ptrs=dict(ws=None)))])
def test_adapted(status, args):
    assert _adapted(**args) == status


def _norm(ptrs=None, **kw):
    d = dict(rows=4, cols=64, gate_rows=4, dtype=abi.BF16, post=abi.NORM_RMS, pre=abi.NORM_RMS,
             eps=1e-6, residual_scale=1.0)
    d.update(kw)
    p = dict(y=P, post_w=P, post_b=None, gate=None, r=P, pre_w=P, pre_b=None, r_out=P, n_out=P)
    p.update(ptrs or {})
    return abi._L.sparoa_block_norm(ctypes.byref(abi.BlockNormDesc(**d)), *p.values(), None)


@pytest.mark.parametrize("status,args", [
    (INVALID, dict(rows=0)), (INVALID, dict(cols=0)), (INVALID, dict(gate_rows=0)),
    (INVALID, dict(post=3)), (INVALID, dict(pre=-1)), (INVALID, dict(dtype=4)),
    (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=float("nan"))),
    (INVALID, dict(residual_scale=float("inf"))), (INVALID, dict(ptrs=dict(y=None, r=None))),
    (INVALID, dict(ptrs=dict(n_out=None))), (INVALID, dict(pre=0, ptrs=dict(r_out=None))),
    (UNSUPPORTED, dict(ptrs=dict(y=ODD))), (UNSUPPORTED, dict(rows=1, cols=1 << 31)),
    (INVALID, dict(rows=1 << 40, cols=1 << 40))])
def test_norm(status, args):
    assert _norm(**args) == status


def test_other_calls_refuse_the_experts_activations():
    fd = abi.fc_desc(4, 64, 32, abi.BF16)
    for act in (abi.ACT_SILU, abi.ACT_GELU):
        assert abi._L.sparoa_fc_dense(ctypes.byref(fd), P, P, None, None, act, P, P, BIG,
                                      None) == INVALID


def test_the_binding_refuses_other_tensors():
    """Host tensors, strides, types and sizes that a kernel would read past."""
    d = abi.block_norm_desc(4, 64, torch.bfloat16, post=abi.NORM_NONE)
    good = torch.zeros(4, 64, dtype=torch.bfloat16)
    for bad in (good, good.float(), good[:2], torch.zeros(64, 4, dtype=torch.bfloat16).t()):
        with pytest.raises(abi.SparoaError):
            abi.sparoa_block_norm(d, bad, None, None, None, None, None, None, None, good)


def test_null_descriptors_and_results():
    L = abi._L
    n = ctypes.c_size_t()
    for fn in (L.sparoa_expert_route_workspace_size, L.sparoa_expert_ffn_workspace_size,
               L.sparoa_fc_adapted_workspace_size):
        assert fn(None, ctypes.byref(n)) == INVALID
    assert L.sparoa_expert_plan_words(8, 2, 4, None) == INVALID
    assert L.sparoa_block_norm(None, *[P] * 9, None) == INVALID
