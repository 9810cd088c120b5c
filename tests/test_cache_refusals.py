"""What the attention calls refuse, before any device work (no GPU needed: the
pointers here are never read)."""
import ctypes

import pytest
import torch

from paper_2511_19457_amd import abi

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P, ODD = 0x10000, 0x10008            # aligned to 16 bytes, and not
BIG = 1 << 44
NAN, INF = float("nan"), float("inf")


def _desc(**kw):
    d = dict(tokens=8, requests=2, heads=8, kv_heads=2, head_dim=64, pages=20, page_size=16,
             table_pages=10, max_queries=8, max_keys=160, dtype=abi.BF16)
    d.update(kw)
    return abi.KvDesc(**d)


# what every call refuses of a descriptor
DESCS = [(INVALID, {k: v}) for k in ("tokens", "requests", "heads", "kv_heads", "head_dim", "pages",
                                    "page_size", "table_pages", "max_queries", "max_keys")
         for v in (0, -1)] + [
    (INVALID, dict(heads=7)), (INVALID, dict(kv_heads=16)), (INVALID, dict(max_keys=161)),
    (INVALID, dict(dtype=3)), (INVALID, dict(dtype=-1)), (UNSUPPORTED, dict(head_dim=12)),
    (UNSUPPORTED, dict(head_dim=264)), (UNSUPPORTED, dict(tokens=1 << 28)),
    (UNSUPPORTED, dict(tokens=1 << 40)), (UNSUPPORTED, dict(requests=1 << 31, table_pages=1)),
    (UNSUPPORTED, dict(requests=1 << 28)), (UNSUPPORTED, dict(pages=1 << 26)),
    (UNSUPPORTED, dict(pages=1 << 62)), (UNSUPPORTED, dict(page_size=1 << 40, pages=1)),
    (UNSUPPORTED, dict(page_size=1 << 20, table_pages=1 << 20, pages=1, max_keys=(1 << 31) - 1))]


def _append(ptrs=None, rot=64, strides=(512, 128, 128), **kw):
    p = dict(q=P, k=P, v=P, freqs=P, positions=None, q_start=P, kv_len=P, table=P, q_out=P * 2, kc=P,
             vc=P)
    p.update(ptrs or {})
    return abi._L.sparoa_kv_append(
        ctypes.byref(_desc(**kw)), rot, 0, p["q"], strides[0], p["k"], strides[1], p["v"],
        strides[2], p["freqs"], p["positions"], p["q_start"], p["kv_len"], p["table"], p["q_out"],
        p["kc"], p["vc"], None)


def _attend(ptrs=None, ws=BIG, opts=None, **kw):
    o = abi.AttentionOpts(**dict(dict(scale=0.125, cap=0.0, window=0, causal=1), **(opts or {})))
    p = dict(q=P, kc=P, vc=P, q_start=P, kv_len=P, table=P, prefix=None, first=None, slopes=None,
             out=P, ws=P)
    p.update(ptrs or {})
    return abi._L.sparoa_paged_attention(ctypes.byref(_desc(**kw)), ctypes.byref(o), *p.values(),
                                         ws, None)


def _tree(ptrs=None, ws=BIG, opts=None, **kw):
    o = abi.AttentionOpts(**dict(dict(scale=0.125, cap=0.0, window=0, causal=1), **(opts or {})))
    p = dict(q=P, kc=P, vc=P, q_start=P, kv_len=P, table=P, mask=P, positions=None, slopes=None,
             out=P, ws=P)
    p.update(ptrs or {})
    return abi._L.sparoa_tree_attention(ctypes.byref(_desc(**kw)), ctypes.byref(o), *p.values(), ws,
                                        None)


def _keep(ptrs=None, layers=1, most=4, **kw):
    p = dict(q_start=P, kv_len=P, table=P, keep=P, kept=P, kc=P, vc=P)
    p.update(ptrs or {})
    return abi._L.sparoa_kv_keep(ctypes.byref(_desc(**kw)), layers, p["q_start"], p["kv_len"],
                                 p["table"], p["keep"], most, p["kept"], p["kc"], p["vc"], None)


@pytest.mark.parametrize("call", [_append, _attend, _tree, _keep])
@pytest.mark.parametrize("status,desc", DESCS)
def test_descriptors(status, desc, call):
    assert call(**desc) == status and abi.sparoa_last_error()


@pytest.mark.parametrize("status,args", [
    (INVALID, dict(rot=63)), (INVALID, dict(rot=66)), (INVALID, dict(rot=-2)),
    (INVALID, dict(rot=0)), (INVALID, dict(ptrs=dict(freqs=None))),
    (INVALID, dict(ptrs=dict(q=None))), (INVALID, dict(ptrs=dict(q_out=None))),
    (INVALID, dict(ptrs=dict(k=None))), (INVALID, dict(ptrs=dict(v=None))),
    (INVALID, dict(ptrs=dict(q_start=None))), (INVALID, dict(ptrs=dict(kv_len=None))),
    (INVALID, dict(ptrs=dict(table=None))), (INVALID, dict(ptrs=dict(kc=None))),
    (INVALID, dict(ptrs=dict(vc=None))), (INVALID, dict(strides=(511, 128, 128))),
    (INVALID, dict(strides=(512, 127, 128))), (INVALID, dict(strides=(512, 128, -128))),
    (INVALID, dict(strides=(768, 768, 768), ptrs=dict(q_out=P))),
    (INVALID, dict(strides=(1 << 61, 128, 128))),
    (UNSUPPORTED, dict(ptrs=dict(k=ODD))), (UNSUPPORTED, dict(ptrs=dict(positions=ODD))),
    (UNSUPPORTED, dict(ptrs=dict(vc=ODD))), (UNSUPPORTED, dict(ptrs=dict(freqs=ODD)))])
def test_append(status, args):
    assert _append(**args) == status and abi.sparoa_last_error()


OPTS = [(INVALID, dict(opts=dict(scale=s))) for s in (0.0, -1.0, NAN, INF,
                                                        2.0 ** -61, 2.0 ** 61)] + [
    (INVALID, dict(opts=dict(cap=c))) for c in (-1.0, NAN, INF, 2.0 ** -61, 2.0 ** 61)] + [
    (INVALID, dict(opts=dict(window=-1))), (WORKSPACE, dict(ws=0)),
    (WORKSPACE, dict(ptrs=dict(ws=None))), (UNSUPPORTED, dict(ptrs=dict(ws=ODD)))] + [
    (INVALID, dict(ptrs={k: None})) for k in ("q", "kc", "vc", "q_start", "kv_len", "table",
                                              "out")] + [
    (UNSUPPORTED, dict(ptrs={k: ODD})) for k in ("q", "kc", "vc", "q_start", "kv_len", "table",
                                                 "out")]


@pytest.mark.parametrize("status,args", OPTS + [
    (UNSUPPORTED, dict(ptrs=dict(prefix=ODD))), (UNSUPPORTED, dict(ptrs=dict(first=ODD))),
    (UNSUPPORTED, dict(ptrs=dict(slopes=ODD)))])
def test_attention(status, args):
    assert _attend(**args) == status and abi.sparoa_last_error()


@pytest.mark.parametrize("status,args", OPTS + [
    (INVALID, dict(ptrs=dict(mask=None))), (INVALID, dict(ptrs=dict(slopes=P))),
    (INVALID, dict(opts=dict(window=4))), (UNSUPPORTED, dict(max_queries=257)),
    (UNSUPPORTED, dict(ptrs=dict(mask=ODD))), (UNSUPPORTED, dict(ptrs=dict(positions=ODD))),
    (UNSUPPORTED, dict(ptrs=dict(slopes=ODD, positions=P)))])
def test_tree(status, args):
    assert _tree(**args) == status and abi.sparoa_last_error()


@pytest.mark.parametrize("status,args", [
    (INVALID, dict(layers=0)), (INVALID, dict(layers=-1)), (INVALID, dict(most=0)),
    (UNSUPPORTED, dict(most=257)), (UNSUPPORTED, dict(layers=65536))] + [
    (INVALID, dict(ptrs={k: None})) for k in ("q_start", "kv_len", "table", "keep", "kept", "kc",
                                              "vc")] + [
    (UNSUPPORTED, dict(ptrs={k: ODD})) for k in ("q_start", "keep", "kept", "kc", "vc")])
def test_keep(status, args):
    assert _keep(**args) == status and abi.sparoa_last_error()


def test_null_descriptors_and_results():
    L, n = abi._L, ctypes.c_size_t()
    o = abi.attention_opts(1.0)
    d = _desc()
    assert L.sparoa_attention_workspace_size(None, ctypes.byref(n)) == INVALID
    assert L.sparoa_attention_workspace_size(ctypes.byref(d), None) == INVALID
    assert L.sparoa_paged_attention(None, ctypes.byref(o), *[P] * 11, BIG, None) == INVALID
    assert L.sparoa_paged_attention(ctypes.byref(d), None, *[P] * 11, BIG, None) == INVALID
    assert L.sparoa_tree_attention(None, ctypes.byref(o), *[P] * 11, BIG, None) == INVALID
    assert L.sparoa_tree_attention(ctypes.byref(d), None, *[P] * 11, BIG, None) == INVALID
    assert L.sparoa_kv_keep(None, 1, P, P, P, P, 4, P, P, P, None) == INVALID
    assert L.sparoa_kv_append(None, 0, 0, *[P, 512] * 3, *[P] * 9, None) == INVALID


@pytest.mark.parametrize("kw", [{}, dict(max_queries=1), dict(tokens=100000, requests=300),
                                dict(table_pages=100000, max_keys=1600000, pages=200000),
                                dict(head_dim=256, dtype=abi.F32)])
def test_workspace(kw):
    """A byte less than what is asked for is refused, for trees, too."""
    size = abi.sparoa_attention_workspace_size(_desc(**kw))
    assert size > 0
    assert _attend(ws=size - 1, **kw) == WORKSPACE and _tree(ws=size - 1, **kw) == WORKSPACE


def test_the_binding_refuses_other_tensors():
    """Host tensors, strides, types and sizes that a kernel would read past."""
    d = abi.kv_desc(4, 1, 2, 1, 64, 3, 16, 2, torch.bfloat16)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    q, kv = torch.zeros(4, 128).bfloat16(), torch.zeros(4, 64).bfloat16()
    cache, o = torch.zeros(3, 1, 16, 64).bfloat16(), abi.attention_opts(1.0)
    with pytest.raises(abi.SparoaError):     # (host tensors)
        abi.sparoa_kv_append(d, q, kv, kv, None, None, i32(2), i32(1), i32(2), q, cache, cache)
    with pytest.raises(abi.SparoaError):
        abi.sparoa_paged_attention(d, o, q, cache, cache, i32(2), i32(1), i32(2), None, None, None,
                                   q, None)
    with pytest.raises(abi.SparoaError):
        abi.sparoa_tree_attention(d, o, q, cache, cache, i32(2), i32(1), i32(2), i32(4), None, None,
                                  q, None)
    with pytest.raises(abi.SparoaError):
        abi.sparoa_kv_keep(d, 1, i32(2), i32(1), i32(2), i32(4), i32(1), cache, cache)
    for bad in (q.float(), q[:3], q.t(), q[:, ::2], torch.zeros(128).bfloat16()):
        with pytest.raises(abi.SparoaError):
            abi._rows(bad, torch.bfloat16, 4, 128, "q", 0)


def test_a_changed_descriptor_is_asked_anew():
    d = abi.kv_desc(4, 2, 8, 2, 64, 3, 16, 2, torch.bfloat16)
    assert d.of()[1:7] == (4, 512, 128, 3 * 2 * 16 * 64, 2, 4) and d.of()[7] == 1
    d.tokens, d.pages, d.max_queries, d.dtype = 9, 5, 65, abi.F32
    assert d.of()[0] is torch.float32
    assert d.of()[1] == 9 and d.of()[4] == 5 * 2 * 16 * 64 and d.of()[7] == 2
