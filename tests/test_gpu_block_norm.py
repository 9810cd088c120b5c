"""The norm between two blocks (sparoa_block_norm) against its formula in
64-bit numpy: row lengths around every kernel's limits, norms, gates shared by
rows, missing operands, outputs in an input's place, rows that hold NaN or
infinity.

Tolerance: one rounding to the dtype (u = 2^-8, 2^-11, 2^-24) of the result,
and fp32 arithmetic: 100 roundings of 2^-24 on every term that is added, which
covers sums of up to 64 elements a thread, their joining over 1024 threads,
the root, the quotient and the products."""
import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -24, "f32": 2.0 ** -149}
F32 = 100 * 2.0 ** -24
EPS = 1e-5


def _abi():
    from paper_2511_19457_amd import abi
    return abi


def _norm(v, err, kind, w, b):
    """(normed v, its absolute error bound), err: that of v."""
    if kind == 0:
        return v, err
    mean = v.mean(1, keepdims=True) if kind == 2 else 0.0
    size = np.abs(v).max(1, keepdims=True)
    d = v - mean
    k = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + EPS)
    worst = err.max(1, keepdims=True)
    derr = err + (worst + F32 * size if kind == 2 else 0.0)
    # a shift e of the elements moves the deviation by at most e
    out, oerr = d * k, (derr + np.abs(d) * k * (worst + derr.max(1, keepdims=True))) * k
    oerr = oerr + F32 * np.abs(out)
    if w is not None:
        out, oerr = out * w, oerr * np.abs(w)
    if b is not None:
        out = out + b
        oerr = oerr + F32 * np.abs(b)
    return out, oerr + F32 * np.abs(out)


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _reference(y, pw, pb, gate, gate_rows, r, nw, nb, post, pre, c, rows, cols):
    v = np.zeros((rows, cols)) if y is None else _np(y)
    err = np.zeros_like(v)
    if y is not None:
        v, err = _norm(v, err, post, _np(pw) if post else None, _np(pb) if post else None)
    if gate is not None:
        g = _np(gate)[np.arange(rows) // gate_rows]
        v, err = v * g, err * np.abs(g) + F32 * np.abs(v * g)
    if r is not None:
        err = err + F32 * (np.abs(v) + np.abs(c * _np(r)))
        v = v + c * _np(r)
    return v, err, _norm(v, err, pre, _np(nw), _np(nb))


def _check(got, ref, err, dt, what):
    g = _np(got)
    bound = err * 1.01 + U[dt] * (np.abs(ref) + err) + TINY[dt]
    bad = ~(np.abs(g - ref) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(g - ref)[bad].max()),
                           float(bound[bad].min()))


def _run(rows, cols, dt, post, pre, gate_rows=None, c=1.0, has_y=True, has_r=True, affine=True,
         write_r=True, in_place=False, mean=0.0, seed=0, stream=None):
    abi, dev = _abi(), torch.device("cuda")
    mk = lambda shape, i, std=1.0: (synth.normal(shape, dt, 7000 + 10 * seed + i, std=std)
                                    .to(dev))
    y = mk((rows, cols), 0, 2.0) + mean if has_y else None
    r = mk((rows, cols), 1) if has_r else None
    y = None if y is None else y.to(synth.normal((1,), dt, 0).dtype).contiguous()
    gate = mk((-(-rows // gate_rows), cols), 2, 0.5) if gate_rows else None
    pw, nw = (mk((cols,), 3), mk((cols,), 4)) if affine else (None, None)
    pb, nb = (mk((cols,), 5, .1), mk((cols,), 6, .1)) if affine else (None, None)
    torch_dt = (y if y is not None else r).dtype
    ref, err, (nref, nerr) = _reference(y, pw, pb, gate, gate_rows, r, nw, nb, post, pre, c, rows,
                                        cols)
    r_out = torch.full((rows, cols), 7.0, dtype=torch_dt, device=dev) if write_r else None
    n_out = torch.full((rows, cols), 7.0, dtype=torch_dt, device=dev)
    if in_place:
        r_out, n_out = r, y
    d = abi.block_norm_desc(rows, cols, torch_dt, post=post, pre=pre, eps=EPS,
                            gate_rows=gate_rows, residual_scale=c)
    abi.sparoa_block_norm(d, y, pw, pb, gate, r, nw, nb, r_out, n_out if pre else None,
                          stream=stream)
    torch.cuda.synchronize()
    what = (rows, cols, dt, post, pre, gate_rows)
    if r_out is not None:
        _check(r_out, ref, err, dt, what + ("r",))
    if pre:
        _check(n_out, nref, nerr, dt, what + ("n",))
    return r_out, n_out


# row lengths: each kernel's longest and the next, odd and single ones
COLS = [1, 7, 8, 100, 512, 520, 1000, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384,
        16392, 20003, 65536, 65544]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cols", COLS)
def test_row_lengths(dt, cols):
    i = COLS.index(cols)
    _run(1 + i % 6, cols, dt, post=i % 3, pre=1 + (i + 1) % 2, gate_rows=1 + i % 3, c=0.5, seed=i)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", [(0, 0), (0, 1), (0, 2), (1, 0), (1, 1), (2, 2)])
@pytest.mark.parametrize("cols", [520, 72, 33])
def test_operands(dt, post, pre, cols):
    _run(9, cols, dt, post, pre, seed=50)
    _run(9, cols, dt, post, pre, gate_rows=4, affine=False, c=-2.0, seed=51)
    _run(9, cols, dt, post, pre, has_r=False, seed=52)
    if pre:
        _run(9, cols, dt, post, pre, has_y=False, write_r=False, seed=53)
    _run(9, cols, dt, post, max(pre, 1), gate_rows=9, in_place=True, seed=54)


@pytest.mark.parametrize("dt", ["f16", "f32"])
@pytest.mark.parametrize("cols", [256, 2048, 131])
def test_layer_norm_around_a_large_mean(dt, cols):
    _run(5, cols, dt, post=2, pre=2, mean=100.0, seed=60)


def test_many_rows():
    _run(70001, 64, "bf16", post=1, pre=1, gate_rows=1000, seed=61)


@pytest.mark.parametrize("cols", [40, 45, 3000])
def test_rows_with_nan_or_infinity_keep_to_themselves(cols):
    abi, dev = _abi(), torch.device("cuda")
    y = synth.normal((6, cols), "bf16", 7900).to(dev)
    r = synth.normal((6, cols), "bf16", 7901).to(dev)
    d = abi.block_norm_desc(6, cols, y.dtype, post=abi.NORM_RMS, pre=abi.NORM_LAYER, eps=EPS)
    clean_r, clean_n = torch.empty_like(r), torch.empty_like(r)
    abi.sparoa_block_norm(d, y, None, None, None, r, None, None, clean_r, clean_n)
    y[1, cols - 1], r[3, 0], y[5, cols // 2] = float("nan"), float("inf"), float("-inf")
    y[4] = 0
    r_out, n_out = torch.empty_like(r), torch.empty_like(r)
    abi.sparoa_block_norm(d, y, None, None, None, r, None, None, r_out, n_out)
    for i in (0, 2):
        assert torch.equal(r_out[i], clean_r[i]) and torch.equal(n_out[i], clean_n[i])
    assert torch.isnan(n_out[[1, 3, 5]]).any(1).all()
    assert torch.equal(r_out[4], r[4]) and torch.isfinite(n_out[4]).all()


def test_on_another_stream():
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        _run(64, 2048, "bf16", 1, 1, gate_rows=64, seed=62)
    _run(64, 2048, "bf16", 1, 1, gate_rows=64, seed=62, stream=s)
