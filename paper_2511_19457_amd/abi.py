"""ctypes binding of libsparoa.so (argument marshalling only).

Every function carries the name of the C entry point it calls.  Device
tensors come from PyTorch (device memory and streams are PyTorch's); no
computation of the hot path happens here.  If the HIP library is missing the
import fails loudly: there is no fallback.
"""
import ctypes
import os
from dataclasses import dataclass

import torch  # must be imported before the library: both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparoa.so")

F32, F16, BF16 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_RELU6, ACT_SILU, ACT_GELU = 0, 1, 2, 3, 4
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
PATH_DENSE_MFMA, PATH_SKIP_MFMA, PATH_DENSE_BW, PATH_SKIP_BW = 0, 1, 2, 3
ROUTE_BLOCK, ROUTE_ELEMENT = 0, 1
PATH_NAMES = {0: "dense_mfma", 1: "skip_mfma", 2: "dense_bw", 3: "skip_bw"}
COMMIT_WORDS_BYTES = 2048   # SPAROA_COMMIT_WORDS_BYTES

_TORCH_DT = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_DT_TORCH = {code: dt for dt, code in _TORCH_DT.items()}

EXPORTS = [
    "sparoa_abi_version", "sparoa_status_string", "sparoa_last_error", "sparoa_mask_words",
    "sparoa_measure_sparsity", "sparoa_measure_sparsity_sync", "sparoa_op_intensity_conv",
    "sparoa_op_intensity_fc", "sparoa_route", "sparoa_conv2d_workspace_size",
    "sparoa_conv2d_skip_block", "sparoa_conv2d_tiling", "sparoa_conv2d", "sparoa_conv2d_dense",
    "sparoa_conv2d_zero_skip", "sparoa_fc_packed_bytes", "sparoa_fc_pack_weights",
    "sparoa_fc_tiling", "sparoa_fc_workspace_size", "sparoa_fc_skip_block", "sparoa_fc",
    "sparoa_fc_dense", "sparoa_fc_zero_skip", "sparoa_maxpool2d", "sparoa_conv2d_routed",
    "sparoa_fc_routed", "sparoa_fc_uses_packed", "sparoa_fc_ops_run",
    "sparoa_fc_measured", "sparoa_conv2d_routed_measured", "sparoa_fc_routed_measured",
    "sparoa_conv2d_split", "sparoa_fc_split", "sparoa_measure_sparsity_preset",
    "sparoa_conv2d_noalloc", "sparoa_conv2d_reads_mask", "sparoa_conv2d_routed_reads_mask",
    "sparoa_block_norm", "sparoa_expert_plan_words", "sparoa_expert_route_workspace_size",
    "sparoa_expert_route", "sparoa_expert_plan_workspace_size", "sparoa_expert_plan",
    "sparoa_expert_ffn_workspace_size", "sparoa_expert_ffn", "sparoa_fc_adapted_workspace_size",
    "sparoa_fc_adapted", "sparoa_kv_append", "sparoa_attention_workspace_size",
    "sparoa_paged_attention", "sparoa_tree_attention", "sparoa_kv_keep",
]


class SparoaError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"sparoa status {status}: {message}")
        self.status = status


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ("n", "c_in", "h", "w", "c_out", "kh", "kw", "sh", "sw", "ph", "pw", "dh", "dw",
                 "groups")] + [("dtype", ctypes.c_int), ("has_bias", ctypes.c_int)]


class FcDesc(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("k", ctypes.c_int64), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("has_bias", ctypes.c_int)]


class Counts(ctypes.Structure):
    _fields_ = [("zeros", ctypes.c_uint64), ("numel", ctypes.c_uint64),
                ("zero_blocks", ctypes.c_uint64), ("num_blocks", ctypes.c_uint64)]

    def as_dict(self):
        return dict(zeros=self.zeros, numel=self.numel, zero_blocks=self.zero_blocks,
                    num_blocks=self.num_blocks)


class Intensity(ctypes.Structure):
    _fields_ = [("macs", ctypes.c_uint64), ("flops", ctypes.c_uint64),
                ("bytes", ctypes.c_uint64), ("intensity", ctypes.c_double)]

    def as_dict(self):
        return dict(macs=self.macs, flops=self.flops, bytes=self.bytes, intensity=self.intensity)


class Thresholds(ctypes.Structure):
    _fields_ = [("sparsity_thr", ctypes.c_double), ("intensity_thr", ctypes.c_double),
                ("mode", ctypes.c_int)]


class FcOp(ctypes.Structure):
    _fields_ = [("desc", FcDesc), ("x", ctypes.c_void_p), ("w_nk", ctypes.c_void_p),
                ("w_packed", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("act", ctypes.c_int),
                ("counts", ctypes.c_void_p), ("mask", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t),
                ("path", ctypes.c_void_p), ("thr", Thresholds)]


class ExpertRouteDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("experts", ctypes.c_int64),
                ("top_k", ctypes.c_int64), ("groups", ctypes.c_int64),
                ("top_groups", ctypes.c_int64), ("group_best", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("score", ctypes.c_int), ("renormalise", ctypes.c_int),
                ("scale", ctypes.c_float)]


class ExpertFfnDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("top_k", ctypes.c_int64),
                ("experts", ctypes.c_int64), ("hidden", ctypes.c_int64),
                ("inner", ctypes.c_int64), ("dtype", ctypes.c_int), ("gated", ctypes.c_int),
                ("has_bias", ctypes.c_int)]


class FcAdaptedDesc(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("k", ctypes.c_int64), ("n", ctypes.c_int64),
                ("adapters", ctypes.c_int64), ("rank", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("has_bias", ctypes.c_int)]


class BlockNormDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("gate_rows", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("post", ctypes.c_int), ("pre", ctypes.c_int),
                ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float)]


class KvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ("tokens", "requests", "heads", "kv_heads", "head_dim", "pages", "page_size",
                 "table_pages", "max_queries", "max_keys")] + [("dtype", ctypes.c_int)]

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        self.__dict__.pop("_of", None)

    def of(self):
        """The tensors' sizes that follow from the fields (a field costs 70 ns to read, as
        much as a question to a tensor; kept until a field is set)."""
        got = self.__dict__.get("_of")
        if got is None:
            got = self.__dict__["_of"] = (
                _DT_TORCH.get(self.dtype), self.tokens, self.heads * self.head_dim,
                self.kv_heads * self.head_dim,
                self.pages * self.kv_heads * self.page_size * self.head_dim, self.requests,
                self.requests * self.table_pages, -(-self.max_queries // 64), self.heads,
                self.head_dim)
        return got


class AttentionOpts(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("window", ctypes.c_int64),
                ("causal", ctypes.c_int)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run __graft_entry__.build() "
                          "(python -c 'import __graft_entry__ as g; g.build()')")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    P = ctypes.POINTER
    sig = {
        "sparoa_abi_version": (ctypes.c_uint32, []),
        "sparoa_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "sparoa_last_error": (ctypes.c_char_p, []),
        "sparoa_mask_words": (ctypes.c_int, [i64, i64, i64, i64, P(i64)]),
        "sparoa_measure_sparsity": (ctypes.c_int, [vp, ctypes.c_int, i64, i64, i64, i64, i64, vp,
                                                   vp, vp, vp]),
        "sparoa_measure_sparsity_sync": (ctypes.c_int, [vp, ctypes.c_int, i64, i64, i64, i64, i64,
                                                        vp, vp, vp, P(Counts), vp]),
        "sparoa_op_intensity_conv": (ctypes.c_int, [P(ConvDesc), P(Intensity)]),
        "sparoa_op_intensity_fc": (ctypes.c_int, [P(FcDesc), P(Intensity)]),
        "sparoa_route": (ctypes.c_int, [P(Counts), P(Intensity), ctypes.c_int, P(Thresholds),
                                        P(ctypes.c_int)]),
        "sparoa_conv2d_workspace_size": (ctypes.c_int, [P(ConvDesc), ctypes.c_int, P(sz)]),
        "sparoa_conv2d_skip_block": (ctypes.c_int, [P(ConvDesc), ctypes.c_int, P(i64), P(i64)]),
        "sparoa_conv2d_tiling": (ctypes.c_int, [P(ConvDesc), ctypes.c_int, P(i64), P(i64)]),
        "sparoa_conv2d_reads_mask": (ctypes.c_int, [P(ConvDesc), ctypes.c_int, P(ctypes.c_int)]),
        "sparoa_conv2d_routed_reads_mask": (ctypes.c_int, [P(ConvDesc), P(Thresholds),
                                                           P(ctypes.c_int)]),
        "sparoa_conv2d": (ctypes.c_int, [P(ConvDesc), ctypes.c_int, vp, vp, vp, vp, ctypes.c_int,
                                         vp, vp, vp, sz, vp, vp]),
        "sparoa_conv2d_dense": (ctypes.c_int, [P(ConvDesc), vp, vp, vp, vp, ctypes.c_int, vp, vp,
                                               sz, vp]),
        "sparoa_conv2d_noalloc": (ctypes.c_int, [P(ConvDesc), ctypes.c_int, vp, vp, vp, vp,
                                                 ctypes.c_int, vp, vp, vp, vp]),
        "sparoa_conv2d_zero_skip": (ctypes.c_int, [P(ConvDesc), vp, vp, vp, vp, ctypes.c_int, vp,
                                                   vp, vp, sz, vp, vp]),
        "sparoa_fc_packed_bytes": (ctypes.c_int, [P(FcDesc), P(sz)]),
        "sparoa_fc_pack_weights": (ctypes.c_int, [P(FcDesc), vp, vp, vp]),
        "sparoa_fc_tiling": (ctypes.c_int, [P(FcDesc), ctypes.c_int, P(i64), P(i64)]),
        "sparoa_fc_workspace_size": (ctypes.c_int, [P(FcDesc), ctypes.c_int, P(sz)]),
        "sparoa_fc_skip_block": (ctypes.c_int, [P(FcDesc), ctypes.c_int, P(i64), P(i64)]),
        "sparoa_fc_uses_packed": (ctypes.c_int, [P(FcDesc), ctypes.c_int, P(ctypes.c_int)]),
        "sparoa_fc_ops_run": (ctypes.c_int, [P(FcOp), i64, P(Thresholds), P(vp), vp]),
        "sparoa_fc_measured": (ctypes.c_int, [P(FcDesc), P(Thresholds), vp, vp, vp, vp, vp,
                                              ctypes.c_int, vp, vp, vp, vp, sz, vp, vp]),
        "sparoa_fc": (ctypes.c_int, [P(FcDesc), ctypes.c_int, vp, vp, vp, vp, ctypes.c_int, vp,
                                     vp, vp, sz, vp, vp]),
        "sparoa_fc_dense": (ctypes.c_int, [P(FcDesc), vp, vp, vp, vp, ctypes.c_int, vp, vp, sz,
                                           vp]),
        "sparoa_fc_zero_skip": (ctypes.c_int, [P(FcDesc), vp, vp, vp, vp, ctypes.c_int, vp, vp,
                                               vp, sz, vp, vp]),
        "sparoa_maxpool2d": (ctypes.c_int, [vp, ctypes.c_int, i64, i64, i64, i64, i64, i64, i64,
                                            vp, vp]),
        "sparoa_conv2d_routed": (ctypes.c_int, [P(ConvDesc), P(Thresholds), vp, vp, vp, vp, vp,
                                                ctypes.c_int, vp, vp, vp, sz, vp, vp]),
        "sparoa_fc_routed": (ctypes.c_int, [P(FcDesc), P(Thresholds), vp, vp, vp, vp, vp, vp,
                                            ctypes.c_int, vp, vp, vp, sz, vp, vp]),
        "sparoa_measure_sparsity_preset": (ctypes.c_int, [vp, ctypes.c_int, i64, i64, i64, i64,
                                                          vp, vp, vp, vp]),
        "sparoa_conv2d_split": (ctypes.c_int, [P(ConvDesc), ctypes.c_double, vp, vp, vp, vp, vp,
                                               ctypes.c_int, vp, vp, vp, sz, vp, vp]),
        "sparoa_fc_split": (ctypes.c_int, [P(FcDesc), ctypes.c_double, vp, vp, vp, vp, vp,
                                           ctypes.c_int, vp, vp, vp, sz, vp, vp]),
        "sparoa_conv2d_routed_measured": (ctypes.c_int, [P(ConvDesc), P(Thresholds), vp, vp, vp,
                                                         vp, vp, ctypes.c_int, vp, vp, vp, sz, vp,
                                                         vp, vp, vp, vp]),
        "sparoa_fc_routed_measured": (ctypes.c_int, [P(FcDesc), P(Thresholds), vp, vp, vp, vp, vp,
                                                     vp, ctypes.c_int, vp, vp, vp, sz, vp, vp, vp,
                                                     vp, vp]),
        "sparoa_expert_plan_words": (ctypes.c_int, [i64, i64, i64, P(i64)]),
        "sparoa_expert_route_workspace_size": (ctypes.c_int, [P(ExpertRouteDesc), P(sz)]),
        "sparoa_expert_route": (ctypes.c_int, [P(ExpertRouteDesc), vp, vp, vp, vp, vp, vp, vp, sz,
                                               vp]),
        "sparoa_expert_plan_workspace_size": (ctypes.c_int, [i64, i64, i64, P(sz)]),
        "sparoa_expert_plan": (ctypes.c_int, [i64, i64, i64, vp, vp, vp, sz, vp]),
        "sparoa_expert_ffn_workspace_size": (ctypes.c_int, [P(ExpertFfnDesc), P(sz)]),
        "sparoa_expert_ffn": (ctypes.c_int, [P(ExpertFfnDesc), ctypes.c_int] + [vp] * 10 +
                              [sz, vp]),
        "sparoa_fc_adapted_workspace_size": (ctypes.c_int, [P(FcAdaptedDesc), P(sz)]),
        "sparoa_fc_adapted": (ctypes.c_int, [P(FcAdaptedDesc), ctypes.c_int] + [vp] * 10 +
                              [sz, vp]),
        "sparoa_block_norm": (ctypes.c_int, [P(BlockNormDesc)] + [vp] * 10),
        "sparoa_kv_append": (ctypes.c_int, [P(KvDesc), i64, ctypes.c_int] + [vp, i64] * 3 +
                             [vp] * 9),
        "sparoa_attention_workspace_size": (ctypes.c_int, [P(KvDesc), P(sz)]),
        "sparoa_paged_attention": (ctypes.c_int, [P(KvDesc), P(AttentionOpts)] + [vp] * 11 +
                                   [sz, vp]),
        "sparoa_tree_attention": (ctypes.c_int, [P(KvDesc), P(AttentionOpts)] + [vp] * 11 +
                                  [sz, vp]),
        "sparoa_kv_keep": (ctypes.c_int, [P(KvDesc), i64] + [vp] * 4 + [i64] + [vp] * 4),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    return L


_L = _load()


def _check(status):
    if status != 0:
        raise SparoaError(status, _L.sparoa_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # Once torch's runtime is up the current stream's handle is read
        # directly (0.3 us): asking for the device count and building a Stream
        # object took 3.4 us of each call, more than a short call's kernel.
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    return stream if isinstance(stream, int) else stream.cuda_stream


def _whole(t, dtype, numel, name):
    """The pointer of a dense device tensor of `dtype` with `numel` elements
    (None stays None): what the kernels would read elsewhere is refused here."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or not t.is_cuda:
        raise SparoaError(1, f"{name}: a contiguous {dtype} device tensor of {numel} elements is "
                             f"wanted, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} "
                             f"on {t.device}")
    return t.data_ptr()


def dtype_code(t):
    return _TORCH_DT[t if isinstance(t, torch.dtype) else t.dtype]


def conv_desc(n, c_in, h, w, c_out, kh, kw, sh=1, sw=1, ph=0, pw=0, dh=1, dw=1, groups=1,
              dtype=BF16, has_bias=0):
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return ConvDesc(n, c_in, h, w, c_out, kh, kw, sh, sw, ph, pw, dh, dw, groups, dtype,
                    int(has_bias))


def fc_desc(m, k, n, dtype=BF16, has_bias=0):
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return FcDesc(m, k, n, dtype, int(has_bias))


@dataclass
class MeasureBuffers:
    """Device buffers of one measurement: counts (4 x uint64), optional mask
    and per-sample counts."""
    counts: torch.Tensor
    mask: torch.Tensor = None
    per_sample: torch.Tensor = None


# ------------------------------------------------------------------ calls

def sparoa_abi_version():
    return _L.sparoa_abi_version()


def sparoa_status_string(status):
    return _L.sparoa_status_string(status).decode()


def sparoa_last_error():
    return _L.sparoa_last_error().decode()


def sparoa_mask_words(rows, cols, block_rows, block_cols):
    w = ctypes.c_int64()
    _check(_L.sparoa_mask_words(rows, cols, block_rows, block_cols, ctypes.byref(w)))
    return w.value


def sparoa_measure_sparsity(x, rows, cols, block_rows, block_cols, samples, counts, mask=None,
                            per_sample=None, stream=None, dtype=None):
    _check(_L.sparoa_measure_sparsity(
        _ptr(x), dtype_code(x) if dtype is None else dtype, rows, cols, block_rows, block_cols,
        samples, _ptr(counts), _ptr(mask), _ptr(per_sample), _stream(stream)))


def sparoa_measure_sparsity_preset(x, rows, cols, block_rows, block_cols, counts, mask,
                                   stream=None, dtype=None, commit=None):
    """Measurement into counters already set to {0, numel, nb, nb} (see sparoa.h);
    commit: zeroed count-commit words, or None."""
    _check(_L.sparoa_measure_sparsity_preset(
        _ptr(x), dtype_code(x) if dtype is None else dtype, rows, cols, block_rows, block_cols,
        _ptr(counts), _ptr(mask), _ptr(commit), _stream(stream)))


def sparoa_measure_sparsity_sync(x, rows, cols, block_rows, block_cols, samples, counts,
                                 mask=None, per_sample=None, stream=None, dtype=None):
    host = Counts()
    _check(_L.sparoa_measure_sparsity_sync(
        _ptr(x), dtype_code(x) if dtype is None else dtype, rows, cols, block_rows, block_cols,
        samples, _ptr(counts), _ptr(mask), _ptr(per_sample), ctypes.byref(host),
        _stream(stream)))
    return host.as_dict()


def sparoa_op_intensity_conv(desc):
    out = Intensity()
    _check(_L.sparoa_op_intensity_conv(ctypes.byref(desc), ctypes.byref(out)))
    return out.as_dict()


def sparoa_op_intensity_fc(desc):
    out = Intensity()
    _check(_L.sparoa_op_intensity_fc(ctypes.byref(desc), ctypes.byref(out)))
    return out.as_dict()


def sparoa_route(counts, intensity, is_depthwise, sparsity_thr, intensity_thr, mode=ROUTE_BLOCK):
    c = Counts(counts["zeros"], counts["numel"], counts["zero_blocks"], counts["num_blocks"])
    i = Intensity(intensity["macs"], intensity["flops"], intensity["bytes"],
                  intensity["intensity"])
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    out = ctypes.c_int()
    _check(_L.sparoa_route(ctypes.byref(c), ctypes.byref(i), int(is_depthwise), ctypes.byref(t),
                           ctypes.byref(out)))
    return out.value


def _pair(fn, desc, path):
    a, b = ctypes.c_int64(), ctypes.c_int64()
    _check(fn(ctypes.byref(desc), path, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def sparoa_conv2d_workspace_size(desc, path):
    s = ctypes.c_size_t()
    _check(_L.sparoa_conv2d_workspace_size(ctypes.byref(desc), path, ctypes.byref(s)))
    return s.value


def sparoa_conv2d_skip_block(desc, path):
    return _pair(_L.sparoa_conv2d_skip_block, desc, path)


def sparoa_conv2d_reads_mask(desc, path):
    """Whether the kernel serving `path` reads x's bitmap."""
    v = ctypes.c_int()
    _check(_L.sparoa_conv2d_reads_mask(ctypes.byref(desc), path, ctypes.byref(v)))
    return bool(v.value)


def sparoa_conv2d_routed_reads_mask(desc, sparsity_thr, intensity_thr, mode):
    """Whether the routed conv's skip kernel reads x's bitmap (else mask may be None)."""
    v = ctypes.c_int()
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    _check(_L.sparoa_conv2d_routed_reads_mask(ctypes.byref(desc), ctypes.byref(t),
                                              ctypes.byref(v)))
    return bool(v.value)


def sparoa_conv2d_tiling(desc, path):
    return _pair(_L.sparoa_conv2d_tiling, desc, path)


def sparoa_conv2d(desc, path, x, w, bias, residual, act, mask, y, workspace=None,
                  executed=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_conv2d(ctypes.byref(desc), path, _ptr(x), _ptr(w), _ptr(bias),
                            _ptr(residual), act, _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes,
                            _ptr(executed), _stream(stream)))


def sparoa_conv2d_noalloc(desc, path, x, w, bias, residual, act, mask, y, executed=None,
                          stream=None):
    """sparoa_conv2d with its split-K scratch in the library's own device array."""
    _check(_L.sparoa_conv2d_noalloc(ctypes.byref(desc), path, _ptr(x), _ptr(w), _ptr(bias),
                                    _ptr(residual), act, _ptr(mask), _ptr(y), _ptr(executed),
                                    _stream(stream)))


def sparoa_conv2d_dense(desc, x, w, bias, residual, act, y, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_conv2d_dense(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias),
                                  _ptr(residual), act, _ptr(y), _ptr(workspace), ws_bytes,
                                  _stream(stream)))


def sparoa_conv2d_zero_skip(desc, x, w, bias, residual, act, mask, y, workspace=None,
                            executed=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_conv2d_zero_skip(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias),
                                      _ptr(residual), act, _ptr(mask), _ptr(y), _ptr(workspace),
                                      ws_bytes, _ptr(executed), _stream(stream)))


def sparoa_fc_packed_bytes(desc):
    s = ctypes.c_size_t()
    _check(_L.sparoa_fc_packed_bytes(ctypes.byref(desc), ctypes.byref(s)))
    return s.value


def sparoa_fc_pack_weights(desc, w_nk, w_packed, stream=None):
    _check(_L.sparoa_fc_pack_weights(ctypes.byref(desc), _ptr(w_nk), _ptr(w_packed),
                                     _stream(stream)))


def sparoa_fc_tiling(desc, path):
    return _pair(_L.sparoa_fc_tiling, desc, path)


def sparoa_fc_workspace_size(desc, path):
    s = ctypes.c_size_t()
    _check(_L.sparoa_fc_workspace_size(ctypes.byref(desc), path, ctypes.byref(s)))
    return s.value


def sparoa_fc_skip_block(desc, path):
    return _pair(_L.sparoa_fc_skip_block, desc, path)


def sparoa_fc(desc, path, x, w, bias, residual, act, mask, y, workspace=None, executed=None,
              stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_fc(ctypes.byref(desc), path, _ptr(x), _ptr(w), _ptr(bias), _ptr(residual),
                        act, _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes, _ptr(executed),
                        _stream(stream)))


def sparoa_fc_dense(desc, x, w, bias, residual, act, y, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_fc_dense(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(residual),
                              act, _ptr(y), _ptr(workspace), ws_bytes, _stream(stream)))


def sparoa_fc_zero_skip(desc, x, w, bias, residual, act, mask, y, workspace=None, executed=None,
                        stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_fc_zero_skip(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias),
                                  _ptr(residual), act, _ptr(mask), _ptr(y), _ptr(workspace),
                                  ws_bytes, _ptr(executed), _stream(stream)))


def sparoa_maxpool2d(x, n, c, h, w, k, s, p, y, stream=None):
    _check(_L.sparoa_maxpool2d(_ptr(x), dtype_code(x), n, c, h, w, k, s, p, _ptr(y),
                               _stream(stream)))


def sparoa_conv2d_routed(desc, sparsity_thr, intensity_thr, mode, counts, x, w, bias, residual,
                         act, mask, y, workspace=None, path=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    _check(_L.sparoa_conv2d_routed(ctypes.byref(desc), ctypes.byref(t), _ptr(counts), _ptr(x),
                                   _ptr(w), _ptr(bias), _ptr(residual), act, _ptr(mask), _ptr(y),
                                   _ptr(workspace), ws_bytes, _ptr(path), _stream(stream)))


def sparoa_fc_routed(desc, sparsity_thr, intensity_thr, mode, counts, x, w_nk, w_packed, bias,
                     residual, act, mask, y, workspace=None, path=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    _check(_L.sparoa_fc_routed(ctypes.byref(desc), ctypes.byref(t), _ptr(counts), _ptr(x),
                               _ptr(w_nk), _ptr(w_packed), _ptr(bias), _ptr(residual), act,
                               _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes, _ptr(path),
                               _stream(stream)))


def sparoa_conv2d_routed_measured(desc, sparsity_thr, intensity_thr, mode, counts, x, w, bias,
                                  residual, act, mask, y, y_counts, y_mask, workspace=None,
                                  path=None, y_commit=None, stream=None):
    """sparoa_conv2d_routed that also measures y into y_counts / y_mask
    (y_mask None: counts only; y_commit: zeroed count-commit words, or None)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    _check(_L.sparoa_conv2d_routed_measured(
        ctypes.byref(desc), ctypes.byref(t), _ptr(counts), _ptr(x), _ptr(w), _ptr(bias),
        _ptr(residual), act, _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes, _ptr(path),
        _ptr(y_counts), _ptr(y_mask), _ptr(y_commit), _stream(stream)))


def sparoa_fc_routed_measured(desc, sparsity_thr, intensity_thr, mode, counts, x, w_nk, w_packed,
                              bias, residual, act, mask, y, y_counts, y_mask, workspace=None,
                              path=None, y_commit=None, stream=None):
    """sparoa_fc_routed that also measures y into y_counts / y_mask
    (y_commit: zeroed count-commit words, or None)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    _check(_L.sparoa_fc_routed_measured(
        ctypes.byref(desc), ctypes.byref(t), _ptr(counts), _ptr(x), _ptr(w_nk), _ptr(w_packed),
        _ptr(bias), _ptr(residual), act, _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes,
        _ptr(path), _ptr(y_counts), _ptr(y_mask), _ptr(y_commit), _stream(stream)))


def sparoa_conv2d_split(desc, sparsity_thr, sample_zeros, x, w, bias, residual, act, mask, y,
                        workspace=None, executed=None, stream=None):
    """One conv split over the skip and dense paths by row tile (see sparoa.h)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_conv2d_split(ctypes.byref(desc), sparsity_thr, _ptr(sample_zeros), _ptr(x),
                                  _ptr(w), _ptr(bias), _ptr(residual), act, _ptr(mask), _ptr(y),
                                  _ptr(workspace), ws_bytes, _ptr(executed), _stream(stream)))


def sparoa_fc_split(desc, sparsity_thr, row_zeros, x, w_nk, bias, residual, act, mask, y,
                    workspace=None, executed=None, stream=None):
    """One FC split over the skip and dense paths by row tile (see sparoa.h)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_L.sparoa_fc_split(ctypes.byref(desc), sparsity_thr, _ptr(row_zeros), _ptr(x),
                              _ptr(w_nk), _ptr(bias), _ptr(residual), act, _ptr(mask), _ptr(y),
                              _ptr(workspace), ws_bytes, _ptr(executed), _stream(stream)))


def sparoa_fc_measured(desc, sparsity_thr, intensity_thr, mode, x, w_nk, w_packed, bias, residual,
                       act, counts, mask, y, workspace=None, path=None, stream=None):
    """Measure -> route -> execute of one FC (see sparoa.h)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    t = Thresholds(sparsity_thr, intensity_thr, mode)
    _check(_L.sparoa_fc_measured(ctypes.byref(desc), ctypes.byref(t), _ptr(x), _ptr(w_nk),
                                 _ptr(w_packed), _ptr(bias), _ptr(residual), act, _ptr(counts),
                                 _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes, _ptr(path),
                                 _stream(stream)))


def sparoa_fc_uses_packed(desc, path):
    v = ctypes.c_int()
    _check(_L.sparoa_fc_uses_packed(ctypes.byref(desc), path, ctypes.byref(v)))
    return bool(v.value)


def fc_op(desc, x, w_nk, w_packed, bias, residual, act, counts, mask, y, workspace=None,
          path=None, thresholds=None):
    """One entry of a sparoa_fc_ops_run batch (pointers captured now).
    thresholds: (sparsity_thr, intensity_thr, mode) of this op, used when the
    batch call passes no thresholds of its own."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    t = Thresholds(*(thresholds or (0.5, 315.0, ROUTE_BLOCK)))
    return FcOp(desc, _ptr(x), _ptr(w_nk), _ptr(w_packed), _ptr(bias), _ptr(residual), act,
                _ptr(counts), _ptr(mask), _ptr(y), _ptr(workspace), ws_bytes, _ptr(path), t)


def fc_op_array(ops):
    return (FcOp * len(ops))(*ops)


def sparoa_fc_ops_run(op_array, sparsity_thr=None, intensity_thr=None, mode=ROUTE_BLOCK,
                      events=None, stream=None):
    """Runs a batch built by fc_op_array with the given thresholds, or with
    each op's own when sparsity_thr is None.  events: flat list of 2n
    recorded torch.cuda.Event objects (or None)."""
    t = None if sparsity_thr is None else ctypes.byref(Thresholds(sparsity_thr, intensity_thr, mode))
    ev = None
    if events is not None:
        ev = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    _check(_L.sparoa_fc_ops_run(op_array, len(op_array), t, ev, _stream(stream)))

# ------------------------------------- transformer-block operators (see sparoa.h)

def _scratch(t):
    """Pointer and bytes of a workspace tensor (or None)."""
    if t is None:
        return None, 0
    if not t.is_contiguous() or not t.is_cuda:
        raise SparoaError(1, "workspace: a contiguous device tensor is wanted")
    return t.data_ptr(), t.numel() * t.element_size()


def expert_route_desc(tokens, experts, top_k, dtype=F32, score=SCORE_SOFTMAX, groups=1,
                      top_groups=1, group_best=1, renormalise=False, scale=1.0):
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return ExpertRouteDesc(tokens, experts, top_k, groups, top_groups, group_best, dtype, score,
                           int(renormalise), scale)


def sparoa_expert_plan_words(tokens, top_k, experts):
    w = ctypes.c_int64()
    _check(_L.sparoa_expert_plan_words(tokens, top_k, experts, ctypes.byref(w)))
    return w.value


def expert_plan_views(plan, tokens, top_k, experts):
    """(offsets [experts + 1], order [tokens * top_k], place [tokens * top_k]) of a plan."""
    slots, head = tokens * top_k, -(-(2 * experts + 2) // 4) * 4
    at = head + -(-slots // 4) * 4
    return plan[:experts + 1], plan[head:head + slots], plan[at:at + slots]


def sparoa_expert_route_workspace_size(desc):
    s = ctypes.c_size_t()
    _check(_L.sparoa_expert_route_workspace_size(ctypes.byref(desc), ctypes.byref(s)))
    return s.value


def sparoa_expert_route(desc, logits, bias, token_mask, idx, weights, plan=None, workspace=None,
                        stream=None):
    """Chosen experts, their weights and (plan not None) the dispatch plan."""
    t, e, slots = desc.tokens, desc.experts, desc.tokens * desc.top_k
    words = 0 if plan is None else sparoa_expert_plan_words(t, desc.top_k, e)
    ws, ws_bytes = _scratch(workspace)
    _check(_L.sparoa_expert_route(
        ctypes.byref(desc), _whole(logits, _DT_TORCH.get(desc.dtype), t * e, "logits"),
        _whole(bias, torch.float32, e, "bias"), _whole(token_mask, torch.uint8, t, "token_mask"),
        _whole(idx, torch.int32, slots, "idx"), _whole(weights, torch.float32, slots, "weights"),
        _whole(plan, torch.int32, words, "plan"), ws, ws_bytes, _stream(stream)))


def sparoa_expert_plan_workspace_size(tokens, top_k, experts):
    s = ctypes.c_size_t()
    _check(_L.sparoa_expert_plan_workspace_size(tokens, top_k, experts, ctypes.byref(s)))
    return s.value


def sparoa_expert_plan(tokens, top_k, experts, idx, plan, workspace, stream=None):
    """The dispatch plan of given choices idx [tokens, top_k]."""
    ws, ws_bytes = _scratch(workspace)
    _check(_L.sparoa_expert_plan(
        tokens, top_k, experts, _whole(idx, torch.int32, tokens * top_k, "idx"),
        _whole(plan, torch.int32, sparoa_expert_plan_words(tokens, top_k, experts), "plan"),
        ws, ws_bytes, _stream(stream)))


def expert_ffn_desc(tokens, top_k, experts, hidden, inner, dtype=BF16, gated=False,
                    has_bias=False):
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return ExpertFfnDesc(tokens, top_k, experts, hidden, inner, dtype, int(gated), int(has_bias))


def sparoa_expert_ffn_workspace_size(desc):
    s = ctypes.c_size_t()
    _check(_L.sparoa_expert_ffn_workspace_size(ctypes.byref(desc), ctypes.byref(s)))
    return s.value


def sparoa_expert_ffn(desc, act, x, w_up, b_up, w_down, b_down, weights, plan, residual, y,
                      workspace, stream=None):
    """The FFN of every token's experts, weighted and summed (see sparoa.h)."""
    d, dt = desc, _DT_TORCH.get(desc.dtype)
    rows, tok = d.experts * d.inner * (2 if d.gated else 1), d.tokens * d.hidden
    ws, ws_bytes = _scratch(workspace)
    _check(_L.sparoa_expert_ffn(
        ctypes.byref(d), act, _whole(x, dt, tok, "x"), _whole(w_up, dt, rows * d.hidden, "w_up"),
        _whole(b_up, dt, rows, "b_up"),
        _whole(w_down, dt, d.experts * d.hidden * d.inner, "w_down"),
        _whole(b_down, dt, d.experts * d.hidden, "b_down"),
        _whole(weights, torch.float32, d.tokens * d.top_k, "weights"),
        _whole(plan, torch.int32, sparoa_expert_plan_words(d.tokens, d.top_k, d.experts), "plan"),
        _whole(residual, dt, tok, "residual"), _whole(y, dt, tok, "y"), ws, ws_bytes,
        _stream(stream)))


def fc_adapted_desc(m, k, n, adapters, rank, dtype=BF16, has_bias=False):
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return FcAdaptedDesc(m, k, n, adapters, rank, dtype, int(has_bias))


def sparoa_fc_adapted_workspace_size(desc):
    s = ctypes.c_size_t()
    _check(_L.sparoa_fc_adapted_workspace_size(ctypes.byref(desc), ctypes.byref(s)))
    return s.value


def sparoa_fc_adapted(desc, act, x, w_nk, bias, lora_a, lora_b, scale, adapter_ids, residual, y,
                      workspace, stream=None):
    """FC with the low-rank adapter of each row's request (see sparoa.h)."""
    d, dt = desc, _DT_TORCH.get(desc.dtype)
    ws, ws_bytes = _scratch(workspace)
    _check(_L.sparoa_fc_adapted(
        ctypes.byref(d), act, _whole(x, dt, d.m * d.k, "x"), _whole(w_nk, dt, d.n * d.k, "w_nk"),
        _whole(bias, dt, d.n, "bias"), _whole(lora_a, dt, d.adapters * d.rank * d.k, "lora_a"),
        _whole(lora_b, dt, d.adapters * d.n * d.rank, "lora_b"),
        _whole(scale, torch.float32, d.adapters, "scale"),
        _whole(adapter_ids, torch.int32, d.m, "adapter_ids"),
        _whole(residual, dt, d.m * d.n, "residual"), _whole(y, dt, d.m * d.n, "y"), ws, ws_bytes,
        _stream(stream)))


def block_norm_desc(rows, cols, dtype=BF16, post=NORM_NONE, pre=NORM_RMS, eps=1e-6,
                    gate_rows=None, residual_scale=1.0):
    """gate_rows: rows that share a gate row (default: all of them)."""
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return BlockNormDesc(rows, cols, rows if gate_rows is None else gate_rows, dtype, post, pre,
                         eps, residual_scale)


def sparoa_block_norm(desc, y, post_w, post_b, gate, r, pre_w, pre_b, r_out, n_out, stream=None):
    """r_out = residual_scale r + gate post(y), n_out = pre(r_out)."""
    dt, c, n = _DT_TORCH.get(desc.dtype), desc.cols, desc.rows * desc.cols
    gates = -(-desc.rows // max(1, desc.gate_rows)) * c
    _check(_L.sparoa_block_norm(
        ctypes.byref(desc), _whole(y, dt, n, "y"), _whole(post_w, dt, c, "post_w"),
        _whole(post_b, dt, c, "post_b"), _whole(gate, dt, gates, "gate"), _whole(r, dt, n, "r"),
        _whole(pre_w, dt, c, "pre_w"), _whole(pre_b, dt, c, "pre_b"),
        _whole(r_out, dt, n, "r_out"), _whole(n_out, dt, n, "n_out"), _stream(stream)))

# ------------------------------------ attention over a paged cache (see sparoa.h)

def _now(stream):
    """(current device, the stream's handle); device -2: none yet."""
    if not torch.cuda.is_initialized():
        return -2, _stream(stream)
    here = torch._C._cuda_getDevice()
    if stream is None:
        return here, torch._C._cuda_getCurrentRawStream(here)
    return here, _stream(stream)


def _on(t, dtype, numel, name, here):
    """As _whole, of the current device `here`."""
    if t is None:
        return None
    if t.numel() == numel and t.dtype is dtype and t.get_device() == here and t.is_contiguous():
        return t.data_ptr()
    _whole(t, dtype, numel, name)
    raise SparoaError(1, f"{name}: a tensor on {t.device}, the current device is {here}")


def _rows(t, dtype, rows, width, name, here):
    """Pointer and row stride of a [rows, width] view whose rows are dense."""
    if t.dim() == 2 and t.dtype is dtype and t.get_device() == here >= 0 \
            and t.shape == (rows, width):
        row, one = t.stride()
        if rows == 1:
            row = width
        if row >= width and (one == 1 or width == 1):
            return t.data_ptr(), row
    raise SparoaError(1, f"{name}: a {dtype} tensor [{rows}, {width}] with dense rows on the "
                         f"current device is wanted, got {t.dtype} {tuple(t.shape)} with "
                         f"strides {t.stride()} on {t.device}")


def kv_desc(tokens, requests, heads, kv_heads, head_dim, pages, page_size, table_pages, dtype=BF16,
            max_queries=None, max_keys=None):
    """max_queries: most rows of a request (default: tokens); max_keys: most keys of a
    request (default: what its pages hold)."""
    if isinstance(dtype, torch.dtype):
        dtype = dtype_code(dtype)
    return KvDesc(tokens, requests, heads, kv_heads, head_dim, pages, page_size, table_pages,
                  tokens if max_queries is None else max_queries,
                  table_pages * page_size if max_keys is None else max_keys, dtype)


def attention_opts(scale, cap=0.0, window=0, causal=True):
    return AttentionOpts(scale, cap, window, int(causal))


def _room(t, here):
    """Pointer and bytes of a workspace tensor (or None) of the current device."""
    if t is None:
        return None, 0
    n = t.numel()
    return _on(t, t.dtype, n, "workspace", here), n * t.element_size()


def sparoa_kv_append(desc, q, k, v, freqs, positions, q_start, kv_len, page_table, q_out, k_cache,
                     v_cache, rot_dim=None, interleaved=False, stream=None):
    """Rotates q and k by position (q to q_out) and puts k and v into the cache (see sparoa.h).
    q [tokens, heads * head_dim], k and v [tokens, kv_heads * head_dim]: views with any row
    stride; q and q_out None: no queries; rot_dim: default head_dim, or 0 without freqs."""
    dt, tokens, wide, narrow, cache, requests, table, _, _, dim = desc.of()
    here, handle = _now(stream)
    if rot_dim is None:
        rot_dim = 0 if freqs is None else dim
    qp, qs = (None, wide) if q is None else _rows(q, dt, tokens, wide, "q", here)
    kp, ks = _rows(k, dt, tokens, narrow, "k", here)
    vp, vs = _rows(v, dt, tokens, narrow, "v", here)
    i32 = torch.int32
    _check(_L.sparoa_kv_append(
        ctypes.byref(desc), rot_dim, interleaved, qp, qs, kp, ks, vp, vs,
        _on(freqs, torch.float64, rot_dim // 2, "freqs", here),
        _on(positions, i32, tokens, "positions", here),
        _on(q_start, i32, requests + 1, "q_start", here), _on(kv_len, i32, requests, "kv_len", here),
        _on(page_table, i32, table, "page_table", here),
        _on(q_out, dt, tokens * wide, "q_out", here), _on(k_cache, dt, cache, "k_cache", here),
        _on(v_cache, dt, cache, "v_cache", here), handle))


def sparoa_attention_workspace_size(desc):
    s = ctypes.c_size_t()
    _check(_L.sparoa_attention_workspace_size(ctypes.byref(desc), ctypes.byref(s)))
    return s.value


def sparoa_paged_attention(desc, opts, q, k_cache, v_cache, q_start, kv_len, page_table,
                           prefix_len, first_key, slopes, out, workspace, stream=None):
    """Attention of every request's rows over its cache (see sparoa.h)."""
    dt, tokens, wide, _, cache, requests, table, _, heads, _ = desc.of()
    here, handle = _now(stream)
    i32 = torch.int32
    _check(_L.sparoa_paged_attention(
        ctypes.byref(desc), ctypes.byref(opts), _on(q, dt, tokens * wide, "q", here),
        _on(k_cache, dt, cache, "k_cache", here), _on(v_cache, dt, cache, "v_cache", here),
        _on(q_start, i32, requests + 1, "q_start", here), _on(kv_len, i32, requests, "kv_len", here),
        _on(page_table, i32, table, "page_table", here),
        _on(prefix_len, i32, requests, "prefix_len", here),
        _on(first_key, i32, tokens, "first_key", here),
        _on(slopes, torch.float32, heads, "slopes", here),
        _on(out, dt, tokens * wide, "out", here), *_room(workspace, here), handle))


def sparoa_tree_attention(desc, opts, q, k_cache, v_cache, q_start, kv_len, page_table, tree_mask,
                          positions, slopes, out, workspace, stream=None):
    """Attention of drafted trees over their contexts (see sparoa.h); tree_mask: the bits in
    int64 [tokens, ceil(max_queries / 64)]."""
    dt, tokens, wide, _, cache, requests, table, words, heads, _ = desc.of()
    here, handle = _now(stream)
    i32 = torch.int32
    _check(_L.sparoa_tree_attention(
        ctypes.byref(desc), ctypes.byref(opts), _on(q, dt, tokens * wide, "q", here),
        _on(k_cache, dt, cache, "k_cache", here), _on(v_cache, dt, cache, "v_cache", here),
        _on(q_start, i32, requests + 1, "q_start", here), _on(kv_len, i32, requests, "kv_len", here),
        _on(page_table, i32, table, "page_table", here),
        _on(tree_mask, torch.int64, tokens * words, "tree_mask", here),
        _on(positions, i32, tokens, "positions", here),
        _on(slopes, torch.float32, heads, "slopes", here),
        _on(out, dt, tokens * wide, "out", here), *_room(workspace, here), handle))


def sparoa_kv_keep(desc, layers, q_start, kv_len, page_table, keep, kept, k_cache, v_cache,
                   stream=None):
    """Accepted drafts' keys and values into place, in `layers` caches (see sparoa.h);
    keep int32 [requests, most]."""
    dt, _, _, _, cache, requests, table, _, _, _ = desc.of()
    here, handle = _now(stream)
    i32, most = torch.int32, keep.shape[1] if keep.dim() == 2 else 0
    _check(_L.sparoa_kv_keep(
        ctypes.byref(desc), layers, _on(q_start, i32, requests + 1, "q_start", here),
        _on(kv_len, i32, requests, "kv_len", here), _on(page_table, i32, table, "page_table", here),
        _on(keep, i32, requests * most, "keep", here), most,
        _on(kept, i32, requests, "kept", here),
        _on(k_cache, dt, layers * cache, "k_cache", here),
        _on(v_cache, dt, layers * cache, "v_cache", here), handle))
