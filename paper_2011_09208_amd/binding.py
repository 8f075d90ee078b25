"""ctypes binding over libwhalesplit.so: argument marshalling only.

Every function has the name of the C entry point it calls (minus the `ws_` prefix)
and takes torch tensors that already live on the GPU; torch is used for device
memory and the current stream, nothing else.  There is no CPU fallback: if the
library has not been built, importing this module raises.
"""
import ctypes
import os
import struct
from operator import attrgetter

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwhalesplit.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2011_09208_amd.buildlib` "
        "(or __graft_entry__.build()); there is no fallback path")

lib = ctypes.CDLL(LIB_PATH)

_p, _i32, _i64, _sz, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float

lib.ws_status_string.restype = ctypes.c_char_p
lib.ws_status_string.argtypes = [ctypes.c_int]
lib.ws_version.restype = ctypes.c_int
lib.ws_version.argtypes = []
lib.ws_fwd_workspace_bytes.restype = _sz
lib.ws_fwd_workspace_bytes.argtypes = [_i32, _i32, _i32]
lib.ws_bwd_workspace_bytes.restype = _sz
lib.ws_bwd_workspace_bytes.argtypes = [_i32, _i32, _i32]
lib.ws_split_fc_fwd.restype = ctypes.c_int
lib.ws_split_fc_fwd.argtypes = [_p, _i64, _p, _i64, _p, _p, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _sz, _p]
lib.ws_split_fc_fwd_static.restype = ctypes.c_int
lib.ws_split_fc_fwd_static.argtypes = [_p, _i64, _p, _i64, _p, _p, _i32, _i32, _i32, _i32, _p, _p, _p, _p]
lib.ws_combine_partials.restype = ctypes.c_int
lib.ws_combine_partials.argtypes = [_p, _p, _p, _i32, _i32, _i64, _p, _p, _p, _p]
lib.ws_split_fc_bwd.restype = ctypes.c_int
lib.ws_split_fc_bwd.argtypes = [_p, _i64, _p, _i64, _p, _p, _p, _i32, _i32, _i32, _i32, _f32,
                                _p, _i64, _i32, _p, _i64, _p, _p, _sz, _p]

lib.ws_split_fc_bwd_sgd.restype = ctypes.c_int
lib.ws_split_fc_bwd_sgd.argtypes = [_p, _i64, _p, _i64, _p, _p, _p, _i32, _i32, _i32, _i32, _f32, _f32,
                                    _p, _i64, _i32, _p, _sz, _p]
lib.ws_split_fc_top1.restype = ctypes.c_int
lib.ws_split_fc_top1.argtypes = [_p, _i64, _p, _i64, _p, _i32, _i32, _i32, _i32, _p, _p, _p, _sz, _p]
lib.ws_combine_top1.restype = ctypes.c_int
lib.ws_combine_top1.argtypes = [_p, _p, _i32, _i32, _i64, _p, _p, _p]
lib.ws_split_fc_predict.restype = ctypes.c_int
lib.ws_split_fc_predict.argtypes = [_p, _i64, _p, _i64, _p, _p, _i32, _i32, _i32, _p, _i64, _p]

lib.ws_probe_mfma_loop.restype = ctypes.c_int
lib.ws_probe_mfma_loop.argtypes = [_p, _i32, _i32, _p, _p]
lib.ws_probe_gemm.restype = ctypes.c_int
lib.ws_probe_gemm.argtypes = [_p, _i64, _p, _i64, _i32, _i32, _i32, _p, _i64, _p]

lib.ws_profile_enable.restype = ctypes.c_int
lib.ws_profile_enable.argtypes = [_i32]
lib.ws_profile_reset.restype = ctypes.c_int
lib.ws_profile_reset.argtypes = []
lib.ws_profile_pause.restype = ctypes.c_int
lib.ws_profile_pause.argtypes = [_i32]
lib.ws_profile_trace_dw.restype = ctypes.c_int
lib.ws_profile_trace_dw.argtypes = [ctypes.c_void_p, _i64]
lib.ws_profile_kernel_count.restype = _i32
lib.ws_profile_kernel_count.argtypes = []
lib.ws_profile_kernel_name.restype = ctypes.c_char_p
lib.ws_profile_kernel_name.argtypes = [_i32]
lib.ws_profile_read.restype = ctypes.c_int
lib.ws_profile_read.argtypes = [_i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]

lib.ws_balance_widths.restype = ctypes.c_int
lib.ws_balance_widths.argtypes = [_i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                  ctypes.c_double, ctypes.c_double, _i32, ctypes.POINTER(_i32), ctypes.POINTER(_i32)]

lib.ws_bridge_gather.restype = ctypes.c_int
lib.ws_bridge_gather.argtypes = [_i32, ctypes.POINTER(_p), ctypes.POINTER(_i64), ctypes.POINTER(_i32), _i32, _i32, _i32,
                                 _p, _i64, _p]
lib.ws_bridge_reduce_partition.restype = ctypes.c_int
lib.ws_bridge_reduce_partition.argtypes = [ctypes.POINTER(_p), ctypes.POINTER(_i64), _i32, _i32, ctypes.POINTER(_p),
                                           ctypes.POINTER(_i64), ctypes.POINTER(_i32), _i32, _p]
lib.ws_bridge_fusable.restype = ctypes.c_int
lib.ws_bridge_fusable.argtypes = [_i32, _i32, ctypes.POINTER(_i64), _i32, _i32, ctypes.POINTER(_i64), ctypes.POINTER(_i32)]

lib.ws_sp2_partial_logits.restype = ctypes.c_int
lib.ws_sp2_partial_logits.argtypes = [_p, _i64, _p, _i64, _i32, _i32, _i32, _p, _i64, _p]
lib.ws_sp2_reduce_stats.restype = ctypes.c_int
lib.ws_sp2_reduce_stats.argtypes = [ctypes.POINTER(_p), ctypes.POINTER(_i64), _i32, _p, _p, _i32, _i32, _p, _p, _p]

lib.ws_rms_norm_fwd.restype = ctypes.c_int
lib.ws_rms_norm_fwd.argtypes = [_p, _i64, _p, _i64, _i32, _p, _f32, _i32, _i32, _p, _i64, _p, _i64, _p, _p]
lib.ws_rms_norm_fwd_mx8.restype = ctypes.c_int
lib.ws_rms_norm_fwd_mx8.argtypes = [_p, _i64, _p, _i64, _i32, _p, _f32, _i32, _i32, _p, _i64, _p, _i64, _p, _i64, _p, _p]
lib.ws_rms_norm_bwd_workspace_bytes.restype = _sz
lib.ws_rms_norm_bwd_workspace_bytes.argtypes = [_i32, _i32]
lib.ws_rms_norm_bwd.restype = ctypes.c_int
lib.ws_rms_norm_bwd.argtypes = [_p, _i64, _p, _i64, _p, _i64, _i32, _p, _p, _i32, _i32, _p, _i64, _p, _p, _sz, _p]

lib.ws_quantize_mx4.restype = ctypes.c_int
lib.ws_quantize_mx4.argtypes = [_p, _i64, _i32, _i32, _p, _i64, _p, _i64, _p]
lib.ws_split_fc_w4_logits.restype = ctypes.c_int
lib.ws_split_fc_w4_logits.argtypes = [_p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i32, _i32, _i32, _p, _i64, _p]
lib.ws_w4_top1_workspace_bytes.restype = _sz
lib.ws_w4_top1_workspace_bytes.argtypes = [_i32, _i32]
lib.ws_split_fc_w4_top1.restype = ctypes.c_int
lib.ws_split_fc_w4_top1.argtypes = [_p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i32, _i32, _i32, _i32, _p, _p, _p, _sz, _p]

lib.ws_grad_workspace_bytes.restype = _sz
lib.ws_grad_workspace_bytes.argtypes = [_i32]
lib.ws_grad_sumsq.restype = ctypes.c_int
lib.ws_grad_sumsq.argtypes = [_p, _p, _p, _p, _p, _i32, _p, _p, _sz, _p]
lib.ws_grad_clip.restype = ctypes.c_int
lib.ws_grad_clip.argtypes = [_p, _p, _p, _p, _p, _i32, _p, _i32, _f32, _p, _p]
lib.ws_grad_clip_sgd.restype = ctypes.c_int
lib.ws_grad_clip_sgd.argtypes = [_p, _p, _p, _p, _p, _p, _p, _p, _i32, _p, _i32, _f32, _f32, _p, _p]

STATIC_SCRATCH_BYTES = 16 << 20
RMS_NORM_MAX_D = 16384
W4_MAX_CLASSES = (1 << 30) - 65536

EXPORTS = ["ws_status_string", "ws_version", "ws_fwd_workspace_bytes", "ws_split_fc_fwd", "ws_split_fc_fwd_static",
           "ws_combine_partials", "ws_bwd_workspace_bytes", "ws_split_fc_bwd", "ws_split_fc_bwd_sgd", "ws_split_fc_predict", "ws_split_fc_top1", "ws_combine_top1",
           "ws_profile_enable", "ws_profile_reset", "ws_profile_pause", "ws_profile_trace_dw", "ws_profile_kernel_count", "ws_profile_kernel_name",
           "ws_profile_read", "ws_balance_widths",
           "ws_bridge_gather", "ws_bridge_reduce_partition", "ws_bridge_fusable",
           "ws_rms_norm_fwd", "ws_rms_norm_fwd_mx8", "ws_rms_norm_bwd_workspace_bytes", "ws_rms_norm_bwd",
           "ws_quantize_mx4", "ws_split_fc_w4_logits", "ws_w4_top1_workspace_bytes", "ws_split_fc_w4_top1",
           "ws_grad_workspace_bytes", "ws_grad_sumsq", "ws_grad_clip", "ws_grad_clip_sgd",
           "ws_sp2_partial_logits", "ws_sp2_reduce_stats", "ws_probe_mfma_loop", "ws_probe_gemm"]


class WhaleSplitError(RuntimeError):
    def __init__(self, status):
        self.status = int(status)
        super().__init__(lib.ws_status_string(self.status).decode())


def _check(status):
    if status != 0:
        raise WhaleSplitError(status)


# Addresses are handed to ctypes as plain integers, and the stream is taken without building a torch.cuda.Stream: a call
# cost 5 us more than its launches with the objects (two launches: 12.8 us, now 7.7).
def _ptr(t):
    return None if t is None else t.data_ptr()


try:
    from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice

    _device = _cuda_getDevice

    def _stream():
        return _cuda_getCurrentRawStream(_cuda_getDevice())
except ImportError:                      # PyTorch's own names, which a build without a GPU lacks: the host functions work there, too
    _device = torch.cuda.current_device

    def _stream():
        return torch.cuda.current_stream().cuda_stream


def status_string(status):
    return lib.ws_status_string(int(status)).decode()


def version():
    return lib.ws_version()


def fwd_workspace_bytes(B, D, C_shard):
    return lib.ws_fwd_workspace_bytes(B, D, C_shard)


def bwd_workspace_bytes(B, D, C_shard):
    return lib.ws_bwd_workspace_bytes(B, D, C_shard)


def split_fc_fwd(X, W_shard, b_shard, labels, class_offset, row_max, row_sumexp, label_logit, workspace):
    """X bf16 [B, D]; W_shard bf16 [C_shard, D]; b_shard fp32 [C_shard] or None; labels int32 [B];
    outputs fp32 [B]; workspace uint8 of at least fwd_workspace_bytes."""
    B, D = X.shape
    C = W_shard.shape[0]
    _check(lib.ws_split_fc_fwd(_ptr(X), X.stride(0), _ptr(W_shard), W_shard.stride(0), _ptr(b_shard),
                               _ptr(labels), B, D, C, int(class_offset), _ptr(row_max), _ptr(row_sumexp),
                               _ptr(label_logit), _ptr(workspace), workspace.numel() * workspace.element_size(),
                               _stream()))


def split_fc_fwd_static(X, W_shard, b_shard, labels, class_offset, row_max, row_sumexp, label_logit):
    """split_fc_fwd without a workspace: the library's built-in device scratch is used (no allocation)."""
    B, D = X.shape
    C = W_shard.shape[0]
    _check(lib.ws_split_fc_fwd_static(_ptr(X), X.stride(0), _ptr(W_shard), W_shard.stride(0), _ptr(b_shard),
                                      _ptr(labels), B, D, C, int(class_offset), _ptr(row_max), _ptr(row_sumexp),
                                      _ptr(label_logit), _stream()))


def combine_partials(row_max, row_sumexp, label_logit, logsumexp, loss_rows, loss_mean=None):
    """Statistics are fp32 [S, B] (row pitch = stride(0)); outputs fp32 [B]; loss_mean fp32 [1] or None."""
    S, B = row_max.shape
    stride = row_max.stride(0) if S > 1 else max(B, row_max.stride(0))
    assert row_sumexp.shape == row_max.shape and label_logit.shape == row_max.shape
    if S > 1:
        assert row_sumexp.stride(0) == stride and label_logit.stride(0) == stride
    _check(lib.ws_combine_partials(_ptr(row_max), _ptr(row_sumexp), _ptr(label_logit), S, B, stride,
                                   _ptr(logsumexp), _ptr(loss_rows), _ptr(loss_mean), _stream()))


def split_fc_bwd(X, W_shard, b_shard, logsumexp, labels, class_offset, grad_scale, dX_partial, accumulate_dx,
                 dW_shard, db_shard, workspace):
    """dX_partial fp32 [B, D]; dW_shard bf16 [C_shard, D]; db_shard fp32 [C_shard] or None."""
    B, D = X.shape
    C = W_shard.shape[0]
    _check(lib.ws_split_fc_bwd(_ptr(X), X.stride(0), _ptr(W_shard), W_shard.stride(0), _ptr(b_shard),
                               _ptr(logsumexp), _ptr(labels), B, D, C, int(class_offset), float(grad_scale),
                               _ptr(dX_partial), dX_partial.stride(0), int(bool(accumulate_dx)),
                               _ptr(dW_shard), dW_shard.stride(0), _ptr(db_shard), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream()))


def split_fc_bwd_sgd(X, W_shard, b_shard, logsumexp, labels, class_offset, grad_scale, lr, dX_partial,
                     accumulate_dx, workspace):
    """As split_fc_bwd, but W_shard (bf16) and b_shard (fp32 or None) are updated in place by -lr * gradient."""
    B, D = X.shape
    C = W_shard.shape[0]
    _check(lib.ws_split_fc_bwd_sgd(_ptr(X), X.stride(0), _ptr(W_shard), W_shard.stride(0), _ptr(b_shard),
                                   _ptr(logsumexp), _ptr(labels), B, D, C, int(class_offset), float(grad_scale),
                                   float(lr), _ptr(dX_partial), dX_partial.stride(0), int(bool(accumulate_dx)),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def split_fc_top1(X, W_shard, b_shard, class_offset, top_logit, top_class, workspace):
    """top_logit fp32 [B], top_class int32 [B] <- the shard's best class per row."""
    B, D = X.shape
    C = W_shard.shape[0]
    _check(lib.ws_split_fc_top1(_ptr(X), X.stride(0), _ptr(W_shard), W_shard.stride(0), _ptr(b_shard), B, D, C,
                                int(class_offset), _ptr(top_logit), _ptr(top_class), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream()))


def combine_top1(top_logit, top_class, best_logit, best_class):
    """[S, B] candidates -> [B] winners."""
    S, B = top_logit.shape
    stride = top_logit.stride(0) if S > 1 else max(B, top_logit.stride(0))
    assert top_class.shape == top_logit.shape and (S == 1 or top_class.stride(0) == stride)
    _check(lib.ws_combine_top1(_ptr(top_logit), _ptr(top_class), S, B, stride, _ptr(best_logit), _ptr(best_class),
                               _stream()))


def split_fc_predict(X, W_shard, b_shard, logsumexp, P):
    """P bf16 [B, C_shard] (row pitch a multiple of 8) <- exp(z - logsumexp)."""
    B, D = X.shape
    C = W_shard.shape[0]
    _check(lib.ws_split_fc_predict(_ptr(X), X.stride(0), _ptr(W_shard), W_shard.stride(0), _ptr(b_shard),
                                   _ptr(logsumexp), B, D, C, _ptr(P), P.stride(0), _stream()))


def profile_enable(max_launches):
    _check(lib.ws_profile_enable(int(max_launches)))


def profile_reset():
    _check(lib.ws_profile_reset())


def profile_pause(paused):
    _check(lib.ws_profile_pause(int(bool(paused))))


def profile_trace_dw(trace):
    """trace: int64 CUDA tensor [tiles, 8] that the dW kernel of the following backward calls fills with
    per-tile clock stamps (see the header), or None to switch tracing off."""
    if trace is None:
        _check(lib.ws_profile_trace_dw(None, 0))
    else:
        assert trace.dtype == torch.int64 and trace.is_contiguous() and trace.shape[1] == 8
        _check(lib.ws_profile_trace_dw(_ptr(trace), trace.shape[0]))


def profile_read():
    """{kernel name: (total_ms, launches)} for every kernel that was timed since the last reset."""
    out = {}
    for k in range(lib.ws_profile_kernel_count()):
        ms, n = ctypes.c_double(0.0), ctypes.c_int64(0)
        _check(lib.ws_profile_read(k, ctypes.byref(ms), ctypes.byref(n)))
        if n.value:
            out[lib.ws_profile_kernel_name(k).decode()] = (ms.value, n.value)
    return out


def balance_widths(C, DF, DM, TG_flop, TG_mem):
    """Shard widths for devices with FLOP/s DF and memory DM; returns (list of widths, feasible)."""
    n = len(DF)
    df = (ctypes.c_double * n)(*[float(v) for v in DF])
    dm = (ctypes.c_double * n)(*[float(v) for v in DM])
    w = (_i32 * n)()
    ok = _i32(0)
    _check(lib.ws_balance_widths(n, df, dm, float(TG_flop), float(TG_mem), int(C), w, ctypes.byref(ok)))
    return list(w), bool(ok.value)


def bridge_gather_args(dim, parts, out):
    """The argument tuple of ws_bridge_gather (without the stream) for 2-D device tensors."""
    n = len(parts)
    other, dtype = out.shape[1 - dim], out.dtype
    ptrs, lds, ext = [], [], []
    for p in parts:
        shape = p.shape
        assert len(shape) == 2 and p.dtype == dtype
        rows, cols = shape
        ld, unit = p.stride()
        assert shape[1 - dim] == other
        assert cols <= 1 or unit == 1
        ptrs.append(p.data_ptr())
        lds.append(ld if rows > 1 else max(cols, ld))
        ext.append(shape[dim])
    ptrs, lds, ext = (_p * n)(*ptrs), (_i64 * n)(*lds), (_i32 * n)(*ext)
    return (int(dim), ptrs, lds, ext, n, int(other), out.element_size(), _ptr(out), out.stride(0))


def bridge_gather(dim, parts, out):
    """Concatenates 2-D device tensors `parts` (same dtype, 2 or 4 bytes per element) into `out` along
    dim 0 (rows: the replicate pattern) or dim 1 (columns: the split pattern)."""
    _check(lib.ws_bridge_gather(*bridge_gather_args(dim, parts, out), _stream()))


def bridge_reduce_partition_args(partials, out_parts):
    """The argument tuple of ws_bridge_reduce_partition (without the stream)."""
    S, R = len(partials), len(out_parts)
    D = partials[0].shape[1]
    rows = [o.shape[0] for o in out_parts]
    assert sum(rows) <= min(p.shape[0] for p in partials)
    pp = (_p * S)(*[p.data_ptr() for p in partials])
    pl = (_i64 * S)(*[p.stride(0) for p in partials])
    op = (_p * R)(*[o.data_ptr() for o in out_parts])
    ol = (_i64 * R)(*[o.stride(0) if n > 1 else max(D, o.stride(0)) for o, n in zip(out_parts, rows)])
    rows = (_i32 * R)(*rows)
    return (pp, pl, S, int(D), op, ol, rows, R)


def bridge_reduce_partition(partials, out_parts):
    """out_parts[r] (fp32 [rows_r, D]) = rows of sum(partials) (fp32 [B, D] each), B = sum of rows_r."""
    _check(lib.ws_bridge_reduce_partition(*bridge_reduce_partition_args(partials, out_parts), _stream()))


def bridge_fusable(gather_dim, src_extents, partition_dim, dst_extents):
    a = (_i64 * len(src_extents))(*[int(v) for v in src_extents])
    b = (_i64 * len(dst_extents))(*[int(v) for v in dst_extents])
    ok = _i32(0)
    _check(lib.ws_bridge_fusable(int(gather_dim), len(src_extents), a, int(partition_dim), len(dst_extents), b,
                                 ctypes.byref(ok)))
    return bool(ok.value)


_BF16, _FP32, _I32, _F64 = torch.bfloat16, torch.float32, torch.int32, torch.float64
_STREAM_TYPES = {_BF16: 2, _FP32: 4}
_BYTE_TYPES = (torch.uint8, torch.float8_e4m3fn)


# A call of the norm spends 3.3 us in its checks and 3.7 in the library: the current device is asked for once.
def _here(t):
    """The current device, where the tensor has to be."""
    dev = t.get_device()
    assert 0 <= dev == _device()
    return dev


def _matrix(t, shape, dtype, dev):
    """(address, row pitch) of a tensor on this device, of this shape and with contiguous rows; (None, 0) for no tensor."""
    if t is None:
        return None, 0
    assert t.dtype is dtype and t.shape == shape and t.get_device() == dev
    ld, unit = t.stride()
    if unit != 1 or ld < shape[1]:                         # a single row or column may have any stride
        assert (unit == 1 or shape[1] == 1) and (ld >= shape[1] or shape[0] == 1)
        ld = max(ld, shape[1])
    return t.data_ptr(), ld


def _bytes_matrix(t, shape, dev):
    """_matrix of 8-bit values of either type."""
    return _matrix(t, shape, _BYTE_TYPES[1] if t.dtype is _BYTE_TYPES[1] else _BYTE_TYPES[0], dev)


def _vector(t, n, dtype, dev):
    if t is None:
        return None
    assert t.dtype is dtype and t.shape == (n,) and t.is_contiguous() and t.get_device() == dev
    return t.data_ptr()


def _scratch(t, dev):
    """(address, bytes) of a workspace."""
    if t is None:
        return None, 0
    assert t.is_contiguous() and t.get_device() == dev
    return t.data_ptr(), t.numel() * t.element_size()


def _stream_type(a, b):
    """Type of the residual stream: of the first tensor that is given, bf16 if there is none."""
    return a.dtype if a is not None else b.dtype if b is not None else _BF16


def rms_norm_fwd(x, residual, gamma, eps, h, y, rstd):
    """h = residual + x, y = h * rstd * gamma.  x, y bf16 [B, D]; residual, h bf16 or fp32 [B, D] or None; gamma fp32 [D];
    rstd fp32 [B] or None.  h may be residual itself."""
    dev, shape = _here(x), x.shape
    B, D = shape
    kind = _stream_type(residual, h)
    _check(lib.ws_rms_norm_fwd(*_matrix(x, shape, _BF16, dev), *_matrix(residual, shape, kind, dev), _STREAM_TYPES[kind], _vector(gamma, D, _FP32, dev),
                               eps, B, D, *_matrix(h, shape, kind, dev), *_matrix(y, shape, _BF16, dev), _vector(rstd, B, _FP32, dev), _stream()))


def rms_norm_fwd_mx8(x, residual, gamma, eps, h, y, y_scales, rstd):
    """rms_norm_fwd with y in 8 bits: y uint8 or float8_e4m3fn [B, D], y_scales uint8 [B, D / 32]."""
    dev, shape = _here(x), x.shape
    B, D = shape
    kind = _stream_type(residual, h)
    _check(lib.ws_rms_norm_fwd_mx8(*_matrix(x, shape, _BF16, dev), *_matrix(residual, shape, kind, dev), _STREAM_TYPES[kind], _vector(gamma, D, _FP32, dev),
                                   eps, B, D, *_matrix(h, shape, kind, dev), *_bytes_matrix(y, shape, dev), *_matrix(y_scales, (B, D // 32), torch.uint8, dev),
                                   _vector(rstd, B, _FP32, dev), _stream()))


def rms_norm_bwd_workspace_bytes(B, D):
    return lib.ws_rms_norm_bwd_workspace_bytes(B, D)


def rms_norm_bwd(dY, h, dres, gamma, rstd, dh, dgamma, workspace):
    """dY fp32 [B, D]; h, dh and dres (or None) bf16 or fp32 [B, D]; gamma fp32 [D]; rstd fp32 [B]; dgamma fp32 [D], or None: then
    workspace may be None, else it has rms_norm_bwd_workspace_bytes.  dh may be dres itself."""
    dev, shape = _here(dY), dY.shape
    B, D = shape
    kind = h.dtype
    _check(lib.ws_rms_norm_bwd(*_matrix(dY, shape, _FP32, dev), *_matrix(h, shape, kind, dev), *_matrix(dres, shape, kind, dev), _STREAM_TYPES[kind],
                               _vector(gamma, D, _FP32, dev), _vector(rstd, B, _FP32, dev), B, D, *_matrix(dh, shape, kind, dev), _vector(dgamma, D, _FP32, dev),
                               *_scratch(workspace, dev), _stream()))


def quantize_mx4(W, W4, W_scales):
    """W bf16 [C, D] -> W4 uint8 [C, D / 2] (two codes to a byte, the first in the low bits), W_scales uint8 [C, D / 32]."""
    dev, (C, D) = _here(W), W.shape
    _check(lib.ws_quantize_mx4(*_matrix(W, W.shape, _BF16, dev), C, D, *_matrix(W4, (C, D // 2), torch.uint8, dev),
                               *_matrix(W_scales, (C, D // 32), torch.uint8, dev), _stream()))


def _w4_args(X, X_scales, W4, W_scales, b_shard, dev):
    shape = X.shape
    B, D = shape
    C = W4.shape[0]
    x = _matrix(X, shape, _BF16, dev) if X_scales is None else _bytes_matrix(X, shape, dev)
    return (*x, *_matrix(X_scales, (B, D // 32), torch.uint8, dev), *_matrix(W4, (C, D // 2), torch.uint8, dev),
            *_matrix(W_scales, (C, D // 32), torch.uint8, dev), _vector(b_shard, C, _FP32, dev), B, D, C)


def split_fc_w4_logits(X, X_scales, W4, W_scales, b_shard, Z):
    """Z fp32 [B, C_shard] (row pitch a multiple of 4) <- X . W^T + b.  X bf16 [B, D] with X_scales None, or uint8 / float8_e4m3fn with
    X_scales uint8 [B, D / 32]; W4, W_scales as quantize_mx4 leaves them; b_shard fp32 [C_shard] or None."""
    dev = _here(X)
    a = _w4_args(X, X_scales, W4, W_scales, b_shard, dev)
    _check(lib.ws_split_fc_w4_logits(*a, *_matrix(Z, (a[9], a[11]), _FP32, dev), _stream()))


def w4_top1_workspace_bytes(B, C_shard):
    return lib.ws_w4_top1_workspace_bytes(B, C_shard)


def split_fc_w4_top1(X, X_scales, W4, W_scales, b_shard, class_offset, top_logit, top_class, workspace):
    """top_logit fp32 [B], top_class int32 [B] <- the shard's best class per row (NaN and class_offset for a row of NaN); inputs as
    split_fc_w4_logits."""
    dev = _here(X)
    a = _w4_args(X, X_scales, W4, W_scales, b_shard, dev)
    _check(lib.ws_split_fc_w4_top1(*a, int(class_offset), _vector(top_logit, a[9], _FP32, dev), _vector(top_class, a[9], _I32, dev),
                                   *_scratch(workspace, dev), _stream()))


_ONES = struct.pack("q", 1) * 4096
_ELEM_BYTES = {kind: struct.pack("i", n) for kind, n in _STREAM_TYPES.items()}


def _int64s(values):
    return struct.pack("%dq" % len(values), *values)


class grad_table:
    """The tables that grad_sumsq, grad_clip and grad_clip_sgd take, of bf16 or fp32 device tensors that are contiguous, or
    matrices with contiguous rows.  It holds addresses: build it again when tensors move or change their shapes."""

    def __init__(self, tensors, by_rows=False):
        self.tensors = tensors = list(tensors)
        self.n = n = len(tensors)
        T = torch.Tensor
        self.bytes = b"".join(map(_ELEM_BYTES.__getitem__, map(attrgetter("dtype"), tensors)))
        places = set(map(T.get_device, tensors))
        self.device = _here(tensors[0]) if tensors else None
        assert len(places) <= 1
        self.flat = n == 0 or not by_rows and 8 * n <= len(_ONES) and all(map(T.is_contiguous, tensors))       # each one long row
        self.data = _int64s(list(map(T.data_ptr, tensors)))
        self._shapes = None
        self._extents = None if self.flat else tuple(map(_int64s, zip(*map(self._by_rows, tensors))))

    # What a call does not need is not asked of 100 tensors (the clipped update takes its extents from the gradients); a table that is kept asks once.
    @property
    def extents(self):
        """Rows, columns and pitches."""
        if self._extents is None:
            cols = _int64s(list(map(torch.Tensor.numel, self.tensors)))
            self._extents = _ONES, cols, cols
        return self._extents

    @property
    def shapes(self):
        if self._shapes is None:
            self._shapes = list(map(attrgetter("shape"), self.tensors))
        return self._shapes

    @staticmethod
    def _by_rows(t):
        """(rows, columns, pitch)"""
        shape, strides = t.shape, t.stride()
        while len(shape) > 2 and shape[0] == 1:
            shape, strides = shape[1:], strides[1:]
        if len(shape) != 2:
            assert t.is_contiguous()
            return 1, t.numel(), t.numel()
        (r, c), (ld, unit) = shape, strides
        assert unit == 1 or c <= 1
        return r, c, ld if r > 1 else c


def _without_leading_ones(shape):
    while len(shape) > 0 and shape[0] == 1:
        shape = shape[1:]
    return shape


def _table(tensors, dev):
    table = tensors if isinstance(tensors, grad_table) else grad_table(tensors)
    assert table.device in (dev, None)
    return table


def grad_workspace_bytes(n):
    return lib.ws_grad_workspace_bytes(n)


def grad_sumsq(grads, sumsq, workspace):
    """sumsq fp64 [1] <- the sum of the squares of all gradients (tensors, or their grad_table)."""
    dev = _here(sumsq)
    g = _table(grads, dev)
    _check(lib.ws_grad_sumsq(g.data, *g.extents, g.bytes, g.n, _vector(sumsq, 1, _F64, dev), *_scratch(workspace, dev), _stream()))


def grad_clip(grads, sumsq, max_norm, norm=None):
    """Scales the gradients in place by min(1, max_norm / norm), norm = sqrt(sum of sumsq fp64 [S]); norm fp32 [1] or None."""
    S, dev = sumsq.numel(), _here(sumsq)
    g = _table(grads, dev)
    _check(lib.ws_grad_clip(g.data, *g.extents, g.bytes, g.n, _vector(sumsq, S, _F64, dev), S, float(max_norm),
                            _vector(norm, 1, torch.float32, dev), _stream()))


def grad_clip_sgd(params, grads, sumsq, max_norm, lr, norm=None):
    """params[i] <- params[i] - lr * k * grads[i] with grad_clip's factor k; the gradients are left as they are.  A gradient has its
    parameter's shape (leading dimensions of 1 aside)."""
    S, dev = sumsq.numel(), _here(sumsq)
    p, g = _table(params, dev), _table(grads, dev)
    if p.shapes != g.shapes:
        assert list(map(_without_leading_ones, p.shapes)) == list(map(_without_leading_ones, g.shapes))
    if not (p.flat and g.flat):                            # one of a pair has a pitch: all are described by their rows
        p, g = [t if not t.flat else grad_table(t.tensors, True) for t in (p, g)]
        assert p.extents[:2] == g.extents[:2]
    ld_params = g.extents[2] if p.flat else p.extents[2]
    _check(lib.ws_grad_clip_sgd(p.data, ld_params, p.bytes, g.data, *g.extents, g.bytes, g.n, _vector(sumsq, S, _F64, dev), S,
                                float(max_norm), float(lr), _vector(norm, 1, torch.float32, dev), _stream()))


def sp2_partial_logits(X_slice, W_slice, Z_partial):
    """Z_partial fp32 [B, C] <- X_slice [B, D_s] . W_slice [C, D_s]^T (column slices may be views)."""
    B, Ds = X_slice.shape
    C = W_slice.shape[0]
    _check(lib.ws_sp2_partial_logits(_ptr(X_slice), X_slice.stride(0), _ptr(W_slice), W_slice.stride(0), B, Ds, C,
                                     _ptr(Z_partial), Z_partial.stride(0), _stream()))


def sp2_reduce_stats(Z_partials, bias, labels, logsumexp, loss_rows):
    S = len(Z_partials)
    B, C = Z_partials[0].shape
    zp = (_p * S)(*[z.data_ptr() for z in Z_partials])
    zl = (_i64 * S)(*[z.stride(0) for z in Z_partials])
    _check(lib.ws_sp2_reduce_stats(zp, zl, S, _ptr(bias), _ptr(labels), B, C, _ptr(logsumexp), _ptr(loss_rows),
                                   _stream()))


def probe_mfma_loop(fragments, rounds, workgroups, sink):
    """fragments: uint8/bf16 tensor of 16 * 512 * 16 bytes; sink fp32 [workgroups * 512]."""
    _check(lib.ws_probe_mfma_loop(_ptr(fragments), int(rounds), int(workgroups), _ptr(sink), _stream()))


def probe_gemm(A, B, C):
    """C [N, M] bf16 <- A [M, K] . B [N, K]^T (bf16), the library's main loop alone."""
    M, K = A.shape
    N = B.shape[0]
    _check(lib.ws_probe_gemm(_ptr(A), A.stride(0), _ptr(B), B.stride(0), M, N, K, _ptr(C), C.stride(0), _stream()))
