"""ctypes binding of ``libconvnet_hotpath.so`` (see ``include/convnet_hotpath.h``).

Argument marshalling only: every function here hands device pointers, extents
and a HIP stream to the C ABI entry point of the same name.  PyTorch supplies
device memory and streams; no arithmetic of the convolution path happens in
Python.  If the library has not been built this module raises -- there is no
fallback path.
"""
import ctypes
import functools
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libconvnet_hotpath.so")

OK = 0
ERR_INVALID_ARG, ERR_TOO_LARGE, ERR_BAD_DTYPE, ERR_WORKSPACE, ERR_MISALIGNED, ERR_HIP = -1, -2, -3, -4, -5, -6
ERR_SCRATCH_LIMIT = -7
NOALLOC_SCRATCH_BYTES = 48 << 20
DTYPE_F32, DTYPE_BF16, DTYPE_BF16_OUT_BF16 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2}
LAYOUT_PLANES, LAYOUT_CHANNELS_LAST = 0, 1
DISTILL_MAX_TOP = 1024
BLOCK_FORMATS = {"e4m3": 0, "e2m1": 1}
BLOCK_VALUES, BLOCK_ROW_FILL = 32, 128
OP_FWD, OP_BWD_DATA, OP_BWD_FILTER = 0, 1, 2

EXPORTS = (
    "conv_fwd", "conv_bwd_data", "conv_bwd_filter", "conv_bwd_filter_noalloc",
    "conv_fwd_ex", "conv_bwd_data_ex", "conv_bwd_filter_ex", "conv_fwd_bias_relu", "conv_bwd_data_relu",
    "conv_fwd_grouped", "conv_bwd_data_grouped", "conv_bwd_filter_grouped", "conv_workspace_bytes_grouped",
    "conv_workspace_bytes", "conv_output_extent", "conv_status_string", "conv_last_hip_error",
    "relu_fwd", "relu_bwd", "maxpool3x3s2_fwd", "maxpool3x3s2_bwd",
    "relu_maxpool3x3s2_fwd", "relu_maxpool3x3s2_bwd", "convert_f32_to_bf16",
    "bias_fwd", "bias_bwd", "bias_bwd_workspace_bytes",
    "fc_fwd", "fc_bwd_data", "fc_bwd_filter", "fc_workspace_bytes", "sgd_update", "sgd_update_multi",
    "group_norm_act_fwd", "group_norm_act_bwd", "group_norm_act_workspace_bytes",
    "distill_loss_fwd", "distill_loss_bwd", "distill_loss_fwd_bwd", "distill_loss_workspace_bytes",
    "quantize_blocks", "dequantize_blocks", "layer_norm_fwd", "layer_norm_bwd", "layer_norm_bwd_kept",
    "layer_norm_workspace_bytes", "fc_bwd_filter_kept", "fc_kept_workspace_bytes", "fc_fwd_q4", "fc_q4_workspace_bytes",
)

_lib = None


class ConvError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib().conv_status_string(status).decode()
        if status == ERR_HIP:
            msg += ": " + lib().conv_last_hip_error().decode()
        super().__init__("%s failed with status %d (%s)" % (where, status, msg))


def lib():
    """The loaded C library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "%s is missing: build it with `python -m paper_1312_5853_amd.build` "
            "(there is no fallback implementation)" % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    vp, i, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    dims = [i] * 9
    for name in ("conv_fwd", "conv_bwd_data", "conv_bwd_filter"):
        f = getattr(L, name)
        f.argtypes = [vp, vp, vp] + dims + [i, vp, sz, vp]
        f.restype = i
        f = getattr(L, name + "_ex")
        f.argtypes = [vp, vp, vp] + dims + [i64, i64, i, vp, sz, vp]
        f.restype = i
        f = getattr(L, name + "_grouped")
        f.argtypes = [vp, vp, vp] + dims + [i, i, vp, sz, vp]
        f.restype = i
    L.conv_bwd_filter_noalloc.argtypes = [vp, vp, vp] + dims + [i, vp]
    L.conv_bwd_filter_noalloc.restype = i
    L.conv_fwd_bias_relu.argtypes = [vp, vp, vp, vp] + dims + [i, i, vp, sz, vp]
    L.conv_fwd_bias_relu.restype = i
    L.conv_bwd_data_relu.argtypes = [vp, vp, vp, vp] + dims + [i, vp, sz, vp]
    L.conv_bwd_data_relu.restype = i
    L.fc_fwd.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
    L.fc_bwd_data.argtypes = [vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.fc_bwd_filter.argtypes = [vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.fc_workspace_bytes.argtypes = [i, i, i, i, i]
    L.fc_workspace_bytes.restype = sz
    f32 = ctypes.c_float
    L.sgd_update.argtypes = [vp, vp, vp, i64, f32, f32, f32, f32, vp]
    L.sgd_update_multi.argtypes = [vp, vp, vp, vp, i, f32, f32, f32, f32, vp]
    for name in ("fc_fwd", "fc_bwd_data", "fc_bwd_filter", "sgd_update", "sgd_update_multi"):
        getattr(L, name).restype = i
    L.conv_workspace_bytes_grouped.argtypes = [i] + dims + [i, i]
    L.conv_workspace_bytes_grouped.restype = sz
    L.conv_workspace_bytes.argtypes = [i] + dims + [i]
    L.conv_workspace_bytes.restype = sz
    L.bias_fwd.argtypes = [vp, vp, i, i, i, i, vp]
    L.bias_fwd.restype = i
    L.bias_bwd.argtypes = [vp, vp, i, i, i, i, vp, sz, vp]
    L.bias_bwd.restype = i
    L.bias_bwd_workspace_bytes.argtypes = [i, i]
    L.bias_bwd_workspace_bytes.restype = sz
    L.conv_output_extent.argtypes = [i, i, i, i]
    L.conv_output_extent.restype = i
    L.conv_status_string.argtypes = [i]
    L.conv_status_string.restype = ctypes.c_char_p
    L.conv_last_hip_error.argtypes = []
    L.conv_last_hip_error.restype = ctypes.c_char_p
    L.relu_fwd.argtypes = [vp, vp, i64, i, vp]
    L.relu_bwd.argtypes = [vp, vp, vp, i64, i, vp]
    L.maxpool3x3s2_fwd.argtypes = [vp, vp, i64, i, i, i, vp]
    L.maxpool3x3s2_bwd.argtypes = [vp, vp, vp, i64, i, i, i, vp]
    L.convert_f32_to_bf16.argtypes = [vp, vp, i64, vp]
    L.convert_f32_to_bf16.restype = i
    L.relu_maxpool3x3s2_fwd.argtypes = [vp, vp, i64, i, i, i, vp]
    L.relu_maxpool3x3s2_bwd.argtypes = [vp, vp, vp, i64, i, i, i, vp]
    for name in ("relu_fwd", "relu_bwd", "maxpool3x3s2_fwd", "maxpool3x3s2_bwd", "relu_maxpool3x3s2_fwd",
                 "relu_maxpool3x3s2_bwd"):
        getattr(L, name).restype = i
    L.group_norm_act_fwd.argtypes = [vp] * 6 + [i, i, i, i, f32, i, i, i, vp, sz, vp]
    L.group_norm_act_bwd.argtypes = [vp] * 9 + [i, i, i, i, i, i, i, vp, sz, vp]
    L.group_norm_act_workspace_bytes.argtypes = [i] * 7
    terms = [i, i, i, f32, f32, f32, i, i, i]
    L.distill_loss_fwd.argtypes = [vp, i64, vp, vp, vp, vp, vp] + terms + [vp, sz, vp]
    L.distill_loss_bwd.argtypes = [vp, i64, vp, vp, vp, vp, vp, f32, vp, i64] + terms + [vp]
    L.distill_loss_fwd_bwd.argtypes = [vp, i64, vp, vp, vp, vp, f32, vp, vp, i64] + terms + [vp, sz, vp]
    L.distill_loss_workspace_bytes.argtypes = [i] * 4
    for name in ("group_norm_act_fwd", "group_norm_act_bwd", "distill_loss_fwd", "distill_loss_bwd",
                 "distill_loss_fwd_bwd"):
        getattr(L, name).restype = i
    for name in ("group_norm_act_workspace_bytes", "distill_loss_workspace_bytes"):
        getattr(L, name).restype = sz
    L.quantize_blocks.argtypes = [vp, i64, vp, vp, i, i, i, i, vp]
    L.dequantize_blocks.argtypes = [vp, vp, vp, i64, i, i, i, i, vp]
    L.layer_norm_fwd.argtypes = [vp, i64, vp, vp, vp, i64, vp, vp, i, i, f32, i, vp]
    L.layer_norm_bwd.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, i, i, i, vp, sz, vp]
    L.layer_norm_bwd_kept.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp, i, i, i, vp, sz, vp]
    L.fc_bwd_filter_kept.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, sz, vp]
    L.fc_fwd_q4.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp]
    for name in ("quantize_blocks", "dequantize_blocks", "layer_norm_fwd", "layer_norm_bwd", "layer_norm_bwd_kept",
                 "fc_bwd_filter_kept", "fc_fwd_q4"):
        getattr(L, name).restype = i
    for name in ("layer_norm_workspace_bytes", "fc_kept_workspace_bytes", "fc_q4_workspace_bytes"):
        getattr(L, name).argtypes = [i] * 4
        getattr(L, name).restype = sz
    _lib = L
    return L


def status_string(status):
    return lib().conv_status_string(int(status)).decode()


# The two questions below have answers that depend on their arguments alone and cost as much host time as a launch: a
# training loop asks them for the same few layers on every step.  Bounded; lru_cache is safe between threads.  The keys are
# plain ints: whatever else stands for a whole number (a 0-d array, which has no hash, or a 0-d tensor, whose hash is its
# identity) is turned into one first, in the public functions here and for the scalars of a call in `_whole`.
@functools.lru_cache(maxsize=1024, typed=True)
def _workspace_bytes(op, N, C, H, W, K, R, S, stride, pad, dtype):
    return int(lib().conv_workspace_bytes(op, N, C, H, W, K, R, S, stride, pad, dtype))


@functools.lru_cache(maxsize=1024, typed=True)
def _out_extent(size, filt, stride, pad):
    return int(lib().conv_output_extent(size, filt, stride, pad))


def _whole(*values):
    return tuple(map(operator.index, values))


def workspace_bytes(op, N, C, H, W, K, R, S, stride, pad, dtype=DTYPE_F32):
    return _workspace_bytes(*_whole(op, N, C, H, W, K, R, S, stride, pad, dtype))


def out_extent(size, filt, stride, pad):
    """P or Q of a layer, asked of the library (conv_output_extent)."""
    return _out_extent(*_whole(size, filt, stride, pad))


def _stream_handle(stream):
    """Handle of `stream`, or of the current device's current stream, as an integer (a Stream object per call would cost
    more than the rest of the marshalling)."""
    if stream is None:
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _ptr(t):
    return t.data_ptr()


def _dtype_of(t):
    if t.dtype == torch.float32:
        return DTYPE_F32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    raise TypeError("unsupported tensor dtype %s" % t.dtype)


class Workspace:
    """A growable device scratch buffer handed to the library as `ws`: for the calls of one stream and one thread (calls
    that overlap would take their sums from each other), and, where a call is captured in a graph, grown to its size
    before that."""

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = None

    def get(self, nbytes):
        if nbytes == 0:
            return None, 0
        if self.buf is None or self.buf.numel() < nbytes:
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self.buf, self.buf.numel()


# Scratch of a call without a `ws` is its own, from PyTorch's allocator, on the stream that the call runs on, so that the
# memory can be given out again when that stream has passed the call; it is held until the library has returned.
_take_scratch = torch._C._cuda_cudaCachingAllocator_raw_alloc
_give_scratch = torch._C._cuda_cudaCachingAllocator_raw_delete


class _Scratch:
    __slots__ = ("at",)

    def __init__(self, nbytes, handle):
        self.at = 0
        self.at = _take_scratch(nbytes, handle)

    def data_ptr(self):
        return self.at

    def __del__(self):
        if self.at:
            _give_scratch(self.at)


def _scratch(ws, nbytes, stream):
    """(buffer, its size) for a call that needs so many bytes: of `ws`, or one of its own; (None, 0) for none."""
    if nbytes == 0:
        return None, 0
    return ws.get(nbytes) if ws is not None else (_Scratch(nbytes, _stream_handle(stream)), nbytes)


def _run(name, op, a, b, out, dims, x_bs, y_bs, dtype, ws, stream):
    need = _workspace_bytes(op, *dims, dtype)
    buf, nbytes = _scratch(ws, need, stream)
    wsp = buf.data_ptr() if buf is not None else 0
    if x_bs or y_bs:
        rc = getattr(lib(), name + "_ex")(_ptr(a), _ptr(b), _ptr(out), *dims, int(x_bs), int(y_bs), dtype,
                                          wsp, nbytes, _stream_handle(stream))
    else:
        rc = getattr(lib(), name)(_ptr(a), _ptr(b), _ptr(out), *dims, dtype, wsp, nbytes, _stream_handle(stream))
    if rc != OK:
        raise ConvError(rc, name)
    return out


def _batch_stride(t):
    """Batch stride in elements of an NCHW tensor whose samples are dense (a
    channel slice of a wider tensor qualifies); 0 when the whole tensor is."""
    n, c, h, w = t.shape
    sn, sc, sh, sw = t.stride()
    if sw != 1 or sh != w or sc != h * w:
        raise ValueError("the [channel][row][col] block of every sample must be dense")
    return 0 if (n == 1 or sn == c * h * w) else sn


def _io_dtype(src, out):
    """dtype code of a forward / backward-data call from its input and output tensors."""
    d = _dtype_of(src)
    if out.dtype == torch.bfloat16:
        if d != DTYPE_BF16:
            raise TypeError("a bfloat16 output needs bfloat16 inputs")
        return DTYPE_BF16_OUT_BF16
    if out.dtype != torch.float32:
        raise TypeError("unsupported output dtype %s" % out.dtype)
    return d


def conv_fwd(x, w, stride, pad, y=None, ws=None, stream=None, out_bf16=False):
    """x [N,C,H,W], w [K,C,R,S] -> y [N,K,P,Q], fp32 (or bfloat16: pass a bfloat16 y, or out_bf16=True, with
    bfloat16 inputs).  x and y may be channel slices of wider NCHW tensors (their batch strides are passed on)."""
    if not (type(stride) is type(pad) is int):
        stride, pad = _whole(stride, pad)
    N, C, H, W = x.shape
    K, Cw, R, S = w.shape
    if C != Cw or not w.is_contiguous():
        raise ValueError("filter tensor does not match the input")
    P, Q = _out_extent(H, R, stride, pad), _out_extent(W, S, stride, pad)
    if y is None:
        y = torch.empty((N, K, P, Q), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=x.device)
    dims = (N, C, H, W, K, R, S, stride, pad)
    return _run("conv_fwd", OP_FWD, x, w, y, dims, _batch_stride(x), _batch_stride(y), _io_dtype(x, y), ws, stream)


def conv_bwd_data(dy, w, H, W, stride, pad, dx=None, ws=None, stream=None, out_bf16=False):
    """dy [N,K,P,Q], w [K,C,R,S] -> dx [N,C,H,W] fp32 or bfloat16 (H, W: the layer's input extent)."""
    if not (type(H) is type(W) is type(stride) is type(pad) is int):
        H, W, stride, pad = _whole(H, W, stride, pad)
    N = dy.shape[0]
    K, C, R, S = w.shape
    if dy.shape[1] != K or not w.is_contiguous():
        raise ValueError("filter tensor does not match the output gradient")
    if dx is None:
        dx = torch.empty((N, C, H, W), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=dy.device)
    dims = (N, C, H, W, K, R, S, stride, pad)
    return _run("conv_bwd_data", OP_BWD_DATA, dy, w, dx, dims, _batch_stride(dx), _batch_stride(dy),
                _io_dtype(dy, dx), ws, stream)


def _dense(*ts):
    for t in ts:
        if t is not None and not t.is_contiguous():
            raise ValueError("this call takes dense tensors")


def conv_fwd_bias_relu(x, w, bias, stride, pad, relu=True, y=None, ws=None, stream=None, out_bf16=False):
    """y = relu(conv_fwd(x, w) + bias[k]) in one call (bias: fp32 [K] or None; relu=False leaves the sum as it is)."""
    if not (type(stride) is type(pad) is int):
        stride, pad = _whole(stride, pad)
    N, C, H, W = x.shape
    K, Cw, R, S = w.shape
    if C != Cw:
        raise ValueError("filter tensor does not match the input")
    if bias is not None and (bias.dtype != torch.float32 or bias.numel() != K):
        raise ValueError("bias must hold one fp32 value per filter")
    P, Q = _out_extent(H, R, stride, pad), _out_extent(W, S, stride, pad)
    if y is None:
        y = torch.empty((N, K, P, Q), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=x.device)
    _dense(x, w, bias, y)
    dims = (N, C, H, W, K, R, S, stride, pad)
    dtype = _io_dtype(x, y)
    buf, nbytes = _scratch(ws, _workspace_bytes(OP_FWD, *dims, dtype), stream)
    wsp = buf.data_ptr() if buf is not None else 0
    bp = _ptr(bias) if bias is not None else 0
    rc = lib().conv_fwd_bias_relu(_ptr(x), _ptr(w), bp, _ptr(y), *dims, 1 if relu else 0, dtype, wsp, nbytes,
                                  _stream_handle(stream))
    if rc != OK:
        raise ConvError(rc, "conv_fwd_bias_relu")
    return y


def conv_bwd_data_relu(dy, w, act, stride, pad, dx=None, ws=None, stream=None):
    """dx = conv_bwd_data(dy, w) where act > 0, else 0 (act [N,C,H,W]: output or input of the ReLU that feeds this
    layer, element type of dx)."""
    if not (type(stride) is type(pad) is int):
        stride, pad = _whole(stride, pad)
    N, C, H, W = act.shape
    K, Cw, R, S = w.shape
    if dy.shape[1] != K or Cw != C:
        raise ValueError("filter tensor does not match the tensors")
    if dx is None:
        dx = torch.empty_like(act)
    if dx.dtype != act.dtype or dx.shape != act.shape:
        raise ValueError("act must have the shape and element type of dx")
    _dense(dy, w, act, dx)
    dims = (N, C, H, W, K, R, S, stride, pad)
    dtype = _io_dtype(dy, dx)
    buf, nbytes = _scratch(ws, _workspace_bytes(OP_BWD_DATA, *dims, dtype), stream)
    wsp = buf.data_ptr() if buf is not None else 0
    rc = lib().conv_bwd_data_relu(_ptr(dy), _ptr(w), _ptr(act), _ptr(dx), *dims, dtype, wsp, nbytes,
                                  _stream_handle(stream))
    if rc != OK:
        raise ConvError(rc, "conv_bwd_data_relu")
    return dx


def conv_bwd_filter(x, dy, R, S, stride, pad, dw=None, ws=None, stream=None):
    """x [N,C,H,W], dy [N,K,P,Q] -> dw [K,C,R,S] fp32."""
    if not (type(R) is type(S) is type(stride) is type(pad) is int):
        R, S, stride, pad = _whole(R, S, stride, pad)
    N, C, H, W = x.shape
    K = dy.shape[1]
    if dw is None:
        dw = torch.empty((K, C, R, S), dtype=torch.float32, device=x.device)
    dims = (N, C, H, W, K, R, S, stride, pad)
    return _run("conv_bwd_filter", OP_BWD_FILTER, x, dy, dw, dims, _batch_stride(x), _batch_stride(dy),
                _dtype_of(x), ws, stream)


def conv_bwd_filter_noalloc(x, dy, R, S, stride, pad, dw=None, stream=None):
    """conv_bwd_filter on dense tensors with the library's built-in scratch: no workspace argument.  `dw` must be
    given by callers that may not allocate (this wrapper allocates it only when it is None)."""
    N, C, H, W = x.shape
    K = dy.shape[1]
    _dense(x, dy, dw)
    if dw is None:
        dw = torch.empty((K, C, R, S), dtype=torch.float32, device=x.device)
    rc = lib().conv_bwd_filter_noalloc(_ptr(x), _ptr(dy), _ptr(dw), N, C, H, W, K, R, S, stride, pad, _dtype_of(x),
                                       _stream_handle(stream))
    if rc != OK:
        raise ConvError(rc, "conv_bwd_filter_noalloc")
    return dw


def _run_grouped(name, op, a, b, out, dims, groups, dtype, ws, stream):
    for t in (a, b, out):
        if not t.is_contiguous():
            raise ValueError("grouped calls take dense tensors")
    need = int(lib().conv_workspace_bytes_grouped(op, *dims, groups, dtype))
    buf, nbytes = _scratch(ws, need, stream)
    wsp = buf.data_ptr() if buf is not None else 0
    rc = getattr(lib(), name)(_ptr(a), _ptr(b), _ptr(out), *dims, groups, dtype, wsp, nbytes, _stream_handle(stream))
    if rc != OK:
        raise ConvError(rc, name)
    return out


def conv_fwd_grouped(x, w, stride, pad, groups, y=None, ws=None, stream=None, out_bf16=False):
    """x [N,C,H,W], w [K,C/groups,R,S] -> y [N,K,P,Q]: column g's filters read column g's channels only."""
    if not (type(stride) is type(pad) is int):
        stride, pad = _whole(stride, pad)
    N, C, H, W = x.shape
    K, Cg, R, S = w.shape
    if Cg * groups != C or K % groups:
        raise ValueError("filter tensor does not match the input and the group count")
    P, Q = _out_extent(H, R, stride, pad), _out_extent(W, S, stride, pad)
    if y is None:
        y = torch.empty((N, K, P, Q), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=x.device)
    return _run_grouped("conv_fwd_grouped", OP_FWD, x, w, y, (N, C, H, W, K, R, S, stride, pad), groups,
                        _io_dtype(x, y), ws, stream)


def conv_bwd_data_grouped(dy, w, H, W, stride, pad, groups, dx=None, ws=None, stream=None, out_bf16=False):
    N = dy.shape[0]
    K, Cg, R, S = w.shape
    C = Cg * groups
    if dy.shape[1] != K or K % groups:
        raise ValueError("filter tensor does not match the output gradient and the group count")
    if dx is None:
        dx = torch.empty((N, C, H, W), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=dy.device)
    return _run_grouped("conv_bwd_data_grouped", OP_BWD_DATA, dy, w, dx, (N, C, H, W, K, R, S, stride, pad), groups,
                        _io_dtype(dy, dx), ws, stream)


def conv_bwd_filter_grouped(x, dy, R, S, stride, pad, groups, dw=None, ws=None, stream=None):
    N, C, H, W = x.shape
    K = dy.shape[1]
    if C % groups or K % groups:
        raise ValueError("channel counts are not multiples of the group count")
    if dw is None:
        dw = torch.empty((K, C // groups, R, S), dtype=torch.float32, device=x.device)
    return _run_grouped("conv_bwd_filter_grouped", OP_BWD_FILTER, x, dy, dw, (N, C, H, W, K, R, S, stride, pad),
                        groups, _dtype_of(x), ws, stream)


def _check(rc, where):
    if rc != OK:
        raise ConvError(rc, where)


def _glue_dtype(*tensors):
    """All tensors of a glue call share one element type (fp32 or bfloat16)."""
    d = _dtype_of(tensors[0])
    for t in tensors[1:]:
        if t.dtype != tensors[0].dtype:
            raise TypeError("the tensors of a glue call must have one dtype")
    return d


def relu_fwd(x, y=None, stream=None):
    if y is None:
        y = torch.empty_like(x)
    _check(lib().relu_fwd(_ptr(x), _ptr(y), x.numel(), _glue_dtype(x, y), _stream_handle(stream)), "relu_fwd")
    return y


def relu_bwd(x, dy, dx=None, stream=None):
    if dx is None:
        dx = torch.empty_like(dy)
    _check(lib().relu_bwd(_ptr(x), _ptr(dy), _ptr(dx), x.numel(), _glue_dtype(x, dy, dx), _stream_handle(stream)),
           "relu_bwd")
    return dx


def _pool_fwd(name, x, y, stream):
    N, C, H, W = x.shape
    if y is None:
        y = torch.empty((N, C, (H - 3) // 2 + 1, (W - 3) // 2 + 1), dtype=x.dtype, device=x.device)
    _check(getattr(lib(), name)(_ptr(x), _ptr(y), N * C, H, W, _glue_dtype(x, y), _stream_handle(stream)), name)
    return y


def _pool_bwd(name, x, dy, dx, stream):
    N, C, H, W = x.shape
    if dx is None:
        dx = torch.empty_like(x)
    _check(getattr(lib(), name)(_ptr(x), _ptr(dy), _ptr(dx), N * C, H, W, _glue_dtype(x, dy, dx),
                                _stream_handle(stream)), name)
    return dx


def maxpool3x3s2_fwd(x, y=None, stream=None):
    return _pool_fwd("maxpool3x3s2_fwd", x, y, stream)


def maxpool3x3s2_bwd(x, dy, dx=None, stream=None):
    return _pool_bwd("maxpool3x3s2_bwd", x, dy, dx, stream)


def relu_maxpool3x3s2_fwd(x, y=None, stream=None):
    return _pool_fwd("relu_maxpool3x3s2_fwd", x, y, stream)


def relu_maxpool3x3s2_bwd(x, dy, dx=None, stream=None):
    return _pool_bwd("relu_maxpool3x3s2_bwd", x, dy, dx, stream)


def bias_fwd(y, b, stream=None):
    """y [N,K,P,Q] += b[k] in place (b fp32)."""
    N, K, P, Q = y.shape
    if not y.is_contiguous() or b.dtype != torch.float32 or b.numel() != K:
        raise ValueError("bias_fwd takes a dense y and one fp32 value per filter")
    _check(lib().bias_fwd(_ptr(y), _ptr(b), N, K, P * Q, _dtype_of(y), _stream_handle(stream)), "bias_fwd")
    return y


def bias_bwd(dy, db=None, ws=None, stream=None):
    """db[k] = sum of dy [N,K,P,Q] over samples and positions, fp32."""
    N, K, P, Q = dy.shape
    if not dy.is_contiguous():
        raise ValueError("bias_bwd takes a dense dy")
    if db is None:
        db = torch.empty((K,), dtype=torch.float32, device=dy.device)
    buf, nbytes = _scratch(ws, int(lib().bias_bwd_workspace_bytes(N, K)), stream)
    _check(lib().bias_bwd(_ptr(dy), _ptr(db), N, K, P * Q, _dtype_of(dy), ctypes.c_void_p(buf.data_ptr()), nbytes,
                          _stream_handle(stream)), "bias_bwd")
    return db


def convert_f32_to_bf16(src, dst=None, stream=None):
    """Round an fp32 tensor to bfloat16 (nearest even) into `dst` (same shape, contiguous)."""
    if dst is None:
        dst = torch.empty(src.shape, dtype=torch.bfloat16, device=src.device)
    if not src.is_contiguous() or not dst.is_contiguous():
        raise ValueError("convert_f32_to_bf16 needs contiguous tensors")
    _check(lib().convert_f32_to_bf16(_ptr(src), _ptr(dst), src.numel(), _stream_handle(stream)), "convert_f32_to_bf16")
    return dst


def _fc_ws(op, N, I, O, ws, stream):
    """(buffer, its address, its size)"""
    buf, nbytes = _scratch(ws, int(lib().fc_workspace_bytes(op, N, I, O, DTYPE_F32)), stream)
    return buf, (buf.data_ptr() if buf is not None else 0), nbytes


def fc_fwd(x, w, bias=None, relu=False, y=None, ws=None, stream=None):
    """x [N,I], w [O,I] (fp32) -> y [N,O] = f(x w^T + bias)."""
    N, I = x.shape
    O, Iw = w.shape
    if I != Iw or (bias is not None and (bias.dtype != torch.float32 or bias.numel() != O)):
        raise ValueError("operands do not match")
    if y is None:
        y = torch.empty((N, O), dtype=torch.float32, device=x.device)
    _dense(x, w, bias, y)
    buf, wsp, nbytes = _fc_ws(OP_FWD, N, I, O, ws, stream)
    bp = _ptr(bias) if bias is not None else 0
    _check(lib().fc_fwd(_ptr(x), _ptr(w), bp, _ptr(y), N, I, O, 1 if relu else 0, _dtype_of(x), wsp, nbytes,
                        _stream_handle(stream)), "fc_fwd")
    return y


def fc_bwd_data(dy, w, dx=None, ws=None, stream=None):
    """dy [N,O], w [O,I] -> dx [N,I]."""
    N, O = dy.shape
    Ow, I = w.shape
    if O != Ow:
        raise ValueError("operands do not match")
    if dx is None:
        dx = torch.empty((N, I), dtype=torch.float32, device=dy.device)
    _dense(dy, w, dx)
    buf, wsp, nbytes = _fc_ws(OP_BWD_DATA, N, I, O, ws, stream)
    _check(lib().fc_bwd_data(_ptr(dy), _ptr(w), _ptr(dx), N, I, O, _dtype_of(dy), wsp, nbytes,
                             _stream_handle(stream)), "fc_bwd_data")
    return dx


def fc_bwd_filter(x, dy, dw=None, ws=None, stream=None):
    """x [N,I], dy [N,O] -> dw [O,I]."""
    N, I = x.shape
    Ny, O = dy.shape
    if N != Ny:
        raise ValueError("operands do not match")
    if dw is None:
        dw = torch.empty((O, I), dtype=torch.float32, device=x.device)
    _dense(x, dy, dw)
    buf, wsp, nbytes = _fc_ws(OP_BWD_FILTER, N, I, O, ws, stream)
    _check(lib().fc_bwd_filter(_ptr(x), _ptr(dy), _ptr(dw), N, I, O, _dtype_of(x), wsp, nbytes,
                               _stream_handle(stream)), "fc_bwd_filter")
    return dw


def sgd_update(w, dw, vel, lr, momentum=0.0, weight_decay=0.0, grad_scale=1.0, stream=None):
    """In place: vel = momentum*vel - lr*(weight_decay*w + grad_scale*dw); w += vel (fp32 tensors of one size)."""
    if not (w.dtype == dw.dtype == vel.dtype == torch.float32) or not (w.numel() == dw.numel() == vel.numel()):
        raise ValueError("sgd_update takes three fp32 tensors of one size")
    _dense(w, dw, vel)
    _check(lib().sgd_update(_ptr(w), _ptr(dw), _ptr(vel), w.numel(), lr, momentum, weight_decay, grad_scale,
                            _stream_handle(stream)), "sgd_update")
    return w


def sgd_update_multi(ws, dws, vels, lr, momentum=0.0, weight_decay=0.0, grad_scale=1.0, stream=None):
    """sgd_update for lists of tensors in one call (one launch per 24 tensors)."""
    n = len(ws)
    if not (len(dws) == len(vels) == n):
        raise ValueError("sgd_update_multi takes three lists of one length")
    for w, dw, vel in zip(ws, dws, vels):
        if not (w.dtype == dw.dtype == vel.dtype == torch.float32) or not (w.numel() == dw.numel() == vel.numel()):
            raise ValueError("sgd_update_multi takes fp32 tensors, each triple of one size")
        _dense(w, dw, vel)
    ptrs = lambda ts: (ctypes.c_void_p * n)(*[t.data_ptr() for t in ts])
    counts = (ctypes.c_int64 * n)(*[w.numel() for w in ws])
    _check(lib().sgd_update_multi(ptrs(ws), ptrs(dws), ptrs(vels), counts, n, lr, momentum, weight_decay, grad_scale,
                                  _stream_handle(stream)), "sgd_update_multi")
    return ws


# Workspace sizes of the calls below: kept for the same reason as those of the convolutions.
@functools.lru_cache(maxsize=1024, typed=True)
def _norm_workspace_bytes(op, N, C, S, groups, layout, dtype):
    return int(lib().group_norm_act_workspace_bytes(op, N, C, S, groups, layout, dtype))


@functools.lru_cache(maxsize=1024, typed=True)
def _loss_workspace_bytes(N, V, K, dtype):
    return int(lib().distill_loss_workspace_bytes(N, V, K, dtype))


# The checks of the calls below, and the handling of their scratch, are written out for speed: the smallest of these calls
# take the GPU less time than Python needs for their arguments.
_F32 = torch.float32
_GLUE_CODES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _glue_code(t):
    code = _GLUE_CODES.get(t.dtype)
    if code is None:
        raise TypeError("unsupported tensor dtype %s" % t.dtype)
    return code


def _on_gpu(d):
    if d < 0:
        raise ValueError("the tensors of a call must be on one GPU")


def _like(t, x, shape, d, what):
    """A tensor of x's shape, element type and GPU."""
    if t.shape != shape:
        raise ValueError("%s must have the shape of its input" % what)
    if t.dtype is not x.dtype:
        raise TypeError("the tensors of a glue call must have one dtype")
    if t.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")


def _dense_f32(t, shape, d, what):
    """A dense fp32 tensor of this shape on GPU d; its address."""
    if t.dtype is not _F32 or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a dense fp32 tensor %s" % (what, list(shape)))
    if t.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")
    return t.data_ptr()


def _new_f32(shape, like):
    return torch.empty(shape, dtype=_F32, device=like.device)


def _current_stream(stream, d):
    """_stream_handle for a call whose tensors are on GPU d (whose state is there, then: 1 us less)."""
    if torch._C._cuda_getDevice() != d or (stream is not None and stream.device_index != d):
        raise ValueError("the tensors of a call must be on the current GPU, and its stream too")
    return torch._C._cuda_getCurrentRawStream(d) if stream is None else stream.cuda_stream


def _channels_last(*tensors):
    for t in tensors:
        if not t.is_contiguous(memory_format=torch.channels_last):
            raise ValueError("the tensors of a normalisation must be dense, all NCHW or all channels last")
    return LAYOUT_CHANNELS_LAST


def group_norm_act_fwd(x, groups, gamma=None, beta=None, eps=1e-5, act="relu", y=None, mean=None, rstd=None, ws=None,
                       stream=None):
    """y = act(group norm of x) for x [N,C,H,W], NCHW or channels last in memory (y has x's order and element type), and
    the statistics that the backward pass needs: (y, mean [N,groups], rstd [N,groups]).  act: "none", "relu" or "silu";
    gamma and beta: fp32 [C], or None."""
    if type(groups) is not int:
        groups, = _whole(groups)
    N, C, H, W = shape = x.shape
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError("unknown activation %r" % (act,))
    if y is None:
        y = torch.empty_like(x)
    dtype = _glue_code(x)
    layout = LAYOUT_PLANES if x.is_contiguous() and y.is_contiguous() else _channels_last(x, y)
    d = x.get_device()
    _like(y, x, shape, d, "y")
    _on_gpu(d)
    gp = 0 if gamma is None else _dense_f32(gamma, (C,), d, "gamma")
    bp = 0 if beta is None else _dense_f32(beta, (C,), d, "beta")
    mp = rp = 0
    if groups > 0:
        per = (N, groups)
        mean = _new_f32(per, x) if mean is None else mean
        rstd = _new_f32(per, x) if rstd is None else rstd
        mp, rp = _dense_f32(mean, per, d, "mean"), _dense_f32(rstd, per, d, "rstd")
    need, wsp = _norm_workspace_bytes(OP_FWD, N, C, H * W, groups, layout, dtype), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = lib().group_norm_act_fwd(x.data_ptr(), gp, bp, y.data_ptr(), mp, rp, N, C, H * W, groups, eps, code, layout, dtype,
                                      wsp, need, handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, "group_norm_act_fwd")
    return y, mean, rstd


def group_norm_act_bwd(x, dy, mean, rstd, gamma=None, beta=None, act="relu", dx=None, dgamma=None, dbeta=None, ws=None,
                       stream=None):
    """(dx, dgamma [C], dbeta [C]) from the forward call's x, mean and rstd and the gradient dy of its y."""
    N, C, H, W = shape = x.shape
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError("unknown activation %r" % (act,))
    groups = mean.shape[1]
    if rstd.shape != mean.shape:
        raise ValueError("mean and rstd must have one shape")
    if dx is None:
        dx = torch.empty_like(x)
    dtype = _glue_code(x)
    layout = (LAYOUT_PLANES if x.is_contiguous() and dy.is_contiguous() and dx.is_contiguous()
              else _channels_last(x, dy, dx))
    d = x.get_device()
    _like(dy, x, shape, d, "dy")
    _like(dx, x, shape, d, "dx")
    _on_gpu(d)
    per, chan = (N, groups), (C,)
    mp, rp = _dense_f32(mean, per, d, "mean"), _dense_f32(rstd, per, d, "rstd")
    gp = 0 if gamma is None else _dense_f32(gamma, chan, d, "gamma")
    bp = 0 if beta is None else _dense_f32(beta, chan, d, "beta")
    dgamma = _new_f32(chan, x) if dgamma is None else dgamma
    dbeta = _new_f32(chan, x) if dbeta is None else dbeta
    dgp, dbp = _dense_f32(dgamma, chan, d, "dgamma"), _dense_f32(dbeta, chan, d, "dbeta")
    need, wsp = _norm_workspace_bytes(OP_BWD_DATA, N, C, H * W, groups, layout, dtype), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = lib().group_norm_act_bwd(x.data_ptr(), dy.data_ptr(), gp, bp, mp, rp, dx.data_ptr(), dgp, dbp, N, C, H * W, groups,
                                      code, layout, dtype, wsp, need, handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, "group_norm_act_bwd")
    return dx, dgamma, dbeta


def _too_large(what):
    """A size of 2^31 or more is refused here: ctypes would hand on its low 32 bits."""
    raise ConvError(ERR_TOO_LARGE, what)


def _rows_of(t, what):
    """(N, V, row stride) of a [N,V] tensor whose rows are dense."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1) or (shape[0] > 1 and stride[0] < shape[1]):
        raise ValueError("%s must be [N, V] with dense rows" % what)
    if shape[0] >> 31 or shape[1] >> 31:
        _too_large("a call on %s" % what)
    return shape[0], shape[1], (stride[0] if shape[0] > 1 else shape[1])


_INDEX_BYTES = {torch.int32: 4, torch.int64: 8}


def _targets(N, labels, top_idx, top_val, d):
    """(addresses of the three, K, bytes of an index, dtype code of the teacher's logits) of a loss call, its targets
    checked."""
    lp, index = 0, 4
    if labels is not None:
        index = _INDEX_BYTES.get(labels.dtype)
        if index is None:
            raise TypeError("labels must be int32 or int64")
        if labels.shape != (N,) or not labels.is_contiguous() or labels.get_device() != d:
            raise ValueError("labels must be a dense tensor with one class per row on the logits' GPU")
        lp = labels.data_ptr()
    if top_idx is None:
        if top_val is not None:
            raise ValueError("top_idx and top_val come together")
        return lp, 0, 0, 0, index, DTYPE_F32
    if top_val is None:
        raise ValueError("top_idx and top_val come together")
    of_top = _INDEX_BYTES.get(top_idx.dtype)
    if of_top is None or (labels is not None and of_top != index):
        raise TypeError("labels and top_idx must have one type, int32 or int64")
    td = _glue_code(top_val)
    shape = top_idx.shape
    if (len(shape) != 2 or shape[0] != N or top_val.shape != shape or not top_idx.is_contiguous()
            or not top_val.is_contiguous() or top_idx.get_device() != d or top_val.get_device() != d):
        raise ValueError("top_idx and top_val must be dense tensors [N, K] on the logits' GPU")
    return lp, top_idx.data_ptr(), top_val.data_ptr(), shape[1], of_top, td


def _gradient_rows(dz, z, N, V, d):
    """dz (a new one for None) and its row stride."""
    if dz is None:
        return torch.empty((N, V), dtype=z.dtype, device=z.device), V
    dN, dV, stride = _rows_of(dz, "dz")
    if dN != N or dV != V:
        raise ValueError("dz must have the shape of z")
    if dz.dtype is not z.dtype:
        raise TypeError("dz must have the element type of z")
    if dz.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")
    return dz, stride


def distill_loss_fwd(z, labels=None, top_idx=None, top_val=None, temperature=1.0, kd_weight=1.0, label_weight=1.0,
                     loss=None, stats=None, ws=None, stream=None):
    """Losses of the logits z [N,V] (fp32 or bfloat16, rows may be apart) against labels [N] and / or a teacher's top
    logits (classes top_idx [N,K], logits top_val [N,K]); indexes int32 or int64, one outside 0..V-1 for none.  Returns
    (loss [N], stats [N,3]); stats is what distill_loss_bwd takes."""
    N, V, zs = _rows_of(z, "z")
    dtype, d = _glue_code(z), z.get_device()
    lp, ip, vp, K, ib, td = _targets(N, labels, top_idx, top_val, d)
    _on_gpu(d)
    loss = _new_f32((N,), z) if loss is None else loss
    stats = _new_f32((N, 3), z) if stats is None else stats
    op, sp = _dense_f32(loss, (N,), d, "loss"), _dense_f32(stats, (N, 3), d, "stats")
    need, wsp = _loss_workspace_bytes(N, V, K, dtype), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = lib().distill_loss_fwd(z.data_ptr(), zs, lp, ip, vp, op, sp, N, V, K, temperature, kd_weight, label_weight, ib, td,
                                    dtype, wsp, need, handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, "distill_loss_fwd")
    return loss, stats


def distill_loss_bwd(z, stats, labels=None, top_idx=None, top_val=None, temperature=1.0, kd_weight=1.0, label_weight=1.0,
                     grad=None, grad_scale=1.0, dz=None, stream=None):
    """dz = grad_scale * grad[n] * d loss[n] / d z (grad [N] fp32, or None for ones) from the forward call's arguments and
    statistics.  dz has z's element type and may be z itself."""
    N, V, zs = _rows_of(z, "z")
    dtype, d = _glue_code(z), z.get_device()
    lp, ip, vp, K, ib, td = _targets(N, labels, top_idx, top_val, d)
    dz, dzs = _gradient_rows(dz, z, N, V, d)
    _on_gpu(d)
    gp = 0 if grad is None else _dense_f32(grad, (N,), d, "grad")
    sp = _dense_f32(stats, (N, 3), d, "stats")
    rc = lib().distill_loss_bwd(z.data_ptr(), zs, lp, ip, vp, sp, gp, grad_scale, dz.data_ptr(), dzs, N, V, K, temperature,
                                kd_weight, label_weight, ib, td, dtype, _current_stream(stream, d))
    if rc != OK:
        raise ConvError(rc, "distill_loss_bwd")
    return dz


def distill_loss_fwd_bwd(z, labels=None, top_idx=None, top_val=None, temperature=1.0, kd_weight=1.0, label_weight=1.0,
                         grad=None, grad_scale=1.0, loss=None, dz=None, ws=None, stream=None):
    """(loss [N], dz [N,V]) of distill_loss_fwd and distill_loss_bwd in one call."""
    N, V, zs = _rows_of(z, "z")
    dtype, d = _glue_code(z), z.get_device()
    lp, ip, vp, K, ib, td = _targets(N, labels, top_idx, top_val, d)
    dz, dzs = _gradient_rows(dz, z, N, V, d)
    _on_gpu(d)
    loss = _new_f32((N,), z) if loss is None else loss
    op = _dense_f32(loss, (N,), d, "loss")
    gp = 0 if grad is None else _dense_f32(grad, (N,), d, "grad")
    need, wsp = _loss_workspace_bytes(N, V, K, dtype), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = lib().distill_loss_fwd_bwd(z.data_ptr(), zs, lp, ip, vp, gp, grad_scale, op, dz.data_ptr(), dzs, N, V, K,
                                        temperature, kd_weight, label_weight, ib, td, dtype, wsp, need, handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, "distill_loss_fwd_bwd")
    return loss, dz


# ---------------------------------------------------------------------------------------------------------------
# Tensors held in blocks, layer normalisation, and the fully connected passes on such tensors
# ---------------------------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=1024, typed=True)
def _layer_norm_workspace_bytes(N, C, dtype):
    return int(lib().layer_norm_workspace_bytes(OP_BWD_DATA, N, C, dtype))


@functools.lru_cache(maxsize=1024, typed=True)
def _fc_kept_workspace_bytes(N, I, O, dtype):
    return int(lib().fc_kept_workspace_bytes(N, I, O, dtype))


@functools.lru_cache(maxsize=1024, typed=True)
def _fc_q4_workspace_bytes(N, I, O, dtype):
    return int(lib().fc_q4_workspace_bytes(N, I, O, dtype))


_BLOCK_BYTES = {"e4m3": 32, "e2m1": 16}
_ROW_BLOCKS = BLOCK_ROW_FILL // BLOCK_VALUES


class Blocks:
    """A tensor [N, cols] held in blocks of 32 values with a shared power of two: `codes` and `scales` (uint8, rows filled up
    to a multiple of 128 values) and the format's name, "e4m3" (8 bits) or "e2m1" (4 bits).  quantize_blocks makes one."""
    __slots__ = ("codes", "scales", "cols", "format")

    def __init__(self, codes, scales, cols, format):
        if type(cols) is not int:
            cols, = _whole(cols)
        bytes_to_32 = _BLOCK_BYTES.get(format)
        if bytes_to_32 is None:
            raise ValueError("unknown block format %r" % (format,))
        shape, blocks = codes.shape, (cols + BLOCK_ROW_FILL - 1) // BLOCK_ROW_FILL * _ROW_BLOCKS
        if codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8:
            raise TypeError("codes and scales are bytes")
        if (cols < 1 or len(shape) != 2 or shape[1] != blocks * bytes_to_32 or scales.shape != (shape[0], blocks)
                or not codes.is_contiguous() or not scales.is_contiguous()):
            raise ValueError("codes and scales must be dense, with rows of %d values and their exponents" % (blocks * BLOCK_VALUES))
        if codes.get_device() != scales.get_device():
            raise ValueError("the tensors of a call must be on one GPU")
        if shape[0] >> 31 or cols >> 31:
            _too_large("Blocks")
        self.codes, self.scales, self.cols, self.format = codes, scales, cols, format

    @classmethod
    def empty(cls, N, cols, format, device="cuda"):
        """Room for N rows of `cols` values."""
        if format not in BLOCK_FORMATS:
            raise ValueError("unknown block format %r" % (format,))
        N, cols = _whole(N, cols)
        pitch = -(-cols // BLOCK_ROW_FILL) * BLOCK_ROW_FILL
        byte = dict(dtype=torch.uint8, device=device)
        return cls(torch.empty((N, pitch if format == "e4m3" else pitch // 2), **byte),
                   torch.empty((N, pitch // BLOCK_VALUES), **byte), cols, format)

    @property
    def shape(self):
        return torch.Size((self.codes.shape[0], self.cols))

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()


def _held(q, format, what):
    if type(q) is not Blocks:
        raise TypeError("%s must be a tensor held in blocks" % what)
    if q.format != format:
        raise ValueError("%s must be held as %s" % (what, format))


def quantize_blocks(x, format, out=None, stream=None):
    """x [N,C] (fp32 or bfloat16, rows may be apart) in blocks of `format`, "e4m3" or "e2m1"."""
    N, C, xs = _rows_of(x, "x")
    dtype, d = _glue_code(x), x.get_device()
    if format not in BLOCK_FORMATS:
        raise ValueError("unknown block format %r" % (format,))
    _on_gpu(d)
    if out is None:
        out = Blocks.empty(N, C, format, x.device)
    else:
        _held(out, format, "out")
        if out.cols != C or out.codes.shape[0] != N:
            raise ValueError("out must have the shape of x")
        if out.codes.get_device() != d:
            raise ValueError("the tensors of a call must be on one GPU")
    rc = lib().quantize_blocks(x.data_ptr(), xs, out.codes.data_ptr(), out.scales.data_ptr(), N, C, BLOCK_FORMATS[format], dtype,
                               _current_stream(stream, d))
    if rc != OK:
        raise ConvError(rc, "quantize_blocks")
    return out


def dequantize_blocks(q, x=None, dtype=torch.float32, stream=None):
    """The values [N,C] of a tensor held in blocks, as fp32 or bfloat16 (exact in both), into x (its type decides) or a new
    tensor of `dtype`."""
    if type(q) is not Blocks:
        raise TypeError("q must be a tensor held in blocks")
    N, C = q.codes.shape[0], q.cols
    d = q.codes.get_device()
    if x is None:
        x = torch.empty((N, C), dtype=dtype, device=q.codes.device)
    xN, xC, xs = _rows_of(x, "x")
    code = _glue_code(x)
    if xN != N or xC != C:
        raise ValueError("x must have the shape of the tensor in blocks")
    if x.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")
    _on_gpu(d)
    rc = lib().dequantize_blocks(q.codes.data_ptr(), q.scales.data_ptr(), x.data_ptr(), xs, N, C, BLOCK_FORMATS[q.format], code,
                                 _current_stream(stream, d))
    if rc != OK:
        raise ConvError(rc, "dequantize_blocks")
    return x


def _rows_like(t, x, N, C, d, what):
    """Row stride of t, a tensor of x's shape [N,C], element type and GPU."""
    tN, tC, stride = _rows_of(t, what)
    if tN != N or tC != C:
        raise ValueError("%s must have the shape [%d, %d]" % (what, N, C))
    if t.dtype is not x.dtype:
        raise TypeError("%s must have the element type of the call's other tensors" % what)
    if t.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")
    return stride


def layer_norm_fwd(x, gamma=None, beta=None, eps=1e-5, y=None, mean=None, rstd=None, stream=None):
    """y = (x - mean) * rstd * gamma + beta for every row of x [N,C] (fp32 or bfloat16, rows may be apart), and the statistics
    that the backward pass needs: (y, mean [N], rstd [N]).  gamma and beta: fp32 [C], or None."""
    N, C, xs = _rows_of(x, "x")
    dtype, d = _glue_code(x), x.get_device()
    _on_gpu(d)
    if y is None:
        y, ys = torch.empty((N, C), dtype=x.dtype, device=x.device), C
    else:
        ys = _rows_like(y, x, N, C, d, "y")
    gp = 0 if gamma is None else _dense_f32(gamma, (C,), d, "gamma")
    bp = 0 if beta is None else _dense_f32(beta, (C,), d, "beta")
    mean = _new_f32((N,), x) if mean is None else mean
    rstd = _new_f32((N,), x) if rstd is None else rstd
    mp, rp = _dense_f32(mean, (N,), d, "mean"), _dense_f32(rstd, (N,), d, "rstd")
    rc = lib().layer_norm_fwd(x.data_ptr(), xs, gp, bp, y.data_ptr(), ys, mp, rp, N, C, eps, dtype, _current_stream(stream, d))
    if rc != OK:
        raise ConvError(rc, "layer_norm_fwd")
    return y, mean, rstd


def _layer_norm_bwd(name, source, dy, N, C, mean, rstd, gamma, dx, dgamma, dbeta, ws, stream):
    dyN, dyC, dys = _rows_of(dy, "dy")
    if dyN != N or dyC != C:
        raise ValueError("dy must have the shape [%d, %d]" % (N, C))
    dtype, d = _glue_code(dy), dy.get_device()
    _on_gpu(d)
    if dx is None:
        dx, dxs = torch.empty((N, C), dtype=dy.dtype, device=dy.device), C
    else:
        dxs = _rows_like(dx, dy, N, C, d, "dx")
    mp, rp = _dense_f32(mean, (N,), d, "mean"), _dense_f32(rstd, (N,), d, "rstd")
    gp = 0 if gamma is None else _dense_f32(gamma, (C,), d, "gamma")
    dgamma = _new_f32((C,), dy) if dgamma is None else dgamma
    dbeta = _new_f32((C,), dy) if dbeta is None else dbeta
    dgp, dbp = _dense_f32(dgamma, (C,), d, "dgamma"), _dense_f32(dbeta, (C,), d, "dbeta")
    need, wsp = _layer_norm_workspace_bytes(N, C, dtype), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = getattr(lib(), name)(*source, dy.data_ptr(), dys, gp, mp, rp, dx.data_ptr(), dxs, dgp, dbp, N, C, dtype, wsp, need,
                                  handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, name)
    return dx, dgamma, dbeta


def layer_norm_bwd(x, dy, mean, rstd, gamma=None, dx=None, dgamma=None, dbeta=None, ws=None, stream=None):
    """(dx, dgamma [C], dbeta [C]) from the forward call's x, mean and rstd and the gradient dy of its y."""
    N, C, xs = _rows_of(x, "x")
    if dy.dtype is not x.dtype:
        raise TypeError("dy must have the element type of x")
    if dy.get_device() != x.get_device():
        raise ValueError("the tensors of a call must be on one GPU")
    return _layer_norm_bwd("layer_norm_bwd", (x.data_ptr(), xs), dy, N, C, mean, rstd, gamma, dx, dgamma, dbeta, ws, stream)


def layer_norm_bwd_kept(q, dy, mean, rstd, gamma=None, dx=None, dgamma=None, dbeta=None, ws=None, stream=None):
    """layer_norm_bwd from x as it was kept in blocks of 8 bits; dx has dy's element type."""
    _held(q, "e4m3", "q")
    if dy.get_device() != q.codes.get_device():
        raise ValueError("the tensors of a call must be on one GPU")
    return _layer_norm_bwd("layer_norm_bwd_kept", (q.codes.data_ptr(), q.scales.data_ptr()), dy, q.codes.shape[0], q.cols, mean,
                           rstd, gamma, dx, dgamma, dbeta, ws, stream)


def fc_bwd_filter_kept(q, dy, dw=None, ws=None, stream=None):
    """q: x [N,I] as it was kept in blocks of 8 bits, dy [N,O] (fp32 or bfloat16) -> dw [O,I] fp32."""
    _held(q, "e4m3", "q")
    N, I = q.codes.shape[0], q.cols
    shape = dy.shape
    if len(shape) != 2 or shape[0] != N or not dy.is_contiguous():
        raise ValueError("dy must be a dense tensor with the rows of q")
    O, dtype, d = shape[1], _glue_code(dy), dy.get_device()
    if O >> 31:
        _too_large("fc_bwd_filter_kept")
    if q.codes.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")
    _on_gpu(d)
    dw = _new_f32((O, I), dy) if dw is None else dw
    wp = _dense_f32(dw, (O, I), d, "dw")
    need, wsp = _fc_kept_workspace_bytes(N, I, O, dtype), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = lib().fc_bwd_filter_kept(q.codes.data_ptr(), q.scales.data_ptr(), dy.data_ptr(), wp, N, I, O, dtype, wsp, need, handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, "fc_bwd_filter_kept")
    return dw


def fc_fwd_q4(x, w, bias=None, relu=False, y=None, ws=None, stream=None, out_bf16=False):
    """x [N,I] (fp32 or bfloat16), w [O,I] held in blocks of 4 bits -> y [N,O] = f(x w^T + bias), fp32 (or bfloat16: pass a
    bfloat16 y, or out_bf16=True, with a bfloat16 x).  x is put into blocks of 4 bits within the call."""
    _held(w, "e2m1", "w")
    O, I = w.codes.shape[0], w.cols
    shape = x.shape
    if len(shape) != 2 or shape[1] != I or not x.is_contiguous():
        raise ValueError("x must be a dense tensor with rows of %d values" % I)
    N, dtype, d = shape[0], _glue_code(x), x.get_device()
    if N >> 31:
        _too_large("fc_fwd_q4")
    if w.codes.get_device() != d:
        raise ValueError("the tensors of a call must be on one GPU")
    _on_gpu(d)
    if y is None:
        y = torch.empty((N, O), dtype=torch.bfloat16 if out_bf16 else _F32, device=x.device)
    elif y.shape != (N, O) or not y.is_contiguous() or y.get_device() != d:
        raise ValueError("y must be a dense tensor [%d, %d] on the GPU of x" % (N, O))
    code = _io_dtype(x, y)
    bp = 0 if bias is None else _dense_f32(bias, (O,), d, "bias")
    need, wsp = _fc_q4_workspace_bytes(N, I, O, code), 0
    handle, own = _current_stream(stream, d), 0
    if need:
        if ws is None:
            own = wsp = _take_scratch(need, handle)
        else:
            buf, need = ws.get(need)
            wsp = buf.data_ptr()
    try:
        rc = lib().fc_fwd_q4(x.data_ptr(), w.codes.data_ptr(), w.scales.data_ptr(), bp, y.data_ptr(), N, I, O, 1 if relu else 0, code,
                             wsp, need, handle)
    finally:
        if own:
            _give_scratch(own)
    if rc != OK:
        raise ConvError(rc, "fc_fwd_q4")
    return y
