"""Masked convolution backward pass (ReLU-derived sparsity) on MI355X.

Thin ctypes binding over libconvbwd.so, the C-ABI declared in
include/convbwd.h.  It only marshals arguments: torch tensors (device memory,
streams) become pointers; every step of the computation runs in the HIP
kernels of the library.  A non-zero status becomes CbwError.  There is no
fallback: if the library is missing, importing the binding's functions
raises.

The operations are those of arXiv 2109.07710: the data gradient computed only
where the forward ReLU footprint is live (output sparsity, Sec. III-B), the
weight gradient skipping all-zero blocks of the incoming gradient (input
sparsity), and the dense data gradient.
"""
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libconvbwd.so")

CBW_OK, CBW_ERR_INVALID_ARG, CBW_ERR_UNSUPPORTED, CBW_ERR_WORKSPACE, CBW_ERR_HIP = 0, -1, -2, -3, -4
CBW_NCHW, CBW_NHWC = 0, 1
CBW_KCRS, CBW_KRSC = 0, 1
CBW_F32, CBW_BF16 = 0, 1
CBW_OP_BWD_DATA, CBW_OP_BWD_DATA_MASKED, CBW_OP_BWD_WEIGHT, CBW_OP_FWD, CBW_OP_BWD_DATA_ELEMENTWISE = 0, 1, 2, 3, 4
CBW_OP_BWD_BOTH = 5
CBW_FLAG_NO_SKIP = 1
CBW_FLAG_SKIP_X_BLOCKS = 2
CBW_FLAG_RELU = 4
CBW_MAX_EXPERTS = 1024
CBW_NORM_NONE, CBW_NORM_RMS, CBW_NORM_LAYER = 0, 1, 2
CBW_GATE_NONE, CBW_GATE_LINEAR, CBW_GATE_SIGMOID = 0, 1, 2
CBW_GRAD_NORM_2, CBW_GRAD_NORM_INF = 0, 1

EXPORTS = ("cbw_status_string", "cbw_validate_desc", "cbw_mask_words", "cbw_dy_mask_words",
           "cbw_workspace_size", "cbw_data_tiling", "cbw_relu_mask_pack", "cbw_nonzero_mask_pack", "conv_bwd_data",
           "conv_bwd_data_masked", "conv_bwd_data_masked_noalloc", "conv_fwd_relu_mask", "conv_bwd_weight_sparse", "conv_bwd_weight_sparse_x", "conv_bwd_sparse",
           "conv_bwd_data_elementwise", "cbw_read_pixel_counts", "cbw_read_weight_work", "cbw_read_stats",
           "cbw_read_live_lists",
           "cbw_read_occupancy", "cbw_set_profile_events",
           "cbw_validate_expert_desc", "cbw_expert_workspace_size", "expert_fwd", "expert_bwd_data", "expert_bwd_weight",
           "cbw_validate_norm_desc", "cbw_norm_workspace_size", "block_norm_fwd", "block_norm_bwd",
           "cbw_grad_workspace_size", "grad_norm", "grad_clip")

_DTYPES = {"bf16": CBW_BF16, "f32": CBW_F32}


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("N", "C", "H", "W", "K", "R", "S", "P", "Q",
                 "stride_h", "stride_w", "pad_h", "pad_w", "act_layout", "w_layout", "dtype")]

    @classmethod
    def make(cls, N, C, H, W, K, R, S, stride=(1, 1), pad=(0, 0), dtype="bf16", w_layout="krsc",
             act_layout="nhwc"):
        if isinstance(stride, int):
            stride = (stride, stride)
        if isinstance(pad, int):
            pad = (pad, pad)
        P = (H + 2 * pad[0] - R) // stride[0] + 1
        Q = (W + 2 * pad[1] - S) // stride[1] + 1
        return cls(N, C, H, W, K, R, S, P, Q, stride[0], stride[1], pad[0], pad[1],
                   {"nhwc": CBW_NHWC, "nchw": CBW_NCHW}[act_layout],
                   {"krsc": CBW_KRSC, "kcrs": CBW_KCRS}[w_layout],
                   {"bf16": CBW_BF16, "f32": CBW_F32}[dtype])


class Stats(ctypes.Structure):
    _fields_ = [("rows_total", ctypes.c_int64), ("rows_live", ctypes.c_int64),
                ("blocks_total", ctypes.c_int64), ("blocks_skipped", ctypes.c_int64)]


class ExpertDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("E", "C", "K", "dtype")] + \
               [(n, ctypes.c_int64) for n in ("rows", "x_stride", "y_stride")]

    @classmethod
    def make(cls, E, rows, C, K, dtype="bf16", x_stride=None, y_stride=None):
        return cls(E, C, K, _DTYPES[dtype], rows, C if x_stride is None else x_stride,
                   K if y_stride is None else y_stride)


class NormDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "gate_rows", "res_stride", "block_stride", "gate_stride")] + \
               [(n, ctypes.c_int32) for n in ("C", "dtype", "res_dtype", "pre_norm", "post_norm", "gate_act")] + \
               [("eps", ctypes.c_float)]

    @classmethod
    def make(cls, rows, C, pre="rms", post="rms", gate="none", gate_rows=1, dtype="bf16", res_dtype="bf16", eps=1e-5,
             res_stride=None, block_stride=None, gate_stride=None):
        kinds = {"none": CBW_NORM_NONE, "rms": CBW_NORM_RMS, "layer": CBW_NORM_LAYER}
        acts = {"none": CBW_GATE_NONE, "linear": CBW_GATE_LINEAR, "sigmoid": CBW_GATE_SIGMOID}
        return cls(rows, gate_rows, *(C if s is None else s for s in (res_stride, block_stride, gate_stride)), C,
                   _DTYPES[dtype], _DTYPES[res_dtype], kinds[pre], kinds[post], acts[gate], eps)


class NormParams(ctypes.Structure):
    """Weights and biases of a block's norms and its residual scale (or their
    gradients): float32 device tensors of C values, or None.  Keeps the tensors."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("_w_pre", "_b_pre", "_w_post", "_b_post", "_scale")]

    def __init__(self, w_pre=None, b_pre=None, w_post=None, b_post=None, scale=None):
        self.tensors = (w_pre, b_pre, w_post, b_post, scale)
        sizes = {t.numel() for t in self.tensors if t is not None}
        if len(sizes) > 1:
            raise ValueError("parameters of different sizes: %s" % sorted(sizes))
        self.size = sizes.pop() if sizes else None
        super().__init__(*(None if t is None else _typed(t, CBW_F32).data_ptr() for t in self.tensors))


class _Grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class GradList:
    """The gradients of a model for grad_norm and grad_clip, and where their
    scaled values go (in place without `outs`).  Keeps the tensors: a program
    makes the list once and uses it as long as its gradients stay where they are."""

    def __init__(self, grads, outs=None):
        self.grads = list(grads)
        self.outs = self.grads if outs is None else list(outs)
        if len(self.outs) != len(self.grads):
            raise ValueError("as many outputs as gradients")
        self.array = (_Grad * max(len(self.grads), 1))()
        for i, (g, o) in enumerate(zip(self.grads, self.outs)):
            dt = _dtype_of(g)
            if o.numel() != g.numel():
                raise ValueError("an output has the size of its gradient")
            self.array[i] = _Grad(_typed(g, dt).data_ptr(), _typed(o, dt).data_ptr(), g.numel(), dt, 0)

    def __len__(self):
        return len(self.grads)


class CbwError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, status_string(status), status))


_lib = None


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libconvbwd.so is not built (%s); run __graft_entry__.build()" % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    dp = ctypes.POINTER(ConvDesc)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    L.cbw_status_string.argtypes = [ctypes.c_int]
    L.cbw_status_string.restype = ctypes.c_char_p
    L.cbw_validate_desc.argtypes = [dp]
    L.cbw_mask_words.argtypes = [dp]
    L.cbw_mask_words.restype = sz
    L.cbw_dy_mask_words.argtypes = [dp]
    L.cbw_dy_mask_words.restype = sz
    L.cbw_workspace_size.argtypes = [dp, ctypes.c_int, ctypes.POINTER(sz)]
    i32p_ = ctypes.POINTER(ctypes.c_int32)
    L.cbw_data_tiling.argtypes = [dp, i32p_, i32p_, i32p_]
    L.cbw_relu_mask_pack.argtypes = [dp, vp, vp, vp]
    L.cbw_nonzero_mask_pack.argtypes = [ctypes.c_int32, ctypes.c_int64, vp, vp, vp]
    L.conv_bwd_data.argtypes = [dp, vp, vp, vp, vp, sz, vp]
    L.conv_bwd_data_masked.argtypes = [dp, vp, vp, vp, vp, vp, sz, ctypes.c_uint32, vp]
    L.conv_bwd_data_masked_noalloc.argtypes = [dp, vp, vp, vp, vp, ctypes.c_uint32, vp]
    L.conv_fwd_relu_mask.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
    L.conv_bwd_weight_sparse.argtypes = [dp, vp, vp, vp, vp, vp, sz, ctypes.c_uint32, vp]
    L.conv_bwd_weight_sparse_x.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, ctypes.c_uint32, vp]
    L.conv_bwd_sparse.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, sz, ctypes.c_uint32, vp]
    L.conv_bwd_data_elementwise.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
    L.cbw_read_pixel_counts.argtypes = [dp, vp, sz, vp, ctypes.POINTER(ctypes.c_int64), vp]
    L.cbw_read_weight_work.argtypes = [dp, vp, sz, vp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), vp]
    L.cbw_read_stats.argtypes = [dp, ctypes.c_int, vp, sz, ctypes.POINTER(Stats), vp]
    i32p = ctypes.POINTER(ctypes.c_int32)
    L.cbw_read_live_lists.argtypes = [dp, vp, sz, ctypes.c_int, vp, i32p, i32p, vp]
    L.cbw_read_occupancy.argtypes = [dp, vp, sz, vp, i32p, i32p, i32p, i32p, vp]
    L.cbw_set_profile_events.argtypes = [ctypes.c_int, vp, vp]
    ep, np_, pp, gp = (ctypes.POINTER(t) for t in (ExpertDesc, NormDesc, NormParams, _Grad))
    u32, i32 = ctypes.c_uint32, ctypes.c_int32
    L.cbw_validate_expert_desc.argtypes = [ep]
    L.cbw_expert_workspace_size.argtypes = [ep, ctypes.POINTER(sz)]
    L.expert_fwd.argtypes = [ep, vp, vp, vp, vp, vp, vp, sz, u32, vp]
    L.expert_bwd_data.argtypes = [ep, vp, vp, vp, vp, vp, vp, sz, vp]
    L.expert_bwd_weight.argtypes = [ep, vp, vp, vp, vp, vp, sz, vp]
    L.cbw_validate_norm_desc.argtypes = [np_]
    L.cbw_norm_workspace_size.argtypes = [np_, ctypes.POINTER(sz)]
    L.block_norm_fwd.argtypes = [np_, vp, vp, vp, pp, vp, vp, vp, vp]
    L.block_norm_bwd.argtypes = [np_, vp, vp, vp, pp, vp, vp, vp, vp, vp, vp, pp, vp, sz, vp]
    L.cbw_grad_workspace_size.argtypes = [gp, i32, ctypes.POINTER(sz)]
    L.grad_norm.argtypes = [gp, i32, i32, vp, vp, sz, vp]
    L.grad_clip.argtypes = [gp, i32, i32, ctypes.c_float, vp, vp, sz, vp]
    for name in EXPORTS:
        if name != "cbw_status_string" and name not in ("cbw_mask_words", "cbw_dy_mask_words"):
            getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def status_string(status):
    return lib().cbw_status_string(status).decode()


def _check(status, where):
    if status != CBW_OK:
        raise CbwError(status, where)


def _ptr(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return ctypes.c_void_p(t.data_ptr())


def _dtype_of(t):
    """The library's type of a tensor."""
    import torch
    if t.dtype == torch.bfloat16:
        return CBW_BF16
    if t.dtype == torch.float32:
        return CBW_F32
    raise ValueError("expected a bfloat16 or float32 tensor, got %s" % t.dtype)


def _typed(t, dtype):
    """A contiguous device tensor of the library's type `dtype`, as it is."""
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    if _dtype_of(t) != dtype:
        raise ValueError("expected a %s tensor" % ("float32" if dtype == CBW_F32 else "bfloat16"))
    return t


_torch_types = None


def _types():
    """torch's types of the library's, and int32."""
    global _torch_types
    if _torch_types is None:
        import torch
        _torch_types = (torch.float32, torch.bfloat16, torch.int32)
    return _torch_types


def _rows(t, rows, cols, stride, dtype):
    """Device pointer of a row tensor [rows][cols] of the given torch type
    whose rows lie `stride` elements apart (None -> NULL)."""
    if t is None:
        return None
    if t.shape == (rows, cols) and t.dtype is dtype and t.is_cuda and t.stride() == (stride, 1):
        return t.data_ptr()
    # not the usual form: name what is wrong, or let pass where a stride has no meaning
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError("expected a tensor of shape (%d, %d), got %s" % (rows, cols, tuple(t.shape)))
    if t.dtype is not dtype:
        raise ValueError("expected a %s tensor, got %s" % (dtype, t.dtype))
    if rows > 0 and (t.stride(1) != 1 and cols > 1 or t.stride(0) != stride and rows > 1):
        raise ValueError("expected rows %d elements apart, got strides %s" % (stride, t.stride()))
    return t.data_ptr()


def _whole(t, numel, dtype):
    """Device pointer of a contiguous tensor of at least `numel` elements of
    the given torch type (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if t.dtype is not dtype or t.numel() < numel or not t.is_contiguous():
        raise ValueError("expected a contiguous %s tensor of %d elements" % (dtype, numel))
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        # the current stream's handle, without a Stream object around it
        # (2.5 us a call less) where this torch hands it out
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return ctypes.c_void_p(raw(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


# ---------------------------------------------------------------- host-only

def cbw_validate_desc(desc):
    return lib().cbw_validate_desc(ctypes.byref(desc))


def cbw_mask_words(desc):
    return lib().cbw_mask_words(ctypes.byref(desc))


def cbw_dy_mask_words(desc):
    return lib().cbw_dy_mask_words(ctypes.byref(desc))


def cbw_workspace_size(desc, op):
    n = ctypes.c_size_t(0)
    _check(lib().cbw_workspace_size(ctypes.byref(desc), op, ctypes.byref(n)), "cbw_workspace_size")
    return n.value


def cbw_data_tiling(desc):
    """(channels per tile, pixel-row capacity, pixel rows per tile) of the
    data-gradient GEMM in its dense and non-skipping modes (host only)."""
    a, b, c = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().cbw_data_tiling(ctypes.byref(desc), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)),
           "cbw_data_tiling")
    return a.value, b.value, c.value


def workspace(desc, op, device="cuda"):
    """A uint8 device tensor of the size `op` needs (allocated by torch)."""
    import torch
    return torch.empty(max(cbw_workspace_size(desc, op), 1), dtype=torch.uint8, device=device)


# ------------------------------------------------------------ device calls

def cbw_relu_mask_pack(desc, X, x_mask, stream=None):
    _check(lib().cbw_relu_mask_pack(ctypes.byref(desc), _ptr(X), _ptr(x_mask), _stream(stream)),
           "cbw_relu_mask_pack")


def cbw_nonzero_mask_pack(dtype, count, t, bits, stream=None):
    _check(lib().cbw_nonzero_mask_pack(dtype, count, _ptr(t), _ptr(bits), _stream(stream)),
           "cbw_nonzero_mask_pack")


def conv_bwd_data(desc, dY, W, dX, ws, stream=None):
    _check(lib().conv_bwd_data(ctypes.byref(desc), _ptr(dY), _ptr(W), _ptr(dX), _ptr(ws), _nbytes(ws),
                               _stream(stream)), "conv_bwd_data")


def conv_bwd_data_masked(desc, dY, W, x_mask, dX, ws, flags=0, stream=None):
    _check(lib().conv_bwd_data_masked(ctypes.byref(desc), _ptr(dY), _ptr(W), _ptr(x_mask), _ptr(dX),
                                      _ptr(ws), _nbytes(ws), flags, _stream(stream)), "conv_bwd_data_masked")


def conv_bwd_data_masked_noalloc(desc, dY, W, x_mask, dX, flags=0, stream=None):
    """conv_bwd_data_masked on the library's built-in scratch (no workspace)."""
    _check(lib().conv_bwd_data_masked_noalloc(ctypes.byref(desc), _ptr(dY), _ptr(W), _ptr(x_mask), _ptr(dX),
                                              flags, _stream(stream)), "conv_bwd_data_masked_noalloc")


def conv_fwd_relu_mask(desc, X, W, Y, y_mask, ws, stream=None):
    """Y = relu(conv(X, W)) and, when y_mask is given, its footprint bits."""
    _check(lib().conv_fwd_relu_mask(ctypes.byref(desc), _ptr(X), _ptr(W), _ptr(Y), _ptr(y_mask), _ptr(ws),
                                    _nbytes(ws), _stream(stream)), "conv_fwd_relu_mask")


def conv_bwd_weight_sparse(desc, X, dY, dy_mask, dW, ws, flags=0, stream=None):
    _check(lib().conv_bwd_weight_sparse(ctypes.byref(desc), _ptr(X), _ptr(dY), _ptr(dy_mask), _ptr(dW),
                                        _ptr(ws), _nbytes(ws), flags, _stream(stream)),
           "conv_bwd_weight_sparse")


def conv_bwd_weight_sparse_x(desc, X, dY, x_mask, dy_mask, dW, ws, flags=0, stream=None):
    _check(lib().conv_bwd_weight_sparse_x(ctypes.byref(desc), _ptr(X), _ptr(dY), _ptr(x_mask), _ptr(dy_mask),
                                          _ptr(dW), _ptr(ws), _nbytes(ws), flags, _stream(stream)),
           "conv_bwd_weight_sparse_x")


def conv_bwd_sparse(desc, X, dY, W, x_mask, dy_mask, dX, dW, ws, flags=0, stream=None):
    """Both gradients in one call (x_mask None: dense data gradient)."""
    _check(lib().conv_bwd_sparse(ctypes.byref(desc), _ptr(X), _ptr(dY), _ptr(W), _ptr(x_mask), _ptr(dy_mask),
                                 _ptr(dX), _ptr(dW), _ptr(ws), _nbytes(ws), flags, _stream(stream)),
           "conv_bwd_sparse")


def both_weight_offset(desc):
    """Byte offset of the weight-gradient part in a conv_bwd_sparse workspace."""
    return (cbw_workspace_size(desc, CBW_OP_BWD_DATA_MASKED) + 255) // 256 * 256


def conv_bwd_data_elementwise(desc, dY, W, x_mask, dX, ws, stream=None):
    _check(lib().conv_bwd_data_elementwise(ctypes.byref(desc), _ptr(dY), _ptr(W), _ptr(x_mask), _ptr(dX),
                                           _ptr(ws), _nbytes(ws), _stream(stream)), "conv_bwd_data_elementwise")


def cbw_read_pixel_counts(desc, ws, stream=None):
    """Per-pixel (tap, k) product counts of the last conv_bwd_data_elementwise
    call on ws (numpy int32 [N*H*W]) and their sum."""
    import numpy as np
    out = np.zeros(desc.N * desc.H * desc.W, np.int32)
    tot = ctypes.c_int64(0)
    _check(lib().cbw_read_pixel_counts(ctypes.byref(desc), _ptr(ws), _nbytes(ws),
                                       out.ctypes.data_as(ctypes.c_void_p), ctypes.byref(tot), _stream(stream)),
           "cbw_read_pixel_counts")
    return out, tot.value


def cbw_read_weight_work(desc, ws, stream=None):
    """Blocks executed per weight-gradient work item: numpy int32 [nsplit][ntiles]."""
    import numpy as np
    ns, nt = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().cbw_read_weight_work(ctypes.byref(desc), _ptr(ws), _nbytes(ws), None, ctypes.byref(ns),
                                      ctypes.byref(nt), _stream(stream)), "cbw_read_weight_work")
    out = np.zeros((ns.value, nt.value), np.int32)
    _check(lib().cbw_read_weight_work(ctypes.byref(desc), _ptr(ws), _nbytes(ws), out.ctypes.data_as(ctypes.c_void_p),
                                      ctypes.byref(ns), ctypes.byref(nt), _stream(stream)), "cbw_read_weight_work")
    return out


def cbw_read_stats(desc, op, ws, stream=None):
    st = Stats()
    _check(lib().cbw_read_stats(ctypes.byref(desc), op, _ptr(ws), _nbytes(ws), ctypes.byref(st),
                                _stream(stream)), "cbw_read_stats")
    return st


def cbw_read_live_lists(desc, ws, group, stream=None):
    """The compacted live-pixel list of one channel group (numpy int32) and the group width."""
    import numpy as np
    n, g = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().cbw_read_live_lists(ctypes.byref(desc), _ptr(ws), _nbytes(ws), group, None, ctypes.byref(n),
                                     ctypes.byref(g), _stream(stream)), "cbw_read_live_lists")
    out = np.zeros(max(n.value, 1), np.int32)
    _check(lib().cbw_read_live_lists(ctypes.byref(desc), _ptr(ws), _nbytes(ws), group,
                                     out.ctypes.data_as(ctypes.c_void_p), ctypes.byref(n), ctypes.byref(g),
                                     _stream(stream)), "cbw_read_live_lists")
    return out[: n.value], g.value


def cbw_read_occupancy(desc, ws, stream=None):
    """The dY block occupancy map [nchunks][ktiles] (numpy uint8), chunk pixels and k-tile width."""
    import numpy as np
    nc, kt, cp, kw = (ctypes.c_int32(0) for _ in range(4))
    args = (ctypes.byref(nc), ctypes.byref(kt), ctypes.byref(cp), ctypes.byref(kw))
    _check(lib().cbw_read_occupancy(ctypes.byref(desc), _ptr(ws), _nbytes(ws), None, *args, _stream(stream)),
           "cbw_read_occupancy")
    out = np.zeros((nc.value, kt.value), np.uint8)
    _check(lib().cbw_read_occupancy(ctypes.byref(desc), _ptr(ws), _nbytes(ws),
                                    out.ctypes.data_as(ctypes.c_void_p), *args, _stream(stream)),
           "cbw_read_occupancy")
    return out, cp.value, kw.value


def cbw_set_profile_events(op, start=None, stop=None):
    """Record events `start`/`stop` around the op's main GEMM kernel on every
    following call of this thread (None, None switches it off): torch.cuda.Event
    objects (recorded once, so that they exist) or raw hipEvent_t handles
    (int)."""
    def handle(e):
        if e is None:
            return None
        return ctypes.c_void_p(e if isinstance(e, int) else e.cuda_event)
    sp, tp = handle(start), handle(stop)
    _check(lib().cbw_set_profile_events(op, sp, tp), "cbw_set_profile_events")


# ------------------------------------------------- products grouped by expert

def _bytes(call, arg, *more):
    n = ctypes.c_size_t(0)
    _check(getattr(lib(), call)(arg, *more, ctypes.byref(n)), call)
    return n.value


def _workspace_of(nbytes, device):
    import torch
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def cbw_validate_expert_desc(desc):
    return lib().cbw_validate_expert_desc(ctypes.byref(desc))


def cbw_expert_workspace_size(desc):
    return _bytes("cbw_expert_workspace_size", ctypes.byref(desc))


def expert_workspace(desc, device="cuda"):
    """A uint8 device tensor of the size the three expert calls need."""
    return _workspace_of(cbw_expert_workspace_size(desc), device)


def _filters(d, W, dtype):
    if W.shape != (d.E, d.K, d.C):
        raise ValueError("expected filters of shape (%d, %d, %d), got %s" % (d.E, d.K, d.C, tuple(W.shape)))
    return _whole(W, 0, dtype)


def expert_fwd(desc, X, W, offsets, Y, y_mask, ws, flags=0, stream=None):
    """Y = X W[e]^T for the rows of every expert e, [offsets[e], offsets[e+1])
    (offsets: int32 on the device); CBW_FLAG_RELU: its ReLU, and y_mask its
    footprint bits (int32 words, or None)."""
    d, types = desc, _types()
    dt, rows, C, K = types[d.dtype], d.rows, d.C, d.K
    _check(lib().expert_fwd(ctypes.byref(d), _rows(X, rows, C, d.x_stride, dt), _filters(d, W, dt),
                            _whole(offsets, d.E + 1, types[2]), _rows(Y, rows, K, d.y_stride, dt),
                            _whole(y_mask, (rows * K + 31) // 32, types[2]), _ptr(ws), _nbytes(ws), flags,
                            _stream(stream)), "expert_fwd")


def expert_bwd_data(desc, dY, W, offsets, x_mask, dX, ws, stream=None):
    """dX = dY W[e], +0.0 where x_mask (None: everywhere live) is dead."""
    d, types = desc, _types()
    dt, rows, C, K = types[d.dtype], d.rows, d.C, d.K
    _check(lib().expert_bwd_data(ctypes.byref(d), _rows(dY, rows, K, d.y_stride, dt), _filters(d, W, dt),
                                 _whole(offsets, d.E + 1, types[2]), _whole(x_mask, (rows * C + 31) // 32, types[2]),
                                 _rows(dX, rows, C, d.x_stride, dt), _ptr(ws), _nbytes(ws), _stream(stream)),
           "expert_bwd_data")


def expert_bwd_weight(desc, X, dY, offsets, dW, ws, stream=None):
    """dW[e] = dY^T X over the rows of every expert e, float32 [E][K][C]."""
    d, types = desc, _types()
    dt, rows, C, K = types[d.dtype], d.rows, d.C, d.K
    _check(lib().expert_bwd_weight(ctypes.byref(d), _rows(X, rows, C, d.x_stride, dt), _rows(dY, rows, K, d.y_stride, dt),
                                   _whole(offsets, d.E + 1, types[2]), _filters(d, dW, types[CBW_F32]), _ptr(ws),
                                   _nbytes(ws), _stream(stream)), "expert_bwd_weight")


# -------------------------------- norms around a block, gate, residual scale

def cbw_validate_norm_desc(desc):
    return lib().cbw_validate_norm_desc(ctypes.byref(desc))


def cbw_norm_workspace_size(desc):
    return _bytes("cbw_norm_workspace_size", ctypes.byref(desc))


def norm_workspace(desc, device="cuda"):
    """A uint8 device tensor of the size block_norm_bwd needs."""
    return _workspace_of(cbw_norm_workspace_size(desc), device)


def _params(p, C):
    if p is None:
        return None
    if p.size is not None and p.size != C:
        raise ValueError("expected parameters of %d values, got %d" % (C, p.size))
    return ctypes.byref(p)


def block_norm_fwd(desc, x, u, gate, params, y, h, stats=None, stream=None):
    """y = x + scale * act(gate) * N_post(u), h = N_pre(y); u, gate and y None:
    h = N_pre(x).  stats (float32 [rows][4], or None): what the backward needs."""
    d, types = desc, _types()
    rows, C, rs, bs, rt, bt = d.rows, d.C, d.res_stride, d.block_stride, types[d.res_dtype], types[d.dtype]
    _check(lib().block_norm_fwd(ctypes.byref(d), _rows(x, rows, C, rs, rt), _rows(u, rows, C, bs, bt),
                                _rows(gate, -(-rows // d.gate_rows), C, d.gate_stride, bt), _params(params, C),
                                _rows(y, rows, C, rs, rt), _rows(h, rows, C, bs, bt), _whole(stats, 4 * rows, types[CBW_F32]),
                                _stream(stream)), "block_norm_fwd")


def block_norm_bwd(desc, y, u, gate, params, stats, dy, dh, dx, du, dgate, grads, ws, stream=None):
    """The gradients of block_norm_fwd's inputs from dy and dh; dy, du, dgate
    and each of grads (a NormParams) may be None."""
    d, types = desc, _types()
    rows, C, rs, bs, rt, bt = d.rows, d.C, d.res_stride, d.block_stride, types[d.res_dtype], types[d.dtype]
    gates, gs = -(-rows // d.gate_rows), d.gate_stride
    _check(lib().block_norm_bwd(ctypes.byref(d), _rows(y, rows, C, rs, rt), _rows(u, rows, C, bs, bt),
                                _rows(gate, gates, C, gs, bt), _params(params, C), _whole(stats, 4 * rows, types[CBW_F32]),
                                _rows(dy, rows, C, rs, rt), _rows(dh, rows, C, bs, bt), _rows(dx, rows, C, rs, rt),
                                _rows(du, rows, C, bs, bt), _rows(dgate, gates, C, gs, bt), _params(grads, C), _ptr(ws),
                                _nbytes(ws), _stream(stream)), "block_norm_bwd")


# ---------------------------------------- norm and clipping of all gradients

_KINDS = {"2": CBW_GRAD_NORM_2, "inf": CBW_GRAD_NORM_INF}


def cbw_grad_workspace_size(grads):
    return _bytes("cbw_grad_workspace_size", grads.array, len(grads))


def grad_workspace(grads, device="cuda"):
    """A uint8 device tensor of the size grad_norm and grad_clip need."""
    return _workspace_of(cbw_grad_workspace_size(grads), device)


def grad_norm(grads, norm, ws, kind="2", stream=None):
    """norm[0] = the norm ("2" or "inf") of a GradList's tensors taken together."""
    _check(lib().grad_norm(grads.array, len(grads.grads), _KINDS[kind], _whole(norm, 1, _types()[CBW_F32]), _ptr(ws),
                           _nbytes(ws), _stream(stream)), "grad_norm")


def grad_clip(grads, max_norm, norm, ws, kind="2", stream=None):
    """The GradList's outputs = its gradients times min(1, max_norm / (norm +
    1e-6)); norm (float32, on the device) = the norm and that factor."""
    _check(lib().grad_clip(grads.array, len(grads.grads), _KINDS[kind], max_norm, _whole(norm, 2, _types()[CBW_F32]),
                           _ptr(ws), _nbytes(ws), _stream(stream)), "grad_clip")
