"""Python binding of libfcngrad (fp16 FCN training-step hot path, gfx950).

Argument marshalling only: every call forwards device pointers of torch
tensors and the current HIP stream to the C ABI declared in
``include/fcngrad.h``; all arithmetic runs in the library's HIP kernels.
PyTorch provides device memory and streams. The library is loaded from
this directory; a missing library raises ``LibraryNotBuilt`` — there is no
fallback path.
"""
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfcngrad.so")

FG_OK, FG_EINVAL, FG_EUNSUPPORTED, FG_EWORKSPACE, FG_ELAUNCH = range(5)
EPI_NONE, EPI_RELU, EPI_GATE, EPI_ACC = 0, 1, 2, 3
OP_FWD, OP_BWD_DATA, OP_BWD_WEIGHT, OP_CONVT = 0, 1, 2, 3
MAX_SEGMENTS = 64
GRAD_F32, GRAD_F16_SCALED = 0, 1
F16, BF16, F32 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_GELU = 0, 1, 2

ENTRY_POINTS = (
    "conv2d_fwd", "conv2d_bwd_data", "conv2d_bwd_weight",
    "conv2d_bwd_weight_checked", "conv_transpose2d_fwd", "grad_group_pack", "grad_unscale_check",
    "grad_group_unpack", "l2_head_grad", "relu_backward",
    "fg_conv_workspace_bytes", "fg_conv_out_dims", "grad_group_plan",
    "fg_conv_kernel_name", "fg_status_string",
    "lars_adam_update", "lars_adam_norms", "lars_adam_apply",
    "fg_lars_adam_workspace_bytes",
    "huber_head_grad", "avg_pool2d_fwd", "avg_pool2d_bwd", "channel_slice_copy",
    "grad_flags_clear", "fg_loss_scale_update", "fg_lr_at", "fg_profile_next_launch",
    "conv2d_bwd_weight_noalloc", "fg_mfma_loop",
    "dropout_fwd", "dropout_bwd",
    "linear_xent_fwd", "linear_xent_grad", "fg_linear_xent_workspace_bytes",
    "act8_pack", "act8_unpack", "fg_act8_bytes",
    "layer_norm_fwd", "layer_norm_bwd", "fg_layer_norm_workspace_bytes",
    "linear_fwd", "linear_bwd", "fg_linear_workspace_bytes",
)
MFMA_LOOP_MAX_WORK = 1 << 28  # blocks * iters accepted by fg_mfma_loop
MFMA_LOOP_FLOPS_PER_BLOCK_ITER = 1 << 20
NOALLOC_SCRATCH_BYTES = 64 << 20


class OptTensor(ctypes.Structure):
    """fg_opt_tensor: one layer's device arrays for lars_adam_update."""
    _fields_ = [("w32", ctypes.c_uint64), ("w16", ctypes.c_uint64),
                ("m", ctypes.c_uint64), ("v", ctypes.c_uint64),
                ("g", ctypes.c_uint64), ("numel", ctypes.c_uint64)]


class OptParams(ctypes.Structure):
    """fg_opt_params."""
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float),
                ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]


class LossScaleState(ctypes.Structure):
    """fg_loss_scale: backoff loss-scale state."""
    _fields_ = [("scale", ctypes.c_double), ("clean", ctypes.c_int32),
                ("interval", ctypes.c_int32), ("s_min", ctypes.c_double),
                ("s_max", ctypes.c_double)]


class LRScheduleParams(ctypes.Structure):
    """fg_lr_schedule."""
    _fields_ = [("base", ctypes.c_double), ("peak", ctypes.c_double),
                ("warmup", ctypes.c_int64), ("every", ctypes.c_int64),
                ("rate", ctypes.c_double)]


class DropoutDesc(ctypes.Structure):
    """fg_dropout_desc. Strides 0: dense."""
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("x_ld", ctypes.c_int64), ("y_ld", ctypes.c_int64),
                ("z_ld", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("p", ctypes.c_double), ("site", ctypes.c_uint32),
                ("step", ctypes.c_uint32), ("dtype", ctypes.c_int32)]

    @classmethod
    def make(cls, rows, cols, p, seed, site=0, step=0, dtype=F16, x_ld=0, y_ld=0, z_ld=0):
        return cls(rows, cols, x_ld, y_ld, z_ld, seed, p, site, step, dtype)


class XentDesc(ctypes.Structure):
    """fg_xent_desc. Strides 0: dense."""
    _fields_ = [("rows", ctypes.c_int64), ("h_ld", ctypes.c_int64),
                ("w_ld", ctypes.c_int64), ("dh_ld", ctypes.c_int64),
                ("dw_ld", ctypes.c_int64), ("scale", ctypes.c_double),
                ("hidden", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("mean", ctypes.c_int32)]

    @classmethod
    def make(cls, rows, hidden, vocab, dtype=F16, mean=True, scale=1.0, h_ld=0, w_ld=0,
             dh_ld=0, dw_ld=0):
        return cls(rows, h_ld, w_ld, dh_ld, dw_ld, scale, hidden, vocab, dtype, int(mean))


class Act8Desc(ctypes.Structure):
    """fg_act8_desc. Stride 0: dense."""
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("x_ld", ctypes.c_int64),
                ("dtype", ctypes.c_int32)]

    @classmethod
    def make(cls, rows, cols, dtype=F16, x_ld=0):
        return cls(rows, cols, x_ld, dtype)


class NormDesc(ctypes.Structure):
    """fg_norm_desc. Strides 0: dense."""
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("x_ld", ctypes.c_int64),
                ("y_ld", ctypes.c_int64), ("add_ld", ctypes.c_int64),
                ("dx_ld", ctypes.c_int64), ("eps", ctypes.c_double), ("dtype", ctypes.c_int32)]

    @classmethod
    def make(cls, rows, cols, eps=1e-5, dtype=F16, x_ld=0, y_ld=0, add_ld=0, dx_ld=0):
        return cls(rows, cols, x_ld, y_ld, add_ld, dx_ld, eps, dtype)


class LinearDesc(ctypes.Structure):
    """fg_linear_desc. Strides 0: dense."""
    _fields_ = [("rows", ctypes.c_int64), ("x_ld", ctypes.c_int64), ("w_ld", ctypes.c_int64),
                ("y_ld", ctypes.c_int64), ("r_ld", ctypes.c_int64), ("z_ld", ctypes.c_int64),
                ("dx_ld", ctypes.c_int64), ("dw_ld", ctypes.c_int64),
                ("fan_in", ctypes.c_int32), ("fan_out", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("act", ctypes.c_int32)]

    @classmethod
    def make(cls, rows, fan_in, fan_out, dtype=F16, act=ACT_NONE, x_ld=0, w_ld=0, y_ld=0, r_ld=0,
             z_ld=0, dx_ld=0, dw_ld=0):
        return cls(rows, x_ld, w_ld, y_ld, r_ld, z_ld, dx_ld, dw_ld, fan_in, fan_out, dtype, act)


class LibraryNotBuilt(RuntimeError):
    pass


class FgError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__(f"{fn}: {status_string(status)}")


class ConvDesc(ctypes.Structure):
    """fg_conv_desc. x_ld / y_ld: pixel strides of the x- and y-shaped
    tensors (0: dense), honoured where that tensor is the pass's output and
    for x where the forward pass and the kernel gradient read it."""
    _fields_ = [(f, ctypes.c_int32) for f in
                ("n", "h", "w", "c", "k", "r", "s", "stride_h", "stride_w",
                 "pad_h", "pad_w", "x_ld", "y_ld")]

    @classmethod
    def make(cls, n, h, w, c, k, r, s, stride=1, pad=0, x_ld=0, y_ld=0):
        return cls(n, h, w, c, k, r, s, stride, stride, pad, pad, x_ld, y_ld)


class Segment(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_uint64), ("numel", ctypes.c_uint64),
                ("offset", ctypes.c_uint64)]


_lib = None


def lib():
    """Load libfcngrad.so (once) and declare every entry point."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise LibraryNotBuilt(
            f"{LIB_PATH} is missing; build it with "
            "`python -m paper_1909_11150_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, u64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_size_t
    pdesc = ctypes.POINTER(ConvDesc)
    pseg = ctypes.POINTER(Segment)
    sigs = {
        "conv2d_fwd": [pdesc, vp, vp, vp, i32, vp, vp, sz, vp],
        "conv2d_bwd_data": [pdesc, vp, vp, vp, i32, vp, vp, sz, vp],
        "conv2d_bwd_weight": [pdesc, vp, vp, vp, vp, sz, vp],
        "conv2d_bwd_weight_checked": [pdesc, vp, vp, vp, vp, vp, sz, vp],
        "conv2d_bwd_weight_noalloc": [pdesc, vp, vp, vp, vp],
        "conv_transpose2d_fwd": [pdesc, vp, vp, vp, i32, vp, vp, sz, vp],
        "grad_group_pack": [pseg, i32, vp, u64, vp],
        "grad_unscale_check": [vp, u64, ctypes.c_float, vp, vp, vp],
        "grad_group_unpack": [vp, u64, pseg, i32, vp],
        "l2_head_grad": [vp, vp, u64, ctypes.c_double, vp, vp],
        "relu_backward": [vp, vp, u64, vp, vp],
        "grad_flags_clear": [vp, i32, vp],
        "fg_loss_scale_update": [ctypes.POINTER(LossScaleState), i32, ctypes.POINTER(i32)],
        "fg_lr_at": [ctypes.POINTER(LRScheduleParams), ctypes.c_int64,
                     ctypes.POINTER(ctypes.c_double)],
        "fg_profile_next_launch": [vp, vp],
        "fg_mfma_loop": [vp, i32, i32, i32, vp],
        "huber_head_grad": [vp, vp, u64, ctypes.c_double, ctypes.c_double, vp, vp],
        "dropout_fwd": [ctypes.POINTER(DropoutDesc), vp, vp, vp, vp, vp],
        "dropout_bwd": [ctypes.POINTER(DropoutDesc), vp, vp, vp, vp, vp],
        "linear_xent_fwd": [ctypes.POINTER(XentDesc)] + [vp] * 8 + [sz, vp],
        "linear_xent_grad": [ctypes.POINTER(XentDesc)] + [vp] * 11 + [sz, vp],
        "act8_pack": [ctypes.POINTER(Act8Desc), vp, vp, vp],
        "act8_unpack": [ctypes.POINTER(Act8Desc), vp, vp, vp],
        "layer_norm_fwd": [ctypes.POINTER(NormDesc)] + [vp] * 7,
        "layer_norm_bwd": [ctypes.POINTER(NormDesc)] + [vp] * 11 + [sz, vp],
        "linear_fwd": [ctypes.POINTER(LinearDesc)] + [vp] * 8 + [sz, vp],
        "linear_bwd": [ctypes.POINTER(LinearDesc)] + [vp] * 11 + [sz, vp],
        "avg_pool2d_fwd": [vp, i32, i32, i32, i32, vp, vp],
        "avg_pool2d_bwd": [vp, vp, i32, i32, i32, i32, vp, vp],
        "channel_slice_copy": [vp, i32, vp, i32, vp, i32, ctypes.c_int64, i32, i32, vp],
        "fg_conv_out_dims": [pdesc, ctypes.c_int, ctypes.POINTER(i32),
                             ctypes.POINTER(i32)],
        "grad_group_plan": [ctypes.POINTER(u64), i32, u64, ctypes.c_uint32,
                            ctypes.c_uint32, ctypes.POINTER(i32),
                            ctypes.POINTER(u64), ctypes.POINTER(i32),
                            ctypes.POINTER(u64)],
    }
    for name, args in sigs.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    L.lars_adam_update.argtypes = [ctypes.POINTER(OptTensor), i32,
                                   ctypes.POINTER(OptParams), vp, i32, vp, vp, sz, vp]
    L.lars_adam_update.restype = ctypes.c_int
    L.lars_adam_norms.argtypes = [ctypes.POINTER(OptTensor), i32, i32, i32,
                                  ctypes.POINTER(OptParams), i32, ctypes.c_float, vp,
                                  vp, sz, vp]
    L.lars_adam_norms.restype = ctypes.c_int
    L.lars_adam_apply.argtypes = [ctypes.POINTER(OptTensor), i32, i32, i32,
                                  ctypes.POINTER(OptParams), i32, ctypes.c_float, vp,
                                  i32, vp, vp, sz, vp]
    L.lars_adam_apply.restype = ctypes.c_int
    L.fg_lars_adam_workspace_bytes.argtypes = [ctypes.POINTER(OptTensor), i32]
    L.fg_lars_adam_workspace_bytes.restype = ctypes.c_size_t
    L.fg_linear_xent_workspace_bytes.argtypes = [ctypes.POINTER(XentDesc), ctypes.c_int]
    L.fg_linear_xent_workspace_bytes.restype = ctypes.c_size_t
    L.fg_act8_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64]
    L.fg_act8_bytes.restype = ctypes.c_size_t
    L.fg_layer_norm_workspace_bytes.argtypes = [ctypes.POINTER(NormDesc)]
    L.fg_layer_norm_workspace_bytes.restype = ctypes.c_size_t
    L.fg_linear_workspace_bytes.argtypes = [ctypes.POINTER(LinearDesc), ctypes.c_int]
    L.fg_linear_workspace_bytes.restype = ctypes.c_size_t
    L.fg_conv_workspace_bytes.argtypes = [pdesc, ctypes.c_int]
    L.fg_conv_workspace_bytes.restype = ctypes.c_size_t
    L.fg_conv_kernel_name.argtypes = [pdesc, ctypes.c_int]
    L.fg_conv_kernel_name.restype = ctypes.c_char_p
    L.fg_status_string.argtypes = [ctypes.c_int]
    L.fg_status_string.restype = ctypes.c_char_p
    _lib = L
    return L


def status_string(status):
    return lib().fg_status_string(status).decode()


def _check(fn, status):
    if status != FG_OK:
        raise FgError(fn, status)


def _p(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libfcngrad must be contiguous")
    return t.data_ptr()


_raw_stream = None  # () -> handle of the current device's current stream


def _s(stream):
    """Stream handle of a call: the caller's, or torch's current one, asked for without
    making a Stream object (3 of the 8 microseconds that a small call takes)."""
    if stream is not None:
        return stream
    if _raw_stream is None:
        return _find_stream()
    return _raw_stream()


def _find_stream():
    global _raw_stream
    import torch
    get, device = (getattr(torch._C, k, None)
                   for k in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
    if get is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    _raw_stream = lambda: get(device())
    return _raw_stream()


# ---- convolution passes ---------------------------------------------------
def kernel_name(desc, op):
    """Main kernel the pass launches for this shape (for grouping timings)."""
    return lib().fg_conv_kernel_name(ctypes.byref(desc), op).decode()


def workspace_bytes(desc, op):
    return lib().fg_conv_workspace_bytes(ctypes.byref(desc), op)


def out_dims(desc, transpose=False):
    p, q = ctypes.c_int32(), ctypes.c_int32()
    _check("fg_conv_out_dims", lib().fg_conv_out_dims(
        ctypes.byref(desc), int(transpose), ctypes.byref(p), ctypes.byref(q)))
    return p.value, q.value


def _ws(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


def conv2d_fwd(desc, x, w, y, epi=EPI_NONE, gate=None, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check("conv2d_fwd", lib().conv2d_fwd(
        ctypes.byref(desc), _p(x), _p(w), _p(y), epi, _p(gate), wp, wb, _s(stream)))


def conv2d_bwd_data(desc, dy, w, dx, epi=EPI_NONE, gate=None, ws=None,
                    stream=None):
    wp, wb = _ws(ws)
    _check("conv2d_bwd_data", lib().conv2d_bwd_data(
        ctypes.byref(desc), _p(dy), _p(w), _p(dx), epi, _p(gate), wp, wb,
        _s(stream)))


def conv2d_bwd_weight(desc, x, dy, dw, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check("conv2d_bwd_weight", lib().conv2d_bwd_weight(
        ctypes.byref(desc), _p(x), _p(dy), _p(dw), wp, wb, _s(stream)))


def conv2d_bwd_weight_noalloc(desc, x, dy, dw, stream=None):
    """conv2d_bwd_weight with its split partials in the library's static
    scratch: no workspace argument, nothing allocated."""
    _check("conv2d_bwd_weight_noalloc", lib().conv2d_bwd_weight_noalloc(
        ctypes.byref(desc), _p(x), _p(dy), _p(dw), _s(stream)))


def conv2d_bwd_weight_checked(desc, x, dy, dw, found_nonfinite, ws=None,
                              stream=None):
    """conv2d_bwd_weight that also sets the device int32 found_nonfinite to 1
    if a written dW element is +-inf or NaN; dw may be a view into a group
    buffer (zero-copy pack)."""
    wp, wb = _ws(ws)
    _check("conv2d_bwd_weight_checked", lib().conv2d_bwd_weight_checked(
        ctypes.byref(desc), _p(x), _p(dy), _p(dw), _p(found_nonfinite), wp, wb,
        _s(stream)))


def opt_tensors(w32, w16, m, v, g):
    """fg_opt_tensor array for lists of per-layer torch tensors."""
    n = len(w32)
    arr = (OptTensor * n)(*[OptTensor(w32[i].data_ptr(), w16[i].data_ptr(),
                                      m[i].data_ptr(), v[i].data_ptr(),
                                      g[i].data_ptr(), w32[i].numel())
                            for i in range(n)])
    return arr


def lars_adam_workspace_bytes(tensors):
    return lib().fg_lars_adam_workspace_bytes(tensors, len(tensors))


def lars_adam_update(tensors, lr, flags, step_count, ws, beta1=0.9, beta2=0.999,
                     eps=1e-8, weight_decay=1e-4, stream=None):
    """Layer-wise adaptive Adam step (see include/fcngrad.h). tensors: from
    opt_tensors(); flags: device int32 tensor of the step's group flags (or
    None); step_count: device int32 tensor of one element."""
    p = OptParams(lr, beta1, beta2, eps, weight_decay)
    wp, wb = _ws(ws)
    nf = 0 if flags is None else flags.numel()
    _check("lars_adam_update", lib().lars_adam_update(
        tensors, len(tensors), ctypes.byref(p), _p(flags), nf, _p(step_count),
        wp, wb, _s(stream)))


def lars_adam_norms(tensors, first, count, step_count, ws, grad_format=GRAD_F32,
                    grad_inv_scale=1.0, beta1=0.9, beta2=0.999, eps=1e-8,
                    weight_decay=1e-4, stream=None):
    """Partial norms of layers [first, first + count) (see include/fcngrad.h);
    the learning rate does not enter."""
    p = OptParams(0.0, beta1, beta2, eps, weight_decay)
    wp, wb = _ws(ws)
    _check("lars_adam_norms", lib().lars_adam_norms(
        tensors, len(tensors), first, count, ctypes.byref(p), grad_format,
        grad_inv_scale, _p(step_count), wp, wb, _s(stream)))


def lars_adam_apply(tensors, lr, flags, step_count, ws, grad_format=GRAD_F32,
                    grad_inv_scale=1.0, beta1=0.9, beta2=0.999, eps=1e-8,
                    weight_decay=1e-4, first=0, count=None, stream=None):
    """Update of layers [first, first + count) (default: all) once
    lars_adam_norms has covered every layer."""
    p = OptParams(lr, beta1, beta2, eps, weight_decay)
    wp, wb = _ws(ws)
    nf = 0 if flags is None else flags.numel()
    if count is None:
        count = len(tensors) - first
    _check("lars_adam_apply", lib().lars_adam_apply(
        tensors, len(tensors), first, count, ctypes.byref(p), grad_format, grad_inv_scale,
        _p(flags), nf, _p(step_count), wp, wb, _s(stream)))


def conv_transpose2d_fwd(desc, x, w, y, epi=EPI_NONE, gate=None, ws=None,
                         stream=None):
    wp, wb = _ws(ws)
    _check("conv_transpose2d_fwd", lib().conv_transpose2d_fwd(
        ctypes.byref(desc), _p(x), _p(w), _p(y), epi, _p(gate), wp, wb,
        _s(stream)))


# ---- gradient path --------------------------------------------------------
def _segments(tensors, offsets):
    arr = (Segment * len(tensors))()
    for i, (t, off) in enumerate(zip(tensors, offsets)):
        arr[i] = Segment(_p(t), t.numel(), off)
    return arr


def grad_group_pack(srcs, offsets, group, stream=None):
    segs = _segments(srcs, offsets)
    _check("grad_group_pack", lib().grad_group_pack(
        segs, len(srcs), _p(group), group.numel(), _s(stream)))


def grad_unscale_check(group, inv_scale, out_f32, flag, numel=None,
                       stream=None):
    n = group.numel() if numel is None else numel
    _check("grad_unscale_check", lib().grad_unscale_check(
        _p(group), n, float(inv_scale), _p(out_f32), _p(flag), _s(stream)))


def grad_group_unpack(group_f32, dsts, offsets, stream=None):
    segs = _segments(dsts, offsets)
    _check("grad_group_unpack", lib().grad_group_unpack(
        _p(group_f32), group_f32.numel(), segs, len(dsts), _s(stream)))


def l2_head_grad(y, t, scale, dy, stream=None):
    _check("l2_head_grad", lib().l2_head_grad(
        _p(y), _p(t), y.numel(), float(scale), _p(dy), _s(stream)))


def huber_head_grad(y, t, scale, delta, dy, stream=None):
    """dy = fp16(scale * clamp(y - t, -delta, delta)); scale = S / numel for
    the loss-scaled mean Huber loss."""
    _check("huber_head_grad", lib().huber_head_grad(
        _p(y), _p(t), y.numel(), float(scale), float(delta), _p(dy), _s(stream)))


def avg_pool2d_fwd(x, y, stream=None):
    """2x2 stride-2 mean pooling of an N x H x W x C fp16 tensor."""
    n, h, w, c = x.shape
    _check("avg_pool2d_fwd", lib().avg_pool2d_fwd(_p(x), n, h, w, c, _p(y), _s(stream)))


def avg_pool2d_bwd(dy, dx, gate=None, stream=None):
    """Gradient of avg_pool2d_fwd into dx (the forward input's shape),
    zero where gate <= 0 if a gate is given."""
    n, h, w, c = dx.shape
    _check("avg_pool2d_bwd", lib().avg_pool2d_bwd(
        _p(dy), _p(gate), n, h, w, c, _p(dx), _s(stream)))


def channel_slice_copy(src, src_ld, dst, dst_ld, npix, nch, gate=None, gate_ld=0,
                       accumulate=False, stream=None):
    """Per pixel, nch channels from src (pixel stride src_ld) to dst (pixel
    stride dst_ld); src, dst, gate: tensors or device addresses (a channel
    offset is an address offset)."""
    def a(x):
        return None if x is None else (x if isinstance(x, int) else x.data_ptr())
    _check("channel_slice_copy", lib().channel_slice_copy(
        a(src), src_ld, a(gate), gate_ld, a(dst), dst_ld, npix, nch, int(accumulate),
        _s(stream)))


# ---- classification head ----------------------------------------------------
# A small call's time is the host's: tensors that are just what is asked for pass one
# look at type, shape and strides.
_codes = {}      # torch element type -> code, filled on first use (torch may be absent)
_types = {}      # and back
_I32 = 100       # not a code of the library's


def _known():
    import torch
    _codes.update({torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32,
                   torch.int32: _I32})
    _types.update({c: t for t, c in _codes.items()})


def dtype_of(t):
    """Element type code (F16, BF16, F32) of a tensor."""
    if not _codes:
        _known()
    c = _codes.get(t.dtype)
    if c is None or c == _I32:
        raise ValueError(f"element type {t.dtype} is not supported")
    return c


def _matrix(name, t, rows, cols, ld, dtype):
    """Address of a rows x cols matrix in t: the tensor has those sizes in some
    shape (its last axis unit-strided, the others one stride) and row stride ld."""
    if t is None:
        return None
    if not _types:
        _known()
    shape, stride, ld = t.shape, t.stride(), ld or cols
    if t.dtype is not _types.get(dtype):
        raise ValueError(f"{name}: element type {t.dtype} where the descriptor says another")
    if shape == (rows, cols) and stride == (ld, 1):
        return t.data_ptr()
    if t.numel() != rows * cols or (rows and (not shape or shape[-1] != cols)):
        raise ValueError(f"{name}: shape {tuple(shape)} where {rows} x {cols} is needed")
    want = 1
    for i in range(len(shape) - 1, -1, -1):
        if rows and shape[i] > 1 and stride[i] != want:
            raise ValueError(f"{name}: strides {stride} where rows {ld} elements apart "
                             "are needed")
        want = ld if i == len(shape) - 1 else want * shape[i]
    return t.data_ptr()


def _vector(name, t, n, dtype):
    if t is None:
        return None
    if not _types:
        _known()
    if t.dtype is not _types[dtype] or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous "
                         f"{'int32' if dtype == _I32 else 'float32'} tensor of {n} elements")
    return t.data_ptr()


def _counter(name, t):
    if t is None:
        return None
    if not _types:
        _known()
    if t.dtype is not _types[_I32] or t.numel() < 1 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor")
    return t.data_ptr()


def _dropout(fn, name, desc, x, y, z, z_name, step_count, stream):
    rows, cols, dtype = desc.rows, desc.cols, desc.dtype
    st = fn(ctypes.byref(desc), _matrix("x", x, rows, cols, desc.x_ld, dtype),
            None if z is None else _matrix(z_name, z, rows, cols, desc.z_ld, dtype),
            _matrix("y", y, rows, cols, desc.y_ld, dtype),
            None if step_count is None else _counter("step_count", step_count), _s(stream))
    if st:
        raise FgError(name, st)


def dropout_fwd(desc, x, y, residual=None, step_count=None, stream=None):
    """y = residual + dropout(x) (see include/fcngrad.h); tensors of desc's element
    type and strides, e.g. channel slices of wider buffers. step_count: device int32
    added to desc.step by the kernel."""
    _dropout(lib().dropout_fwd, "dropout_fwd", desc, x, y, residual, "residual", step_count,
             stream)


def dropout_bwd(desc, dy, dx, gate=None, step_count=None, stream=None):
    """Gradient of dropout_fwd's x from dy into dx, zero where gate <= 0."""
    _dropout(lib().dropout_bwd, "dropout_bwd", desc, dy, dx, gate, "gate", step_count, stream)


def linear_xent_workspace_bytes(desc, grad):
    return lib().fg_linear_xent_workspace_bytes(ctypes.byref(desc), int(grad))


def _xent_args(desc, h, w, target, loss, lse, totals, weight):
    n, hidden, dtype = desc.rows, desc.hidden, desc.dtype
    return (ctypes.byref(desc), _matrix("h", h, n, hidden, desc.h_ld, dtype),
            _matrix("w", w, desc.vocab, hidden, desc.w_ld, dtype),
            _vector("target", target, n, _I32),
            None if weight is None else _vector("weight", weight, n, F32),
            _vector("loss", loss, n, F32), None if lse is None else _vector("lse", lse, n, F32),
            None if totals is None else _vector("totals", totals, 2, F32))


def linear_xent_fwd(desc, h, w, target, loss, lse=None, totals=None, weight=None, ws=None,
                    stream=None):
    """Softmax cross entropy of the logits h w^T (see include/fcngrad.h): fp32 losses per
    row, their log-sum-exp, and the sums of losses and weights. ws: uint8 tensor of
    linear_xent_workspace_bytes(desc, False)."""
    wp, wb = _ws(ws)
    _check("linear_xent_fwd", lib().linear_xent_fwd(
        *_xent_args(desc, h, w, target, loss, lse, totals, weight), wp, wb, _s(stream)))


def linear_xent_grad(desc, h, w, target, loss, dh, dw, lse=None, totals=None, weight=None,
                     found_nonfinite=None, ws=None, stream=None):
    """linear_xent_fwd with the gradients of desc.scale times the losses' sum (or weighted
    mean, desc.mean) into dh and dw (either may be None). found_nonfinite: device int32
    raised if dw holds an infinity or NaN. ws: linear_xent_workspace_bytes(desc, True)."""
    wp, wb = _ws(ws)
    _check("linear_xent_grad", lib().linear_xent_grad(
        *_xent_args(desc, h, w, target, loss, lse, totals, weight),
        _matrix("dh", dh, desc.rows, desc.hidden, desc.dh_ld, desc.dtype),
        _matrix("dw", dw, desc.vocab, desc.hidden, desc.dw_ld, desc.dtype),
        _counter("found_nonfinite", found_nonfinite), wp, wb, _s(stream)))


# ---- residual blocks ----------------------------------------------------------
# Tensors have to be on the device whose current stream takes the call.
_device = None   # () -> index of the current device


def _current():
    """Index of the current device; no tensor's where there is no GPU."""
    if _device is None:
        return _find_device()
    return _device()


def _find_device():
    global _device
    import torch
    if not _types:
        _known()
    if not (torch.cuda.is_initialized() or torch.cuda.is_available()):
        return -2
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _device()


def _here(name, t, cur):
    if t.get_device() != cur:
        raise ValueError(f"{name} is on {t.device}, not on the current GPU")
    return t.data_ptr()


def _rows_of(name, t, rows, cols, ld, dtype, cur):
    """Address of a rows x cols matrix; None stays."""
    if t is None:
        return None
    if (t.get_device() == cur and t.dtype is _types.get(dtype) and t.shape == (rows, cols)
            and t.stride() == (ld or cols, 1)):
        return t.data_ptr()
    p = _matrix(name, t, rows, cols, ld, dtype)
    _here(name, t, cur)
    return p


def _bytes(name, t, n, cur):
    if t.element_size() != 1 or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous uint8 tensor of {n} bytes")
    _here(name, t, cur)
    return t.data_ptr()


def _per_channel(name, t, n, dtype, cur):
    if t is None:
        return None
    if (t.get_device() == cur and t.dtype is _types.get(dtype) and t.numel() == n
            and t.is_contiguous()):
        return t.data_ptr()
    if t.dtype is not _types.get(dtype) or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {_types.get(dtype)} tensor of {n} elements")
    return _here(name, t, cur)


def _flag(name, t, cur):
    if t is None:
        return None
    p = _counter(name, t)
    _here(name, t, cur)
    return p


def _scratch(ws, cur):
    return (None, 0) if ws is None else (_bytes("ws", ws, 0, cur), ws.numel())


def act8_bytes(rows, cols):
    """Bytes of an 8-bit checkpoint of rows x cols values."""
    return lib().fg_act8_bytes(rows, cols)


def _checkpoint(name, t, rows, cols, cur):
    return None if t is None else _bytes(name, t, lib().fg_act8_bytes(rows, cols), cur)


def act8_pack(desc, x, packed, stream=None):
    """8-bit checkpoint of x (see include/fcngrad.h). packed: uint8 tensor of
    act8_bytes(desc.rows, desc.cols)."""
    n, c, cur = desc.rows, desc.cols, _current()
    st = lib().act8_pack(
        ctypes.byref(desc), _rows_of("x", x, n, c, desc.x_ld, desc.dtype, cur),
        _checkpoint("packed", packed, n, c, cur), _s(stream))
    if st:
        raise FgError("act8_pack", st)


def act8_unpack(desc, packed, x, stream=None):
    """The values of an 8-bit checkpoint, into x."""
    n, c, cur = desc.rows, desc.cols, _current()
    st = lib().act8_unpack(
        ctypes.byref(desc), _checkpoint("packed", packed, n, c, cur),
        _rows_of("x", x, n, c, desc.x_ld, desc.dtype, cur), _s(stream))
    if st:
        raise FgError("act8_unpack", st)


def layer_norm_workspace_bytes(desc):
    return lib().fg_layer_norm_workspace_bytes(ctypes.byref(desc))


def layer_norm_fwd(desc, x, y, weight=None, bias=None, stats=None, packed=None, stream=None):
    """Layer norm of each row (see include/fcngrad.h). stats: fp32 rows x 2, mean and rstd;
    packed: the 8-bit checkpoint of x; both for layer_norm_bwd."""
    n, c, dt, cur = desc.rows, desc.cols, desc.dtype, _current()
    st = lib().layer_norm_fwd(
        ctypes.byref(desc), _rows_of("x", x, n, c, desc.x_ld, dt, cur),
        _per_channel("weight", weight, c, dt, cur), _per_channel("bias", bias, c, dt, cur),
        _rows_of("y", y, n, c, desc.y_ld, dt, cur), _per_channel("stats", stats, 2 * n, F32, cur),
        _checkpoint("packed", packed, n, c, cur), _s(stream))
    if st:
        raise FgError("layer_norm_fwd", st)


def layer_norm_bwd(desc, dy, stats, x=None, packed=None, weight=None, add=None, dx=None,
                   dweight=None, dbias=None, found_nonfinite=None, ws=None, stream=None):
    """Gradients of layer_norm_fwd from x or its checkpoint `packed`; add: another gradient of
    x, added to dx. ws: uint8 tensor of layer_norm_workspace_bytes(desc)."""
    n, c, dt, cur = desc.rows, desc.cols, desc.dtype, _current()
    wp, wb = _scratch(ws, cur)
    st = lib().layer_norm_bwd(
        ctypes.byref(desc), _rows_of("dy", dy, n, c, desc.y_ld, dt, cur),
        _rows_of("x", x, n, c, desc.x_ld, dt, cur), _checkpoint("packed", packed, n, c, cur),
        _per_channel("stats", stats, 2 * n, F32, cur),
        _per_channel("weight", weight, c, dt, cur),
        _rows_of("add", add, n, c, desc.add_ld, dt, cur),
        _rows_of("dx", dx, n, c, desc.dx_ld, dt, cur),
        _per_channel("dweight", dweight, c, dt, cur), _per_channel("dbias", dbias, c, dt, cur),
        _flag("found_nonfinite", found_nonfinite, cur), wp, wb, _s(stream))
    if st:
        raise FgError("layer_norm_bwd", st)


def linear_workspace_bytes(desc, grad):
    return lib().fg_linear_workspace_bytes(ctypes.byref(desc), int(grad))


def linear_fwd(desc, x, w, y, bias=None, residual=None, z=None, packed_z=None, ws=None,
               stream=None):
    """y = residual + act(x w^T + bias) (see include/fcngrad.h). z, packed_z: what an
    activation's backward pass needs of z = x w^T + bias, in desc's type or in 8 bits. ws:
    uint8 tensor of linear_workspace_bytes(desc, False); without packed_z and of up to 64 rows
    (32 where fan_out > 8192) none where fan_in >= 8."""
    n, k, m, dt, cur = desc.rows, desc.fan_in, desc.fan_out, desc.dtype, _current()
    wp, wb = _scratch(ws, cur)
    st = lib().linear_fwd(
        ctypes.byref(desc), _rows_of("x", x, n, k, desc.x_ld, dt, cur),
        _rows_of("w", w, m, k, desc.w_ld, dt, cur), _per_channel("bias", bias, m, dt, cur),
        _rows_of("residual", residual, n, m, desc.r_ld, dt, cur),
        _rows_of("y", y, n, m, desc.y_ld, dt, cur), _rows_of("z", z, n, m, desc.z_ld, dt, cur),
        _checkpoint("packed_z", packed_z, n, m, cur), wp, wb, _s(stream))
    if st:
        raise FgError("linear_fwd", st)


def linear_bwd(desc, dy, x=None, packed_x=None, w=None, z=None, packed_z=None, dx=None, dw=None,
               dbias=None, found_nonfinite=None, ws=None, stream=None):
    """Gradients of linear_fwd from dy: dx (reads w), dw (reads x or its checkpoint packed_x),
    dbias; z or its checkpoint packed_z with an activation (ReLU has no slope where a code is 0:
    z, or y of linear_fwd without residual, keeps the smallest positive ones). ws: uint8 tensor
    of linear_workspace_bytes(desc, True)."""
    n, k, m, dt, cur = desc.rows, desc.fan_in, desc.fan_out, desc.dtype, _current()
    wp, wb = _scratch(ws, cur)
    st = lib().linear_bwd(
        ctypes.byref(desc), _rows_of("dy", dy, n, m, desc.y_ld, dt, cur),
        _rows_of("x", x, n, k, desc.x_ld, dt, cur),
        _checkpoint("packed_x", packed_x, n, k, cur),
        _rows_of("w", w, m, k, desc.w_ld, dt, cur), _rows_of("z", z, n, m, desc.z_ld, dt, cur),
        _checkpoint("packed_z", packed_z, n, m, cur),
        _rows_of("dx", dx, n, k, desc.dx_ld, dt, cur),
        _rows_of("dw", dw, m, k, desc.dw_ld, dt, cur), _per_channel("dbias", dbias, m, dt, cur),
        _flag("found_nonfinite", found_nonfinite, cur), wp, wb, _s(stream))
    if st:
        raise FgError("linear_bwd", st)


def grad_flags_clear(flags, stream=None):
    """Zero a device int32 tensor of non-finite flags with a library kernel."""
    _check("grad_flags_clear", lib().grad_flags_clear(_p(flags), flags.numel(),
                                                      _s(stream)))


def profile_next_launch(start, stop):
    """Arm two torch.cuda.Events (timing enabled) around the main kernel of
    the next convolution call on this thread; None, None disarms."""
    for e in (start, stop):  # torch creates an event at its first record
        if e is not None and not e.cuda_event:
            e.record()
    a = None if start is None else start.cuda_event
    b = None if stop is None else stop.cuda_event
    _check("fg_profile_next_launch", lib().fg_profile_next_launch(a, b))


def mfma_loop(out, blocks, iters, operands=0, stream=None):
    """Register-only MFMA chains (fg_mfma_loop): out is a float32 device
    tensor of at least blocks * 256 elements; blocks * iters * 2^20 flops."""
    if (not out.is_floating_point() or out.element_size() != 4
            or out.numel() < blocks * 256):
        raise ValueError("fg_mfma_loop needs blocks * 256 float32 outputs")
    _check("fg_mfma_loop", lib().fg_mfma_loop(_p(out), blocks, iters, operands, _s(stream)))


def loss_scale_update(state, found_nonfinite):
    """Advance a LossScaleState by one step's outcome; True if it applies."""
    applied = ctypes.c_int32()
    _check("fg_loss_scale_update", lib().fg_loss_scale_update(
        ctypes.byref(state), int(bool(found_nonfinite)), ctypes.byref(applied)))
    return bool(applied.value)


def lr_at(params, k):
    """Learning rate of applied step k under an LRScheduleParams."""
    out = ctypes.c_double()
    _check("fg_lr_at", lib().fg_lr_at(ctypes.byref(params), int(k), ctypes.byref(out)))
    return out.value


def relu_backward(dy, act, out, stream=None):
    _check("relu_backward", lib().relu_backward(
        _p(dy), _p(act), dy.numel(), _p(out), _s(stream)))


def grad_group_plan(numels, cap_bytes, align_bytes=256, elem_bytes=2):
    """Host planner in the library: returns (group_of, offset_of, group_numel)."""
    n = len(numels)
    u64a = (ctypes.c_uint64 * n)(*numels)
    gof = (ctypes.c_int32 * n)()
    oof = (ctypes.c_uint64 * n)()
    gnum = (ctypes.c_uint64 * n)()
    ng = ctypes.c_int32()
    _check("grad_group_plan", lib().grad_group_plan(
        u64a, n, cap_bytes, align_bytes, elem_bytes, gof, oof,
        ctypes.byref(ng), gnum))
    return list(gof), list(oof), list(gnum[:ng.value])
