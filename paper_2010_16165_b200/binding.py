"""Thin ctypes binding over the C-ABI library (include/fupruner.h).

Argument marshalling only: every step of fusing, pruning and running the network happens
inside the library's CUDA kernels.  PyTorch is used for device memory and streams.
The library is required - there is no fallback; a missing build raises ImportError here.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libfupruner.so")

FP_OK = 0
FP_ERR_ARG, FP_ERR_DESC, FP_ERR_SHAPE, FP_ERR_NONFINITE, FP_ERR_CUDA = -1, -2, -3, -4, -5
FP_ERR_NOMEM, FP_ERR_UNSUPPORTED, FP_ERR_TIMEOUT, FP_ERR_EMPTY_LAYER, FP_ERR_BOUNDS = -6, -7, -8, -9, -10
FP_DTYPE_F32, FP_DTYPE_BF16, FP_DTYPE_F16 = 0, 1, 2
FP_COMPUTE_BF16_TC, FP_COMPUTE_FP32, FP_COMPUTE_BF16_SIMT = 0, 1, 2
FP_NORM_L1, FP_NORM_L2 = 0, 1
FP_ACT_NONE, FP_ACT_RELU, FP_ACT_GELU, FP_ACT_GELU_TANH, FP_ACT_SILU = range(5)
FP_ADAMW_BLOCK = 256
(FP_Q_N_CONVS, FP_Q_CONV_K_FUSED, FP_Q_CONV_K_KEPT, FP_Q_CONV_C_KEPT, FP_Q_MASK, FP_Q_RANK, FP_Q_N_CLASSES,
 FP_Q_FLOPS, FP_Q_BYTES, FP_Q_N_OPS, FP_Q_OP_INFO, FP_Q_OP_OUTPUT, FP_Q_DEVICE_STATUS, FP_Q_N_LAUNCHES,
 FP_Q_OP_TIMES, FP_Q_CONV_BANK_ELEMS, FP_Q_ALL_MASKS, FP_Q_OP_PLAN) = range(18)

EXPORTS = ["fp_fuse", "fp_prune", "fp_forward", "fp_forward_host", "fp_forward_host_async", "fp_score", "fp_query", "fp_destroy",
           "fp_last_error", "fp_rank_filters_static", "fp_soft_prune_epoch", "fp_soft_prune_finish",
           "fp_debug_expire_wait", "fp_fuse_with_allocator", "fp_linear_forward", "fp_linear_backward", "fp_linear_workspace",
           "fp_linear_backward_workspace", "fp_linear_status", "fp_cross_entropy", "fp_adamw_step"]
FP_STATIC_RANK_MAX_FILTERS = 4096
OP_PLAN_FIELDS = ("tps", "cg", "groups", "groups2", "a_stages", "b_stages", "stays", "epi_warps", "alternate", "n_tile")
CONV_KERNELS = ("", "conv_tc_kernel", "conv_split_kernel", "stem_pool_kernel", "chain_tc_kernel", "resident_net_kernel", "conv_simt_kernel",
                "conv_pair_kernel", "chain_quad_kernel")


class fp_node(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("op", "in0", "in1", "K", "C", "R", "S", "stride", "pad", "pad_lo", "block_id", "aggressive",
                 "reserved")] + [("pad_", ctypes.c_int32)] + \
               [("w_off", ctypes.c_int64), ("b_off", ctypes.c_int64), ("bn_off", ctypes.c_int64)]


class fp_model_desc(ctypes.Structure):
    _fields_ = [("n_nodes", ctypes.c_int32), ("nodes", ctypes.POINTER(fp_node)),
                ("in_C", ctypes.c_int32), ("in_H", ctypes.c_int32), ("in_W", ctypes.c_int32),
                ("in_dtype", ctypes.c_int32), ("compute", ctypes.c_int32), ("bn_eps", ctypes.c_float),
                ("use_graph", ctypes.c_int32), ("keep_outputs", ctypes.c_int32), ("scatter", ctypes.c_int32)]


class fp_op_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("kind", "conv_index", "K", "C", "R", "S", "stride", "pad", "K_pad", "C_pad", "H", "W", "P", "Q",
                 "res_mode", "relu")] + \
               [("flops_per_image", ctypes.c_double), ("bytes_per_image", ctypes.c_double),
                ("bytes_fixed", ctypes.c_double), ("chain", ctypes.c_int32), ("kernel", ctypes.c_int32)]


def _struct(name, **fields):
    """A ctypes structure from space-separated field names by type, in the order given."""
    return type(name, (ctypes.Structure,), {"_fields_": [(f, t) for key, (t, names) in fields.items() for f in names.split()]})


fp_linear_args = _struct("fp_linear_args", a=(ctypes.c_int64, "M N K"), b=(ctypes.c_int32, "dtype y_dtype bias_dtype act res_first reserved"),
                         c=(ctypes.c_void_p, "d_x d_w d_bias d_res d_y d_pre"), d=(ctypes.c_int64, "ld_x ld_w ld_res ld_y ld_pre"))
fp_linear_grad_args = _struct("fp_linear_grad_args", a=(ctypes.c_int64, "M N K"), b=(ctypes.c_int32, "dtype dw_dtype act accumulate"),
                              c=(ctypes.c_void_p, "d_dy d_pre d_x d_w d_dx d_dw d_db d_dz"),
                              d=(ctypes.c_int64, "ld_dy ld_pre ld_x ld_w ld_dx ld_dw ld_dz"))
fp_cross_entropy_args = _struct("fp_cross_entropy_args", a=(ctypes.c_int64, "rows classes"), b=(ctypes.c_int32, "dtype label_bytes"),
                                c=(ctypes.c_int64, "ignore_index"), d=(ctypes.c_float, "label_smoothing grad_scale"),
                                e=(ctypes.c_void_p, "d_logits d_labels d_row_grad d_loss d_dlogits"), f=(ctypes.c_int64, "ld_logits ld_dlogits"))
fp_adamw_tensor = _struct("fp_adamw_tensor", a=(ctypes.c_int64, "n per_row"), b=(ctypes.c_int32, "p_dtype g_dtype state_bits reserved"),
                          c=(ctypes.c_void_p, "d_p d_g d_m d_v d_m_scale d_v_scale d_mask"))
fp_adamw_hyper = _struct("fp_adamw_hyper", a=(ctypes.c_double, "lr beta1 beta2 eps weight_decay grad_scale"), b=(ctypes.c_int64, "step"),
                         c=(ctypes.c_void_p, "d_lr d_grad_scale d_step"))


# The same layouts for struct: a call's arguments are packed in a quarter of the time that a ctypes structure takes.
_LINEAR, _LINEAR_GRAD, _CROSS_ENTROPY, _ADAMW_TENSOR, _ADAMW_HYPER = (struct.Struct(f) for f in ("3q6i6P5q", "3q4i8P7q", "2q2iq2f5P2q", "2q4i7P", "6dq3P"))


ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
DEALLOC_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class TorchAllocator:
    """PyTorch's caching allocator as the library's device allocator (argument marshalling only: the two callbacks hand
    sizes and pointers through).  Keep the object alive as long as the handle."""

    def __init__(self):
        import torch
        self.n_alloc = self.n_free = 0
        self.live = {}

        def _alloc(nbytes, _user):
            try:
                ptr = torch.cuda.caching_allocator_alloc(int(nbytes))
            except Exception:
                return None
            self.n_alloc += 1
            self.live[ptr] = int(nbytes)
            return ptr

        def _free(ptr, _user):
            self.n_free += 1
            self.live.pop(ptr, None)
            torch.cuda.caching_allocator_delete(ptr)

        self.alloc, self.dealloc = ALLOC_FN(_alloc), DEALLOC_FN(_free)


class FpError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"fupruner status {status}: {message}")
        self.status = status


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2010_16165_b200.build` "
                              "(there is no fallback path)")
        L = ctypes.CDLL(_LIB_PATH)
        L.fp_last_error.restype = ctypes.c_char_p
        L.fp_fuse.argtypes = [ctypes.POINTER(fp_model_desc), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                              ctypes.c_size_t, ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p)]
        L.fp_fuse_with_allocator.argtypes = [ctypes.POINTER(fp_model_desc), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                             ctypes.c_size_t, ctypes.c_int32, ALLOC_FN, DEALLOC_FN, ctypes.c_void_p,
                                             ctypes.POINTER(ctypes.c_void_p)]
        L.fp_prune.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        L.fp_forward.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        L.fp_forward_host.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        L.fp_forward_host_async.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        L.fp_score.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]
        L.fp_query.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t]
        L.fp_destroy.argtypes = [ctypes.c_void_p]
        L.fp_soft_prune_epoch.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        L.fp_soft_prune_finish.argtypes = [ctypes.c_void_p]
        L.fp_debug_expire_wait.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        L.fp_rank_filters_static.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        for f in ("fp_linear_forward", "fp_linear_backward"):
            getattr(L, f).argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        for f in ("fp_linear_workspace", "fp_linear_backward_workspace"):
            getattr(L, f).argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)]
        L.fp_linear_status.argtypes = [ctypes.POINTER(ctypes.c_int32)]
        L.fp_cross_entropy.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        L.fp_adamw_step.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        _lib = L
    return _lib


def _check(status):
    if status != FP_OK:
        raise FpError(status, lib().fp_last_error().decode())


def make_nodes(node_dicts):
    arr = (fp_node * len(node_dicts))()
    for a, n in zip(arr, node_dicts):
        for k in ("op", "in0", "in1", "K", "C", "R", "S", "stride", "pad", "pad_lo", "block_id", "aggressive",
                  "w_off", "b_off", "bn_off"):
            setattr(a, k, int(n[k]))
    return arr


def fp_fuse(net, d_weights, d_bn, max_batch, compute=FP_COMPUTE_BF16_TC, in_dtype=FP_DTYPE_F32, use_graph=0,
            keep_outputs=0, scatter=0, allocator=None):
    """net: workloads.Net; d_weights/d_bn: CUDA float32 torch tensors; allocator: None (the library uses cudaMalloc) or an
    object with ctypes callbacks `alloc` / `dealloc` (TorchAllocator).  Returns an opaque handle."""
    nodes = make_nodes(net.nodes)
    desc = fp_model_desc(len(net.nodes), nodes, net.in_C, net.in_H, net.in_W, in_dtype, compute,
                         float(net.bn_eps), use_graph, keep_outputs, scatter)
    h = ctypes.c_void_p()
    if allocator is None:
        _check(lib().fp_fuse(ctypes.byref(desc), d_weights.data_ptr(), d_weights.numel(), d_bn.data_ptr(),
                             d_bn.numel(), max_batch, ctypes.byref(h)))
    else:
        _check(lib().fp_fuse_with_allocator(ctypes.byref(desc), d_weights.data_ptr(), d_weights.numel(), d_bn.data_ptr(),
                                            d_bn.numel(), max_batch, allocator.alloc, allocator.dealloc, None, ctypes.byref(h)))
    return h


def fp_prune(h, ratios=None, masks=None, norm=FP_NORM_L1):
    """ratios: sequence of one float per convolution, or None.  masks: dict/list conv -> uint8 array, or None."""
    r = None
    if ratios is not None:
        r = np.ascontiguousarray(ratios, dtype=np.float64)
    mptr = None
    keep = []
    if masks is not None:
        n = fp_query_int(h, FP_Q_N_CONVS)
        mptr = (ctypes.c_void_p * n)()
        for ci in range(n):
            m = masks.get(ci) if isinstance(masks, dict) else masks[ci]
            if m is None:
                mptr[ci] = None
            else:
                m = np.ascontiguousarray(m, dtype=np.uint8)
                keep.append(m)
                mptr[ci] = m.ctypes.data
    _check(lib().fp_prune(h, norm, r.ctypes.data if r is not None else None, mptr))


def fp_forward(h, d_input, batch, d_logits, stream=None):
    """d_input / d_logits: CUDA torch tensors; stream: torch.cuda.Stream or None (default stream)."""
    _check(lib().fp_forward(h, d_input.data_ptr(), batch, d_logits.data_ptr(),
                            stream.cuda_stream if stream is not None else None))


def fp_forward_host(h, h_input, batch, h_logits, stream=None):
    """h_input / h_logits: host buffers (numpy arrays or pinned CPU torch tensors)."""
    pin = h_input.ctypes.data if isinstance(h_input, np.ndarray) else h_input.data_ptr()
    pout = h_logits.ctypes.data if isinstance(h_logits, np.ndarray) else h_logits.data_ptr()
    _check(lib().fp_forward_host(h, pin, batch, pout, stream.cuda_stream if stream is not None else None))


def fp_forward_host_async(h, h_input, batch, h_logits, stream=None):
    """fp_forward_host without the wait: h_logits is valid once `stream` has been synchronised."""
    pin = h_input.ctypes.data if isinstance(h_input, np.ndarray) else h_input.data_ptr()
    pout = h_logits.ctypes.data if isinstance(h_logits, np.ndarray) else h_logits.data_ptr()
    _check(lib().fp_forward_host_async(h, pin, batch, pout, stream.cuda_stream if stream is not None else None))


def fp_score(h, conv_index, norm=FP_NORM_L1):
    K = fp_query_int(h, FP_Q_CONV_K_FUSED, conv_index)
    out = np.empty(K, dtype=np.float64)
    _check(lib().fp_score(h, conv_index, norm, out.ctypes.data))
    return out


def fp_query_int(h, what, index=0):
    v = ctypes.c_int32()
    _check(lib().fp_query(h, what, index, ctypes.byref(v), 4))
    return v.value


def fp_query_array(h, what, index, dtype, count):
    out = np.empty(count, dtype=dtype)
    _check(lib().fp_query(h, what, index, out.ctypes.data, out.nbytes))
    return out


def fp_query_plan(h, index):
    """The form that operator `index` has in conv_tc_kernel: OP_PLAN_FIELDS -> int (zeros where another kernel computes it)."""
    return dict(zip(OP_PLAN_FIELDS, fp_query_array(h, FP_Q_OP_PLAN, index, np.int32, len(OP_PLAN_FIELDS)).tolist()))


def fp_query_op(h, index):
    o = fp_op_info()
    _check(lib().fp_query(h, FP_Q_OP_INFO, index, ctypes.byref(o), ctypes.sizeof(o)))
    return o


def fp_rank_filters_static(d_filters, K, per_filter, norm, q, d_rank, d_mask, stream=None):
    """Allocation-free selection for one bank: d_filters fp32 CUDA tensor (K*per_filter), d_rank int32[K] and
    d_mask uint8[K] CUDA tensors provided by the caller.  Asynchronous on `stream`."""
    _check(lib().fp_rank_filters_static(d_filters.data_ptr(), K, per_filter, norm, q, d_rank.data_ptr(),
                                        d_mask.data_ptr(), stream.cuda_stream if stream is not None else None))


def fp_soft_prune_epoch(h, ratios=None, d_updates=None, norm=FP_NORM_L2):
    """One pass of Algorithm 1's loop body.  d_updates: CUDA float32 tensor (concatenated addends of all fused
    banks, see conv_bank_elems) or None."""
    r = np.ascontiguousarray(ratios, dtype=np.float64) if ratios is not None else None
    _check(lib().fp_soft_prune_epoch(h, norm, r.ctypes.data if r is not None else None,
                                     d_updates.data_ptr() if d_updates is not None else None))


def fp_soft_prune_finish(h):
    _check(lib().fp_soft_prune_finish(h))


def fp_debug_expire_wait(h, stream=None):
    """Diagnostic: lets one bounded device-side wait run out (see the header); the next FP_Q_DEVICE_STATUS reports it."""
    _check(lib().fp_debug_expire_wait(h, stream.cuda_stream if stream is not None else None))


def conv_bank_elems(h):
    """Weights in the fused fp32 bank of every convolution of the description (0 where absorbed)."""
    out = []
    for ci in range(fp_query_int(h, FP_Q_N_CONVS)):
        v = ctypes.c_int64()
        _check(lib().fp_query(h, FP_Q_CONV_BANK_ELEMS, ci, ctypes.byref(v), 8))
        out.append(int(v.value))
    return out


def fp_destroy(h):
    _check(lib().fp_destroy(h))


def masks_and_ranks(h):
    n_convs, n = fp_query_int(h, FP_Q_N_CONVS), fp_query_int(h, FP_Q_ALL_MASKS, 0)
    raw = fp_query_array(h, FP_Q_ALL_MASKS, 1, np.uint8, 4 * n_convs + 5 * n)
    ints = raw[:4 * (n_convs + n)].view(np.int32)
    masks = raw[4 * (n_convs + n):]
    out, at = {}, 0
    for ci, K in enumerate(ints[:n_convs].tolist()):
        end = at + K
        out[ci] = (masks[at:end], ints[n_convs + at:n_convs + end]) if K else (None, None)
        at = end
    return out


def op_infos(h):
    return [fp_query_op(h, i) for i in range(fp_query_int(h, FP_Q_N_OPS))]


# ---- the training step around pruning (see the header's section of that name) ----------------------------------------

_dtype_codes = None


def _dtypes():
    global _dtype_codes
    if _dtype_codes is None:
        import torch
        _dtype_codes = {torch.float32: FP_DTYPE_F32, torch.bfloat16: FP_DTYPE_BF16, torch.float16: FP_DTYPE_F16}
    return _dtype_codes


def _dtype(t, name):
    code = _dtypes().get(t.dtype)
    if code is None:
        raise ValueError(f"{name} has dtype {t.dtype}")
    return code


def _matrix(t, shape, name, dtype=None):
    """(address, row stride) of a tensor of that shape whose rows are contiguous; (0, 0) of None."""
    if t is None:
        return 0, 0
    if t.shape != shape or not t.is_cuda or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"{name} is {tuple(t.shape)} {t.dtype} on {t.device}: a CUDA tensor of {shape}, {dtype} is wanted")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError(f"{name}: neighbours of a row must be neighbours in memory (strides {t.stride()})")
    return t.data_ptr(), ld


def _vector(t, n, name, dtype=None):
    """Address of a contiguous vector of n elements; 0 of None."""
    if t is None:
        return 0
    if t.shape != (n,) or not t.is_cuda or (dtype is not None and t.dtype is not dtype) or (n > 1 and t.stride() != (1,)):
        raise ValueError(f"{name} is {tuple(t.shape)} {t.dtype} on {t.device}: a contiguous CUDA vector of {n}, {dtype} is wanted")
    return t.data_ptr()


def _scratch(work):
    return (None, 0) if work is None else (work.data_ptr(), work.numel() * work.element_size())


def _linear_values(x, w, y, bias, res, pre, act, res_first):
    (M, K), N, dt = x.shape, w.shape[0], x.dtype
    out = (M, N)
    px, lx = _matrix(x, (M, K), "x")
    pw, lw = _matrix(w, (N, K), "w", dt)
    py, ly = _matrix(y, out, "y")
    pr, lr = _matrix(res, out, "res", dt) if res is not None else (0, 0)
    pp, lp = _matrix(pre, out, "pre", dt) if pre is not None else (0, 0)
    return (M, N, K, _dtype(x, "x"), _dtype(y, "y"), 0 if bias is None else _dtype(bias, "bias"), act, 1 if res_first else 0, 0,
            px, pw, _vector(bias, N, "bias"), pr, py, pp, lx, lw, lr, ly, lp)


def _linear_args(*tensors):
    return fp_linear_args(*_linear_values(*tensors))


def fp_linear_forward(x, w, y, bias=None, res=None, pre=None, act=FP_ACT_NONE, res_first=False, work=None, stream=None):
    """y = act(x w' + bias) + res, or act(x w' + bias + res) with res_first.  x (M, K), w (N, K), res and pre (M, N): bf16 or
    f16 CUDA tensors with contiguous rows; y and bias: the same type or float32.  pre receives what the activation is taken of.
    work: uint8 tensor of at least fp_linear_workspace bytes, or None where that is 0."""
    a = _LINEAR.pack(*_linear_values(x, w, y, bias, res, pre, act, res_first))
    p, n = _scratch(work)
    _check(lib().fp_linear_forward(a, p, n, stream.cuda_stream if stream is not None else None))


def fp_linear_workspace(x, w, y, bias=None, res=None, pre=None, act=FP_ACT_NONE, res_first=False):
    """Bytes of scratch that fp_linear_forward needs for these tensors."""
    n = ctypes.c_size_t()
    _check(lib().fp_linear_workspace(_LINEAR.pack(*_linear_values(x, w, y, bias, res, pre, act, res_first)), ctypes.byref(n)))
    return n.value


def _linear_grad_values(dy, x, w, dx, dw, db, dz, pre, act, accumulate):
    M, N = dy.shape
    K, dt, dy_shape = next((t.shape[1] for t in (x, w, dx, dw) if t is not None), 1), dy.dtype, (M, N)
    pdy, ldy = _matrix(dy, dy_shape, "dy")
    px, lx = _matrix(x, (M, K), "x", dt)
    pw, lw = _matrix(w, (N, K), "w", dt)
    pdx, ldx = _matrix(dx, (M, K), "dx", dt)
    pdw, ldw = _matrix(dw, (N, K), "dw")
    pdz, ldz = _matrix(dz, dy_shape, "dz", dt)
    pp, lp = _matrix(pre, dy_shape, "pre", dt)
    out = dw if dw is not None else db
    code = _dtype(out, "dw") if out is not None else _dtype(dy, "dy")
    return (M, N, K, _dtype(dy, "dy"), code, act, 1 if accumulate else 0, pdy, pp, px, pw, pdx, pdw,
            _vector(db, N, "db", None if out is None else out.dtype), pdz, ldy, lp, lx, lw, ldx, ldw, ldz)


def _linear_grad_args(*tensors):
    return fp_linear_grad_args(*_linear_grad_values(*tensors))


def fp_linear_backward(dy, x, w, dx=None, dw=None, db=None, dz=None, pre=None, act=FP_ACT_NONE, accumulate=False, work=None, stream=None):
    """Gradients of fp_linear_forward, each where a tensor is given for it: dz = dy * act'(pre), dx = dz w, dw = dz' x, db = sum of
    dz's rows (added to dw and db with accumulate).  x may be None without dw, w without dx.  dw and db: the inputs' type or
    float32, both the same.  work: at least fp_linear_backward_workspace bytes, or None where that is 0."""
    a = _LINEAR_GRAD.pack(*_linear_grad_values(dy, x, w, dx, dw, db, dz, pre, act, accumulate))
    p, n = _scratch(work)
    _check(lib().fp_linear_backward(a, p, n, stream.cuda_stream if stream is not None else None))


def fp_linear_backward_workspace(dy, x, w, dx=None, dw=None, db=None, dz=None, pre=None, act=FP_ACT_NONE, accumulate=False):
    """Bytes of scratch that fp_linear_backward needs for these tensors."""
    n = ctypes.c_size_t()
    _check(lib().fp_linear_backward_workspace(_LINEAR_GRAD.pack(*_linear_grad_values(dy, x, w, dx, dw, db, dz, pre, act, accumulate)), ctypes.byref(n)))
    return n.value


def fp_linear_status():
    """FP_OK, or FP_ERR_TIMEOUT where a device-side wait of the layers' kernels ran out since the last call (synchronises)."""
    v = ctypes.c_int32()
    _check(lib().fp_linear_status(ctypes.byref(v)))
    return v.value


def fp_cross_entropy(logits, labels, loss=None, dlogits=None, row_grad=None, label_smoothing=0.0, ignore_index=-100, grad_scale=1.0, stream=None):
    """Softmax cross-entropy of every row of logits (rows, classes) with int32 or int64 labels (rows): loss (rows, float32) and dlogits
    = grad_scale * row_grad * d loss / d logits, of the logits' type (it may be the logits themselves); either may be None."""
    rows, classes = logits.shape
    px, lx = _matrix(logits, (rows, classes), "logits")
    pd, ld = _matrix(dlogits, (rows, classes), "dlogits", logits.dtype)
    torch_f32, label_bytes = _f32_and_labels()
    size = label_bytes.get(labels.dtype)
    if size is None:
        raise ValueError(f"labels have dtype {labels.dtype}")
    a = _CROSS_ENTROPY.pack(rows, classes, _dtype(logits, "logits"), size, ignore_index, label_smoothing, grad_scale, px,
                            _vector(labels, rows, "labels"), _vector(row_grad, rows, "row_grad", torch_f32), _vector(loss, rows, "loss", torch_f32), pd, lx, ld)
    _check(lib().fp_cross_entropy(a, stream.cuda_stream if stream is not None else None))


_label_codes = None


def _f32_and_labels():
    global _label_codes
    if _label_codes is None:
        import torch
        _label_codes = torch.float32, {torch.int32: 4, torch.int64: 8}
    return _label_codes


class AdamwTensors:
    """The table of a network's tensors for fp_adamw_step; holds the tensors, whose addresses it has."""

    def __init__(self, array, tensors):
        self.array, self.tensors = array, tensors


def fp_adamw_tensors(tensors):
    """tensors: dicts of CUDA tensors - p (float32, bf16 or f16; updated), g, m, v (float32 like p's shape, or e4m3 codes: float8_e4m3fn
    or uint8 with float32 m_scale and v_scale, one for every FP_ADAMW_BLOCK elements) and optionally mask (uint8, one for every row of p,
    or for every len / mask elements of a vector).  All contiguous; what the step writes may be listed once.  Returns the table that
    fp_adamw_step takes, made once for buffers that stay: a gradient that is allocated anew needs a new table."""
    import torch
    f8 = (torch.uint8, torch.float8_e4m3fn)
    rows, written, read = [], [], []
    for t in tensors:
        p, g, m, v, mask = t["p"], t["g"], t["m"], t["v"], t.get("mask")
        n, bits = p.numel(), 8 if m.dtype in f8 else 32
        blocks = -(-n // FP_ADAMW_BLOCK)
        for k, x in t.items():
            if x is not None and (not x.is_cuda or not x.is_contiguous()):
                raise ValueError(f"{k}: a contiguous CUDA tensor is wanted")
        if g.numel() != n or m.numel() != n or v.numel() != n or m.dtype not in (f8 if bits == 8 else (torch.float32,)) or v.dtype != m.dtype:
            raise ValueError("p, g, m and v must have one size, m and v one type (float32, or e4m3 codes)")
        if bits == 8 and any(t[k].dtype != torch.float32 or t[k].numel() != blocks for k in ("m_scale", "v_scale")):
            raise ValueError(f"m_scale and v_scale must be {blocks} float32")
        per_row = 0
        if mask is not None and n:
            if mask.dtype != torch.uint8 or not mask.numel() or n % mask.numel():
                raise ValueError("mask must be uint8, one entry for every row of p")
            per_row = n // mask.numel()
        out, into = [p.data_ptr(), m.data_ptr(), v.data_ptr()], [g.data_ptr()]
        if bits == 8:
            out += [t["m_scale"].data_ptr(), t["v_scale"].data_ptr()]
        if per_row:
            into.append(mask.data_ptr())
        rows.append(_ADAMW_TENSOR.pack(n, per_row, _dtype(p, "p"), _dtype(g, "g"), bits, 0, out[0], into[0], out[1], out[2], *(out[3:] or (0, 0)),
                                       into[1] if per_row else 0))
        if n:
            written += out
            read += into
    once = set(written)
    if len(once) != len(written) or not once.isdisjoint(read):
        raise ValueError("a tensor that the step writes (p, m, v, m_scale or v_scale) is listed twice, or is another one's gradient or mask")
    array = (fp_adamw_tensor * len(rows)).from_buffer(bytearray(b"".join(rows))) if rows else (fp_adamw_tensor * 0)()
    return AdamwTensors(array, [dict(t) for t in tensors])


def fp_adamw_step(table, lr, step=1, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0, d_lr=None, d_grad_scale=None,
                  d_step=None, stream=None):
    """One AdamW step (number `step`, from 1) over all tensors of a table.  d_lr, d_grad_scale (float32) and d_step (int64): CUDA tensors of
    one element that are read when the kernel runs, in place of the numbers - for a captured step."""
    h = _ADAMW_HYPER.pack(lr, beta1, beta2, eps, weight_decay, grad_scale, step, _scalar(d_lr, "float32", "d_lr"),
                          _scalar(d_grad_scale, "float32", "d_grad_scale"), _scalar(d_step, "int64", "d_step"))
    _check(lib().fp_adamw_step(ctypes.addressof(table.array), len(table.array), h,
                               stream.cuda_stream if stream is not None else None))


def _scalar(t, dtype, name):
    """Address of a CUDA tensor of one element; 0 of None."""
    if t is None:
        return 0
    if str(t.dtype) != "torch." + dtype or t.numel() != 1 or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor of one {dtype} is wanted")
    return t.data_ptr()
