"""What the training-step calls refuse, before any GPU is asked: sizes, types, strides, alignment, missing buffers."""
import ctypes

import pytest

from paper_2010_16165_b200 import binding as B

P = 1 << 20          # an address that is never read: every call below is refused, or only asked for its scratch
X, W, Y, Z = (P * k for k in (2, 3, 4, 5))       # others


def linear(**kw):
    d = dict(M=4, N=8, K=16, dtype=B.FP_DTYPE_BF16, y_dtype=B.FP_DTYPE_BF16, bias_dtype=B.FP_DTYPE_F32, act=0, res_first=0, reserved=0, d_x=X, d_w=W,
             d_bias=P, d_res=None, d_y=Y, d_pre=None, ld_x=16, ld_w=16, ld_res=8, ld_y=8, ld_pre=8)
    d.update(kw)
    return B.fp_linear_args(**d)


def grads(**kw):
    d = dict(M=4, N=8, K=16, dtype=B.FP_DTYPE_BF16, dw_dtype=B.FP_DTYPE_F32, act=0, accumulate=0, d_dy=Y, d_pre=None, d_x=X, d_w=W, d_dx=P, d_dw=6 * P,
             d_db=7 * P, d_dz=None, ld_dy=8, ld_pre=8, ld_x=16, ld_w=16, ld_dx=16, ld_dw=16, ld_dz=8)
    d.update(kw)
    return B.fp_linear_grad_args(**d)


def loss(**kw):
    d = dict(rows=4, classes=8, dtype=B.FP_DTYPE_F32, label_bytes=8, ignore_index=-100, label_smoothing=0.0, grad_scale=1.0, d_logits=P, d_labels=P,
             d_row_grad=None, d_loss=P, d_dlogits=P + 4096, ld_logits=8, ld_dlogits=8)
    d.update(kw)
    return B.fp_cross_entropy_args(**d)


def tensor(**kw):
    d = dict(n=64, per_row=0, p_dtype=0, g_dtype=0, state_bits=32, reserved=0, d_p=P, d_g=P, d_m=P, d_v=P, d_m_scale=None, d_v_scale=None, d_mask=None)
    d.update(kw)
    return B.fp_adamw_tensor(**d)


def hyper(**kw):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, d_lr=None, d_grad_scale=None, d_step=None)
    d.update(kw)
    return B.fp_adamw_hyper(**d)


def message():
    return B.lib().fp_last_error().decode()


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), B.FP_ERR_ARG), (dict(N=0), B.FP_ERR_ARG), (dict(K=0), B.FP_ERR_ARG), (dict(M=(1 << 30) + 1), B.FP_ERR_BOUNDS),
    (dict(K=1 << 31, ld_x=1 << 31, ld_w=1 << 31), B.FP_ERR_BOUNDS), (dict(dtype=B.FP_DTYPE_F32), B.FP_ERR_UNSUPPORTED), (dict(dtype=7), B.FP_ERR_UNSUPPORTED),
    (dict(y_dtype=B.FP_DTYPE_F16), B.FP_ERR_UNSUPPORTED), (dict(bias_dtype=B.FP_DTYPE_F16), B.FP_ERR_UNSUPPORTED), (dict(act=5), B.FP_ERR_ARG),
    (dict(act=-1), B.FP_ERR_ARG), (dict(res_first=2), B.FP_ERR_ARG), (dict(reserved=1), B.FP_ERR_ARG), (dict(d_x=None), B.FP_ERR_ARG),
    (dict(d_w=None), B.FP_ERR_ARG), (dict(d_y=None), B.FP_ERR_ARG), (dict(ld_x=15), B.FP_ERR_ARG), (dict(ld_w=0), B.FP_ERR_ARG), (dict(ld_y=7), B.FP_ERR_ARG),
    (dict(d_res=Z, ld_res=7), B.FP_ERR_ARG), (dict(d_pre=Z, ld_pre=-8), B.FP_ERR_ARG), (dict(d_x=P + 1), B.FP_ERR_ARG),
    (dict(d_y=X), B.FP_ERR_ARG), (dict(d_y=W), B.FP_ERR_ARG), (dict(d_y=P), B.FP_ERR_ARG), (dict(d_pre=Y), B.FP_ERR_ARG), (dict(d_pre=X), B.FP_ERR_ARG),
    (dict(d_pre=Z, d_res=Z), B.FP_ERR_ARG), (dict(d_res=Y, y_dtype=B.FP_DTYPE_F32), B.FP_ERR_ARG), (dict(d_res=Y, ld_res=9), B.FP_ERR_ARG),
    (dict(y_dtype=B.FP_DTYPE_F32, d_y=P + 2), B.FP_ERR_ARG), (dict(d_bias=P + 2), B.FP_ERR_ARG), (dict(ld_x=1 << 39), B.FP_ERR_ARG)])
def test_linear(kw, status):
    a, n = linear(**kw), ctypes.c_size_t(77)
    assert B.lib().fp_linear_forward(ctypes.addressof(a), None, 0, None) == status
    assert "fp_linear_forward" in message()
    assert B.lib().fp_linear_workspace(ctypes.addressof(a), ctypes.byref(n)) == status
    assert n.value == 77


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), B.FP_ERR_ARG), (dict(N=0), B.FP_ERR_ARG), (dict(K=-3), B.FP_ERR_ARG), (dict(N=1 << 31, ld_dy=1 << 31), B.FP_ERR_BOUNDS),
    (dict(dtype=B.FP_DTYPE_F32), B.FP_ERR_UNSUPPORTED), (dict(dw_dtype=B.FP_DTYPE_F16), B.FP_ERR_UNSUPPORTED), (dict(act=9), B.FP_ERR_ARG),
    (dict(accumulate=-1), B.FP_ERR_ARG), (dict(act=B.FP_ACT_GELU), B.FP_ERR_ARG), (dict(d_dy=None), B.FP_ERR_ARG), (dict(d_x=None), B.FP_ERR_ARG),
    (dict(d_w=None), B.FP_ERR_ARG), (dict(d_dx=None, d_dw=None, d_db=None), B.FP_ERR_ARG), (dict(ld_dy=7), B.FP_ERR_ARG), (dict(ld_x=8), B.FP_ERR_ARG),
    (dict(ld_w=8), B.FP_ERR_ARG), (dict(ld_dx=8), B.FP_ERR_ARG), (dict(ld_dw=8), B.FP_ERR_ARG), (dict(d_dz=Y, ld_dz=9), B.FP_ERR_ARG),
    (dict(d_dx=Y), B.FP_ERR_ARG), (dict(d_dx=X), B.FP_ERR_ARG), (dict(d_dx=W), B.FP_ERR_ARG), (dict(d_dw=W), B.FP_ERR_ARG), (dict(d_dz=X), B.FP_ERR_ARG),
    (dict(d_dw=P), B.FP_ERR_ARG), (dict(d_db=6 * P), B.FP_ERR_ARG), (dict(act=1, d_pre=Z, d_dz=Z), B.FP_ERR_ARG),
    (dict(d_dw=Z + 2), B.FP_ERR_ARG), (dict(d_dy=P + 1), B.FP_ERR_ARG), (dict(M=0, d_db=P + 2), B.FP_ERR_ARG)])
def test_linear_gradients(kw, status):
    a, n = grads(**kw), ctypes.c_size_t(77)
    assert B.lib().fp_linear_backward(ctypes.addressof(a), None, 0, None) == status
    assert "fp_linear_backward" in message()
    assert B.lib().fp_linear_backward_workspace(ctypes.addressof(a), ctypes.byref(n)) == status
    assert n.value == 77


def test_scratch_of_linear():
    """Operands that start at 16-byte boundaries need none; each that does not is copied, its rows rounded up to 16 bytes."""
    def need(a, f=B.lib().fp_linear_workspace):
        n = ctypes.c_size_t()
        assert f(ctypes.addressof(a), ctypes.byref(n)) == B.FP_OK
        return n.value
    def up(n):
        return -(-n // 256) * 256
    back = B.lib().fp_linear_backward_workspace
    assert need(linear()) == 0 and need(linear(M=0, d_x=None, d_y=None, d_w=None)) == 0
    assert need(linear(d_x=X + 2)) == up(4 * 16 * 2)
    assert need(linear(M=100, ld_x=17)) == up(100 * 16 * 2)
    assert need(linear(M=1, ld_x=17)) == 0
    assert need(linear(K=15, ld_x=15, ld_w=15, N=1000, ld_y=1000)) == up(4 * 16 * 2) + up(1000 * 16 * 2)
    assert need(grads(), back) == 0
    assert need(grads(act=1, d_pre=Z), back) == up(4 * 8 * 2)
    assert need(grads(act=1, d_pre=Z, d_dz=8 * P, ld_dz=8), back) == 0
    assert need(grads(act=1, d_pre=Z, d_dz=8 * P, ld_dz=9), back) == up(4 * 8 * 2)
    assert need(grads(act=1, d_pre=Z, d_dx=None, d_dw=None), back) == 0
    assert need(grads(ld_x=17, ld_w=17), back) == up(4 * 16 * 2) + up(8 * 16 * 2)
    assert need(grads(ld_x=17, ld_w=17, d_dw=None, d_db=None), back) == up(8 * 16 * 2)
    assert need(grads(M=0), back) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), B.FP_ERR_ARG), (dict(classes=0), B.FP_ERR_ARG), (dict(rows=1 << 31), B.FP_ERR_BOUNDS), (dict(classes=1 << 31, ld_logits=1 << 31), B.FP_ERR_BOUNDS),
    (dict(dtype=3), B.FP_ERR_UNSUPPORTED), (dict(label_bytes=2), B.FP_ERR_ARG), (dict(label_smoothing=-0.1), B.FP_ERR_ARG),
    (dict(label_smoothing=1.5), B.FP_ERR_ARG), (dict(label_smoothing=float("nan")), B.FP_ERR_ARG), (dict(d_logits=None), B.FP_ERR_ARG),
    (dict(d_labels=None), B.FP_ERR_ARG), (dict(d_loss=None, d_dlogits=None), B.FP_ERR_ARG), (dict(ld_logits=7), B.FP_ERR_ARG),
    (dict(ld_dlogits=7), B.FP_ERR_ARG), (dict(d_dlogits=P, ld_logits=9), B.FP_ERR_ARG), (dict(d_logits=P + 2), B.FP_ERR_ARG), (dict(d_labels=P + 4), B.FP_ERR_ARG),
    (dict(d_loss=P + 1), B.FP_ERR_ARG)])
def test_cross_entropy(kw, status):
    a = loss(**kw)
    assert B.lib().fp_cross_entropy(ctypes.addressof(a), None) == status
    assert "fp_cross_entropy" in message()


@pytest.mark.parametrize("kw,hk,status", [
    (dict(n=-1), {}, B.FP_ERR_ARG), (dict(n=1 << 41), {}, B.FP_ERR_BOUNDS), (dict(p_dtype=3), {}, B.FP_ERR_UNSUPPORTED), (dict(g_dtype=-1), {}, B.FP_ERR_UNSUPPORTED),
    (dict(state_bits=16), {}, B.FP_ERR_UNSUPPORTED), (dict(reserved=1), {}, B.FP_ERR_ARG), (dict(d_p=None), {}, B.FP_ERR_ARG), (dict(d_g=None), {}, B.FP_ERR_ARG),
    (dict(d_m=None), {}, B.FP_ERR_ARG), (dict(d_v=None), {}, B.FP_ERR_ARG), (dict(state_bits=8), {}, B.FP_ERR_ARG), (dict(d_mask=P, per_row=0), {}, B.FP_ERR_ARG),
    (dict(d_p=P + 2), {}, B.FP_ERR_ARG), (dict(d_m=P + 2), {}, B.FP_ERR_ARG), ({}, dict(beta1=1.0), B.FP_ERR_ARG), ({}, dict(beta2=-0.1), B.FP_ERR_ARG),
    ({}, dict(eps=-1.0), B.FP_ERR_ARG), ({}, dict(step=0), B.FP_ERR_ARG), ({}, dict(lr=float("inf")), B.FP_ERR_ARG), ({}, dict(grad_scale=float("nan")), B.FP_ERR_ARG),
    ({}, dict(d_lr=P + 2), B.FP_ERR_ARG), ({}, dict(d_step=P + 4), B.FP_ERR_ARG)])
def test_adamw(kw, hk, status):
    arr, h = (B.fp_adamw_tensor * 2)(tensor(), tensor(**kw)), hyper(**hk)
    assert B.lib().fp_adamw_step(ctypes.addressof(arr), 2, ctypes.addressof(h), None) == status
    assert "fp_adamw_step" in message()


def test_null_arguments():
    L, n = B.lib(), ctypes.c_size_t()
    h, a, g = hyper(), linear(), grads()
    assert L.fp_linear_forward(None, None, 0, None) == B.FP_ERR_ARG
    assert L.fp_linear_backward(None, None, 0, None) == B.FP_ERR_ARG
    assert L.fp_linear_workspace(None, ctypes.byref(n)) == B.FP_ERR_ARG
    assert L.fp_linear_workspace(ctypes.addressof(a), None) == B.FP_ERR_ARG
    assert L.fp_linear_backward_workspace(ctypes.addressof(g), None) == B.FP_ERR_ARG
    assert L.fp_linear_status(None) == B.FP_ERR_ARG
    assert L.fp_cross_entropy(None, None) == B.FP_ERR_ARG
    assert L.fp_adamw_step(None, 1, ctypes.addressof(h), None) == B.FP_ERR_ARG
    assert L.fp_adamw_step(None, -1, ctypes.addressof(h), None) == B.FP_ERR_ARG
    assert L.fp_adamw_step(None, 0, None, None) == B.FP_ERR_ARG


def test_struct_sizes_match_the_header():
    assert [ctypes.sizeof(s) for s in (B.fp_linear_args, B.fp_linear_grad_args, B.fp_cross_entropy_args, B.fp_adamw_tensor, B.fp_adamw_hyper)] == \
        [136, 160, 96, 88, 80]


def test_host_tensors_and_wrong_shapes_are_refused_by_the_binding():
    torch = pytest.importorskip("torch")
    x, w, y = (torch.zeros(s, dtype=torch.bfloat16) for s in ((4, 16), (8, 16), (4, 8)))
    with pytest.raises(ValueError):
        B.fp_linear_forward(x, w, y)
    with pytest.raises(ValueError):
        B.fp_linear_backward(y, x, w, dx=x)
    with pytest.raises(ValueError):
        B.fp_cross_entropy(y.float(), torch.zeros(4, dtype=torch.int64), torch.zeros(4))
    with pytest.raises(ValueError):
        B.fp_adamw_tensors([dict(p=torch.zeros(4), g=torch.zeros(4), m=torch.zeros(4), v=torch.zeros(4))])
