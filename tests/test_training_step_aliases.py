"""Outputs of the training-step calls that are another buffer of the call are refused, before any GPU is asked; what the header allows is not."""
import ctypes

import pytest

from paper_2010_16165_b200 import binding as B

P = 1 << 20          # addresses that are never read
X, W, Y, Z, A, C = (P * k for k in (2, 3, 4, 5, 6, 7))


def refused(status):
    """Whether a call was refused for such an output, and not for its addresses, which no GPU knows (or for the lack of one)."""
    return status == B.FP_ERR_ARG and "output" in B.lib().fp_last_error().decode()


def cross_entropy(**kw):
    d = dict(rows=4, classes=8, dtype=B.FP_DTYPE_F32, label_bytes=4, ignore_index=-100, label_smoothing=0.0, grad_scale=1.0, d_logits=X, d_labels=W, d_row_grad=Y,
             d_loss=Z, d_dlogits=A, ld_logits=8, ld_dlogits=8)
    d.update(kw)
    a = B.fp_cross_entropy_args(**d)
    return B.lib().fp_cross_entropy(ctypes.addressof(a), None)


@pytest.mark.parametrize("kw", [dict(d_loss=X), dict(d_loss=W), dict(d_loss=Y), dict(d_loss=A), dict(d_dlogits=W), dict(d_dlogits=Y),
                                dict(d_loss=W, d_dlogits=None), dict(d_loss=None, d_dlogits=Y), dict(d_loss=X, d_dlogits=X)])
def test_cross_entropy(kw):
    assert refused(cross_entropy(**kw))


@pytest.mark.parametrize("kw", [{}, dict(d_dlogits=X), dict(d_row_grad=None), dict(d_loss=None), dict(d_dlogits=None), dict(d_row_grad=None, d_loss=None), dict(d_labels=Y)])
def test_cross_entropy_of_other_buffers(kw):
    assert not refused(cross_entropy(**kw))


def linear(**kw):
    d = dict(M=4, N=8, K=16, dtype=B.FP_DTYPE_BF16, y_dtype=B.FP_DTYPE_BF16, bias_dtype=B.FP_DTYPE_BF16, act=0, res_first=0, reserved=0, d_x=X, d_w=W,
             d_bias=A, d_res=Z, d_y=Y, d_pre=C, ld_x=16, ld_w=16, ld_res=8, ld_y=8, ld_pre=8)
    d.update(kw)
    a = B.fp_linear_args(**d)
    return B.lib().fp_linear_forward(ctypes.addressof(a), None, 0, None)


@pytest.mark.parametrize("kw", [dict(d_y=A), dict(d_pre=A), dict(d_pre=A, d_res=None), dict(d_pre=Z), dict(d_pre=Y)])
def test_linear(kw):
    assert refused(linear(**kw))


@pytest.mark.parametrize("kw", [{}, dict(d_y=Z), dict(d_bias=None), dict(d_bias=None, d_pre=None), dict(d_bias=Z), dict(d_x=Z, d_w=Z, d_bias=Z)])
def test_linear_of_other_buffers(kw):
    assert not refused(linear(**kw))


def scratch_refused(status):
    return status == B.FP_ERR_ARG and "scratch is" in B.lib().fp_last_error().decode() and "another buffer" in B.lib().fp_last_error().decode()


@pytest.mark.parametrize("work", [X, W, Y, Z, A, C])
def test_scratch_of_linear(work):
    """Rows 17 elements apart are copied into scratch, which is no other buffer of the call then; where none is needed it is not looked at."""
    for ld, wanted in ((17, True), (16, False)):
        a = B.fp_linear_args(M=4, N=8, K=16, dtype=B.FP_DTYPE_BF16, y_dtype=B.FP_DTYPE_BF16, bias_dtype=B.FP_DTYPE_BF16, act=0, res_first=0, reserved=0, d_x=X, d_w=W,
                             d_bias=A, d_res=Z, d_y=Y, d_pre=C, ld_x=ld, ld_w=16, ld_res=8, ld_y=8, ld_pre=8)
        assert scratch_refused(B.lib().fp_linear_forward(ctypes.addressof(a), work, 1 << 16, None)) == wanted


@pytest.mark.parametrize("work", [X, W, Y, Z, A, C, 8 * P, 9 * P])
def test_scratch_of_linear_gradients(work):
    for ld, wanted in ((17, True), (16, False)):
        a = B.fp_linear_grad_args(M=4, N=8, K=16, dtype=B.FP_DTYPE_BF16, dw_dtype=B.FP_DTYPE_F32, act=1, accumulate=0, d_dy=Y, d_pre=Z, d_x=X, d_w=W, d_dx=A, d_dw=C,
                                  d_db=8 * P, d_dz=9 * P, ld_dy=8, ld_pre=8, ld_x=ld, ld_w=16, ld_dx=16, ld_dw=16, ld_dz=8)
        assert scratch_refused(B.lib().fp_linear_backward(ctypes.addressof(a), work, 1 << 16, None)) == wanted


@pytest.mark.parametrize("kw,work", [(dict(act=0), Z), (dict(d_dw=None), X), (dict(d_dx=None), W)])
def test_scratch_in_place_of_what_is_not_read(kw, work):
    d = dict(M=4, N=8, K=16, dtype=B.FP_DTYPE_BF16, dw_dtype=B.FP_DTYPE_F32, act=1, accumulate=0, d_dy=Y, d_pre=Z, d_x=X, d_w=W, d_dx=A, d_dw=C,
             d_db=8 * P, d_dz=None, ld_dy=9, ld_pre=8, ld_x=16, ld_w=16, ld_dx=16, ld_dw=16, ld_dz=8)
    d.update(kw)
    a = B.fp_linear_grad_args(**d)
    assert not scratch_refused(B.lib().fp_linear_backward(ctypes.addressof(a), work, 1 << 16, None))


def adamw(hyper=None, **kw):
    d = dict(n=64, per_row=8, p_dtype=0, g_dtype=0, state_bits=8, reserved=0, d_p=X, d_g=W, d_m=Y, d_v=Z, d_m_scale=A, d_v_scale=C, d_mask=8 * P)
    d.update(kw)
    ts = (B.fp_adamw_tensor * 2)(B.fp_adamw_tensor(n=64, p_dtype=0, g_dtype=0, state_bits=32, d_p=20 * P, d_g=21 * P, d_m=22 * P, d_v=23 * P), B.fp_adamw_tensor(**d))
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, d_lr=9 * P, d_grad_scale=10 * P, d_step=11 * P)
    h.update(hyper or {})
    h = B.fp_adamw_hyper(**h)
    return B.lib().fp_adamw_step(ctypes.addressof(ts), 2, ctypes.addressof(h), None)


@pytest.mark.parametrize("kw", [dict(d_g=X), dict(d_m=X), dict(d_v=X), dict(d_v=Y), dict(d_m=W), dict(d_m_scale=Z), dict(d_v_scale=A), dict(d_m_scale=W), dict(d_mask=X), dict(d_mask=C),
                                dict(d_g=X, state_bits=32), dict(d_m=Z, state_bits=32), dict(d_mask=Y, state_bits=32),
                                dict(hyper=dict(d_lr=X)), dict(hyper=dict(d_step=Z)), dict(hyper=dict(d_grad_scale=20 * P)), dict(hyper=dict(d_lr=C))])
def test_adamw(kw):
    assert refused(adamw(**kw))


@pytest.mark.parametrize("kw", [{}, dict(d_mask=None), dict(d_mask=W), dict(d_m_scale=X, d_v_scale=X, state_bits=32), dict(n=0, d_g=X, d_m=X, d_v=X),
                                dict(hyper=dict(d_lr=W, d_step=None, d_grad_scale=W)), dict(hyper=dict(d_lr=None, d_step=None, d_grad_scale=None))])
def test_adamw_of_other_buffers(kw):
    assert not refused(adamw(**kw))
