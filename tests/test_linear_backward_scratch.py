"""Scratch of a layer's gradients where dz and dy have alignments of their own (host only: no address is read)."""
import ctypes

import pytest

from paper_2010_16165_b200 import binding as B

P = 1 << 20
M, N, K = 4, 8, 16
NEED = 256                # M x N elements of 2 bytes, rounded up


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("d_dy,ld_dy", [(P, 8), (P, 9), (P + 2, 8)])
@pytest.mark.parametrize("d_dz,ld_dz", [(None, 0), (2 * P, 8), (2 * P, 16), (2 * P, 9), (2 * P + 2, 8)])
def test_scratch_for_dz(act, d_dy, ld_dy, d_dz, ld_dz):
    """None where the products can read d_dz, or without an activation d_dy, in place."""
    a = B.fp_linear_grad_args(M=M, N=N, K=K, dtype=B.FP_DTYPE_BF16, dw_dtype=B.FP_DTYPE_F32, act=act, d_dy=d_dy, ld_dy=ld_dy, d_pre=3 * P, ld_pre=8,
                              d_x=4 * P, ld_x=16, d_w=5 * P, ld_w=16, d_dx=6 * P, ld_dx=16, d_dw=7 * P, ld_dw=16, d_dz=d_dz, ld_dz=ld_dz)
    n = ctypes.c_size_t()
    assert B.lib().fp_linear_backward_workspace(ctypes.addressof(a), ctypes.byref(n)) == B.FP_OK
    inside = (d_dz is not None and (d_dz, ld_dz) in ((2 * P, 8), (2 * P, 16))) or (act == 0 and (d_dy, ld_dy) == (P, 8))
    assert n.value == (0 if inside else NEED)
