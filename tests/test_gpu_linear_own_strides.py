"""Gradients of a layer whose buffers have strides and alignments of their own, each independent of the others, against exact sums.

All values are small whole numbers: products and sums of them are exact in 32 bits (and cutting a sum loses nothing), so a result
equals the 64-bit one rounded to its type.
"""
import itertools

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def placed(gen, M, N, dtype, pad, offset):
    flat = torch.randint(-3, 4, (offset + M * (N + pad),), generator=gen, device="cuda").to(dtype)
    return flat[offset:].view(M, N + pad)[:, :N]


def one(B, M, N, K, at, act="none", out=torch.float32, accumulate=False, want="xwb", dtype=torch.bfloat16):
    """`at`: (pad, offset) of dy, dz, x, w by name; a multiple of eight elements each is what can be read in place."""
    gen = torch.Generator(device="cuda").manual_seed(M + 3 * N + 7 * K)
    dy, x, w = placed(gen, M, N, dtype, *at["dy"]), placed(gen, M, K, dtype, *at["x"]), placed(gen, N, K, dtype, *at["w"])
    pre = placed(gen, M, N, dtype, *at["dy"]) if act != "none" else None
    dz = placed(gen, M, N, dtype, *at["dz"])
    dx = torch.full((M, K), 7.0, device="cuda", dtype=dtype) if "x" in want else None
    dw = torch.full((N, K), 2.0, device="cuda", dtype=out) if "w" in want else None
    db = torch.full((N,), 3.0, device="cuda", dtype=out) if "b" in want else None
    kw = dict(dx=dx, dw=dw, db=db, dz=dz, pre=pre, act=1 if act == "relu" else 0, accumulate=accumulate)
    xs, ws = (x if "w" in want else None), (w if "x" in want else None)
    work = torch.empty(B.fp_linear_backward_workspace(dy, xs, ws, **kw), dtype=torch.uint8, device="cuda")
    B.fp_linear_backward(dy, xs, ws, work=work, **kw)
    d = dy.double() * ((pre > 0).double() if act == "relu" else 1.0)
    assert torch.equal(dz.double(), d)
    if "x" in want:
        assert torch.equal(dx, (d @ w.double()).to(dtype))
    if "w" in want:
        assert torch.equal(dw, (d.t() @ x.double() + 2.0 * accumulate).to(out))
    if "b" in want:
        assert torch.equal(db, (d.sum(0) + 3.0 * accumulate).to(out))


ALIGNED, WIDER, SHIFTED, ODD = (0, 0), (8, 0), (0, 3), (1, 0)


@pytest.mark.parametrize("M,N,K", [(4, 8, 16), (40, 72, 136), (200, 264, 88), (1, 64, 64), (3000, 2048, 264)])
@pytest.mark.parametrize("dy,dz", [(ALIGNED, ODD), (ALIGNED, SHIFTED), (WIDER, ODD), (ODD, ALIGNED), (SHIFTED, WIDER), (ODD, SHIFTED), (ALIGNED, WIDER)])
def test_dz_lies_otherwise_than_dy(B, M, N, K, dy, dz):
    for act in ("none", "relu"):
        for want in ("xwb", "x", "w", "b"):
            one(B, M, N, K, dict(dy=dy, dz=dz, x=ALIGNED, w=ALIGNED), act, want=want, accumulate="w" in want and "b" in want)


@pytest.mark.parametrize("M,N,K", [(40, 72, 136), (300, 264, 520)])
def test_every_buffer_lies_as_it_likes(B, M, N, K):
    for i, (dy, dz, x, w) in enumerate(itertools.product((ALIGNED, ODD), (ALIGNED, SHIFTED), (WIDER, ODD), (ALIGNED, SHIFTED))):
        one(B, M, N, K, dict(dy=dy, dz=dz, x=x, w=w), ("none", "relu")[i % 2], (torch.float32, torch.float16)[i // 2 % 2], bool(i & 4), dtype=torch.float16)


def test_dz_beside_a_dy_that_is_read_in_place_needs_no_scratch(B):
    dy, x, w = (torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((4, 8), (4, 16), (8, 16)))
    dz = torch.zeros(4, 9, device="cuda", dtype=torch.bfloat16)[:, :8]
    dx, dw = torch.empty(4, 16, device="cuda", dtype=torch.bfloat16), torch.empty(8, 16, device="cuda")
    assert B.fp_linear_backward_workspace(dy, x, w, dx=dx, dw=dw, dz=dz) == 0
    B.fp_linear_backward(dy, x, w, dx=dx, dw=dw, dz=dz)
    assert not dx.any() and not dw.any() and not dz.any()
