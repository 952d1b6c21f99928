"""Cross-entropy of finite logits of any size: values that mask classes, and rows that lie far from zero, against 64 bits.

Tolerances.  With m the row's maximum: e^(x-m) is off by 2^-22 and by 2^-23 |x - m| of itself, at most 2^-23 beside the sum (a e^-a < 1); a sum
of C terms and its rescalings by (C / 16 + 60) 2^-22 = r of itself, so log s by r.  x_y - m is one rounded difference, 2^-24 of itself, and the
loss a rounded sum of the two.  A probability is off by r + 2^-23 |x - m| of itself, a gradient by a rounding of its type more.
"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def check(B, x, lab):
    M, C = x.shape
    loss, dx = torch.empty(M, device="cuda"), torch.empty_like(x)
    B.fp_cross_entropy(x, lab, loss, dlogits=dx)
    X, r, own = x.double(), (C / 16 + 60) * 2.0 ** -22, lab[:, None]
    below = X - X.amax(1, keepdim=True)
    logp = torch.log_softmax(below, 1)                   # (of the differences: those of values near 1e30 keep their logarithm)
    want = -logp.gather(1, own)[:, 0]
    assert ((loss.double() - want).abs() <= r + 2.0 ** -23 * below.gather(1, own)[:, 0].abs() + 2.0 ** -23 * want.abs()).all()
    p = logp.exp()
    err = (r + 2.0 ** -23 * below.abs()) * p + 2.0 ** -126
    g = p.scatter_add(1, own, -torch.ones_like(p[:, :1]))
    err = err + 2.0 ** -23 * g.abs()
    assert ((dx.double() - g).abs() <= err + torch.finfo(x.dtype).eps / 2 * (g.abs() + err)).all()


# rows in registers of 8, 32 and 256 threads, in shared memory of one block and of eight, and read twice
SIZES = [(5, 12), (9, 104), (3, 1000), (6, 4096), (300, 12000), (3, 131072), (2, 1800000)]


@pytest.mark.parametrize("fill", [-1e9, -1e10, -1e15, -1e20, -1e30])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,C", SIZES)
def test_a_finite_mask_over_all_that_a_thread_has(B, M, C, dtype, fill):
    """Classes filled with a large negative value: every `period`th 16-byte unit of a row, for each number of threads that share one, half of the
    classes at random, and all but the label."""
    gen = torch.Generator(device="cuda").manual_seed(C)
    E, at = 16 // dtype.itemsize, torch.arange(C, device="cuda")
    masks = [(at // E) % period == 1 for period in (2, 8, 32, 256, 512, 1024, 2048, 4096)] + [torch.rand(C, generator=gen, device="cuda") < 0.5, at >= 0]
    for mask in masks:
        x = (torch.randn(M, C, generator=gen, device="cuda") * 3).to(dtype)
        x[:, mask] = fill
        free = (~mask).nonzero()[:, 0]
        lab = free[torch.randint(0, len(free), (M,), generator=gen, device="cuda")] if len(free) else torch.randint(0, C, (M,), generator=gen, device="cuda")
        x[torch.arange(M, device="cuda"), lab] = 1.5
        check(B, x, lab)


@pytest.mark.parametrize("base", [1e6, 9.9e6, 1e7, 1.1e7, 1e8, 1e9, 3e9, 1e10, 1e12, 1e15, 1e20, 1e30, 1e36, 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,C", SIZES)
def test_rows_far_from_zero(B, M, C, dtype, base):
    gen = torch.Generator(device="cuda").manual_seed(C + 1)
    for sign in (1, -1):
        step = sign * base * torch.finfo(dtype).eps * torch.randint(0, 4, (M, C), generator=gen, device="cuda")
        x = (sign * base - step).to(dtype)
        assert x.isfinite().all()
        check(B, x, torch.randint(0, C, (M,), generator=gen, device="cuda"))


@pytest.mark.parametrize("M,C", SIZES)
def test_a_label_that_is_masked_costs_what_the_mask_is(B, M, C):
    gen = torch.Generator(device="cuda").manual_seed(C + 2)
    x = torch.randn(M, C, generator=gen, device="cuda")
    lab = torch.randint(0, C, (M,), generator=gen, device="cuda")
    x[torch.arange(M, device="cuda"), lab] = -1e10
    check(B, x, lab)
