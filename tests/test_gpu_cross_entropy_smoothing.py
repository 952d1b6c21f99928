"""Smoothed cross-entropy where the mean of the logits is large beside what the loss is made of, against 64 bits.

With x_y the label's logit and m the maximum, loss = log s + (m - x_y) - e mean(x - x_y).  log s is off by r = (C / 16 + 60) 2^-22 (see the other tests of the
loss), m - x_y by a rounding, and the mean, a sum of C rounded differences in a thread's and then a tree's order, by (C / 32 + 44) 2^-24 of the
mean of |x - x_y|.  Three roundings of the result are 2^-22 of its terms.
"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(5, 12), (9, 104), (3, 1000), (300, 12000), (3, 131072), (2, 1800000)]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def check(B, x, lab, e):
    M, C = x.shape
    loss = torch.empty(M, device="cuda")
    B.fp_cross_entropy(x, lab, loss, label_smoothing=e)
    X, own = x.double(), lab[:, None]
    m, y = X.amax(1), X.gather(1, own)[:, 0]
    log_s, mean, size = torch.logsumexp(X - m[:, None], 1), (X - y[:, None]).mean(1), (X - y[:, None]).abs().mean(1)
    e = float(torch.tensor(e, dtype=torch.float32))
    want = log_s + (m - y) - e * mean
    err = (C / 16 + 60) * 2.0 ** -22 + e * (C / 32 + 44) * 2.0 ** -24 * size + 2.0 ** -22 * (log_s + (m - y) + e * mean.abs())
    assert ((loss.double() - want).abs() <= err).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,C", SIZES)
def test_classes_masked_by_the_lowest_value(B, M, C, dtype):
    """Their mean is finite, though the sum of two of them is not."""
    gen = torch.Generator(device="cuda").manual_seed(C)
    x = (torch.randn(M, C, generator=gen, device="cuda") * 3).to(dtype)
    x[:, 1::2] = torch.finfo(dtype).min
    check(B, x, torch.randint(0, C // 2, (M,), generator=gen, device="cuda") * 2, 0.1)
    x[:, 2:] = torch.finfo(dtype).min
    check(B, x, torch.zeros(M, dtype=torch.int64, device="cuda"), 0.1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,C", SIZES)
def test_rows_of_one_value(B, M, C, dtype):
    lab = torch.arange(M, device="cuda") % C
    for v in (torch.finfo(dtype).max, torch.finfo(dtype).min, 1e4, -3.0, 0.0):
        check(B, torch.full((M, C), v, device="cuda", dtype=dtype), lab, 0.1)


@pytest.mark.parametrize("M,C", SIZES)
def test_logits_with_a_common_offset(B, M, C):
    gen = torch.Generator(device="cuda").manual_seed(C + 1)
    for offset in (1e3, -1e4, 1e6):
        x = torch.randn(M, C, generator=gen, device="cuda") * 3 + offset
        for e in (0.1, 0.7):
            check(B, x, torch.randint(0, C, (M,), generator=gen, device="cuda"), e)


@pytest.mark.parametrize("M,C", SIZES)
def test_all_of_the_target_smoothed(B, M, C):
    gen = torch.Generator(device="cuda").manual_seed(C + 2)
    x = torch.randn(M, C, generator=gen, device="cuda") * 3
    lab = torch.randint(0, C, (M,), generator=gen, device="cuda")
    check(B, x, lab, 1.0)
    # and with a class of probability 0, the label's or another one's, the loss is infinite, whatever the smoothing
    loss = torch.empty(M, device="cuda")
    for own in (True, False):
        z = x.clone()
        z[0, lab[0] if own else (lab[0] + 1) % C] = -float("inf")
        for e in (0.25, 1.0):
            B.fp_cross_entropy(z, lab, loss, label_smoothing=e)
            assert loss[0] == float("inf") and loss[1:].isfinite().all()


@pytest.mark.parametrize("M,C", SIZES)
def test_rows_without_a_loss(B, M, C):
    """Rows without a label have loss 0, labels outside the classes NaN, and so have NaN, +inf and rows of -inf."""
    gen = torch.Generator(device="cuda").manual_seed(C + 3)
    x = torch.randn(M, C, generator=gen, device="cuda")
    lab = torch.randint(0, C, (M,), generator=gen, device="cuda")
    loss = torch.empty(M, device="cuda")
    for row in (float("nan"), float("inf"), -float("inf")):
        z = x.clone()
        z[1, :] = row if row < 0 else z[1, :]
        z[1, C - 1] = row
        B.fp_cross_entropy(z, lab, loss, label_smoothing=0.3)
        assert loss[1].isnan() and loss[0].isfinite()
        other = lab.clone()
        other[1] = -100
        B.fp_cross_entropy(z, other, loss, label_smoothing=0.3)
        assert loss[1] == 0 and loss[0].isfinite()
    lab[0] = C
    B.fp_cross_entropy(x, lab, loss, label_smoothing=0.3)
    assert loss[0].isnan() and loss[1].isfinite()
