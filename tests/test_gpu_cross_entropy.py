"""Softmax cross-entropy and its gradient against 64-bit arithmetic.

Tolerances.  With m the row's maximum, e^(x-m) is off by 2^-22 and by 2^-23 |x - m| of itself (rounded argument), which is at most 2^-23 in all beside
the sum, since a e^-a < 1; a sum of C terms in a thread's and then a tree's order is off by at most (C / 32 + 40) 2^-24 of it
(at least 32 threads share a row) - and every rescaling by another maximum by 2^-22, of which a thread has at most as many as terms.
So log s is off by r = (C / 16 + 60) 2^-22 at most, a probability by r + 2^-23 |x - m| of itself.  x_y - m and mean x - m are off
by 2^-23 of |x| and |m|; the mean's sum by (C / 32 + 40) 2^-24 of the mean of |x|.  The gradient is rounded to its type.
"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def check(B, x, lab, smoothing=0.0, scale=1.0, row_grad=None, ignore=-100, in_place=False, pad=0, offset=0, outputs="lg"):
    M, C = x.shape
    loss = torch.full((M,), 5.0, device="cuda") if "l" in outputs else None
    flat = torch.full((offset + M * (C + pad) + 8,), 3.0, device="cuda", dtype=x.dtype)
    dx = flat[offset:offset + M * (C + pad)].view(M, C + pad)[:, :C]
    X = x.double()
    if in_place:
        dx = x
    B.fp_cross_entropy(x, lab, loss, dlogits=dx if "g" in outputs else None, row_grad=row_grad, label_smoothing=smoothing, ignore_index=ignore, grad_scale=scale)
    torch.cuda.synchronize()
    m = X.amax(1, keepdim=True)
    p = torch.softmax(X, 1)
    there = lab != ignore
    q = torch.full_like(X, smoothing / C)
    at = torch.where(there, lab, 0).long()
    q[torch.arange(M, device="cuda"), at] += 1 - smoothing
    r = (C / 16 + 60) * 2.0 ** -22
    want = torch.logsumexp(X, 1) - (1 - smoothing) * X.gather(1, at[:, None])[:, 0] - smoothing * X.mean(1)
    err = r + 2.0 ** -22 * (X.gather(1, at[:, None])[:, 0].abs() + 2 * m[:, 0].abs()) + smoothing * (C / 32 + 40) * 2.0 ** -24 * X.abs().mean(1) + 2.0 ** -23 * want.abs()
    want, err = torch.where(there, want, 0.0), torch.where(there, err, 0.0)
    if loss is not None:
        assert ((loss.double() - want).abs() <= err).all()
    if "g" in outputs:
        g = scale * (row_grad.double() if row_grad is not None else torch.ones(M, dtype=torch.float64, device="cuda")) * there
        want = g[:, None] * (p - q)
        err = g.abs()[:, None] * ((r + 2.0 ** -23 * (X - m).abs()) * p + 2.0 ** -22 * q + 2.0 ** -22 * (p - q).abs() + 2.0 ** -126)
        step = torch.finfo(x.dtype).eps / 2 * (want.abs() + err) + (2.0 ** -25 if x.dtype == torch.float16 else 2.0 ** -126)
        assert ((dx.double() - want).abs() <= err + step).all()
    if not in_place:
        own = torch.zeros_like(flat, dtype=torch.bool)
        own[offset:offset + M * (C + pad)].view(M, C + pad)[:, :C] = "g" in outputs
        assert (flat[~own] == 3).all()
    return loss, dx


def logits(M, C, dtype, seed=0, scale=3.0, pad=0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 * M + C + seed)
    flat = (torch.randn(offset + M * (C + pad), generator=gen, device="cuda") * scale).to(dtype)
    return flat[offset:].view(M, C + pad)[:, :C], torch.randint(0, C, (M,), generator=gen, device="cuda")


DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,C", [(1, 1), (3, 2), (5, 10), (300, 100), (64, 1000), (33, 1001), (7, 4096), (9, 8191), (4, 32000), (150, 33333), (3, 131072),
                                 (2, 150001), (1, 500003), (2, 880000), (1000, 31), (20, 16384), (2000, 2500)])
def test_sizes(B, M, C, dtype):
    x, lab = logits(M, C, dtype)
    check(B, x, lab, scale=1.0 / M)
    check(B, x, lab.int(), smoothing=0.1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (8, 0), (3, 5), (4, 4)])
@pytest.mark.parametrize("M,C", [(6, 1000), (3, 40001), (40, 17)])
def test_strides_and_alignment(B, M, C, dtype, pad, offset):
    x, lab = logits(M, C, dtype, pad=pad, offset=offset)
    check(B, x, lab, smoothing=0.05, pad=pad, offset=offset)


@pytest.mark.parametrize("M,C", [(50, 30), (20, 5000), (3, 140000)])
def test_rows_without_a_label_in_place_and_weighted(B, M, C):
    for dtype in DTYPES:
        x, lab = logits(M, C, dtype)
        lab[::3] = -100
        g = torch.linspace(-2, 2, M, device="cuda")
        check(B, x, lab, smoothing=0.1, row_grad=g, scale=0.25)
        check(B, x.clone(), lab, row_grad=g, in_place=True)
        lab[lab == -100] = 1                             # an index inside the range may be the one that is ignored
        check(B, x, lab, ignore=1)
        check(B, x, lab, outputs="l")
        check(B, x, lab, outputs="g")


@pytest.mark.parametrize("C", [7, 3000, 70000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_extreme_logits(B, C, dtype):
    """The type's largest and lowest values, masked classes (-inf or the lowest value), one class left, equal logits."""
    top = torch.finfo(dtype).max
    x, lab = logits(8, C, dtype)
    lab[:] = 1
    x[0] = -top
    x[1, 2:] = -top
    x[2, 2:] = -float("inf")
    x[3] = -float("inf"); x[3, 1] = -top
    x[4] = 0; x[4, 1] = top
    x[5] = top
    x[6] = x[6, 0]
    loss = torch.empty(8, device="cuda")
    dx = torch.empty_like(x)
    B.fp_cross_entropy(x, lab, loss, dlogits=dx)
    X = x.double()
    want = -torch.log_softmax(X, 1)[:, 1]                # (a logsumexp of such values loses the logarithm even in 64 bits)
    r = (C / 16 + 60) * 2.0 ** -22
    assert ((loss.double() - want).abs() <= r + 2.0 ** -21 * torch.where(want > 1e4, want, torch.zeros_like(want)) + 2.0 ** -20).all()
    p = torch.softmax(X, 1)
    p[:, 1] -= 1
    assert ((dx.double() - p).abs() <= 2 * r + torch.finfo(dtype).eps / 2 * p.abs() + 2.0 ** -25).all()


@pytest.mark.parametrize("C", [5, 2000, 60000, 200000])
def test_what_is_not_finite_stays_in_its_row(B, C):
    x, lab = logits(9, C, torch.float32)
    clean, cg = check(B, x, lab)
    x[1, C - 1] = float("nan")
    x[3, 0] = float("inf")
    x[5] = -float("inf")
    lab[7] = C                                           # outside the classes
    lab[8] = -1
    loss, dx = torch.empty(9, device="cuda"), torch.empty(9, C, device="cuda")
    B.fp_cross_entropy(x, lab, loss, dlogits=dx)
    bad = torch.tensor([0, 1, 0, 1, 0, 1, 0, 1, 1], device="cuda").bool()
    assert loss[bad].isnan().all() and dx[bad].isnan().all()
    assert torch.equal(loss[~bad], clean[~bad]) and torch.equal(dx[~bad], cg[~bad])
    lab[:] = -100                                        # nothing is asked of the rows: nothing comes of them
    B.fp_cross_entropy(x, lab, loss, dlogits=dx)
    assert (loss == 0).all() and (dx == 0).all()


def test_masked_label_costs_infinity(B):
    x, lab = logits(3, 50, torch.float32)
    x[1, lab[1]] = -float("inf")
    loss = torch.empty(3, device="cuda")
    B.fp_cross_entropy(x, lab, loss)
    assert loss[1] == float("inf") and loss[0].isfinite() and loss[2].isfinite()


def test_gradient_against_differences(B):
    """(loss(x + h e_j) - loss(x - h e_j)) / 2h differs from the gradient by h^2 / 6 of a third derivative below 1/4 and by the losses'
    errors over h."""
    x, lab = logits(6, 12, torch.float32, scale=1.0)
    h = 2.0 ** -6
    dx = torch.empty_like(x)
    B.fp_cross_entropy(x, lab, None, dlogits=dx, label_smoothing=0.2)
    for j in range(12):
        got = []
        for s in (h, -h):
            y, loss = x.clone(), torch.empty(6, device="cuda")
            y[:, j] += s
            B.fp_cross_entropy(y, lab, loss, label_smoothing=0.2)
            got.append(loss.double())
        assert ((got[0] - got[1]) / (2 * h) - dx[:, j].double()).abs().max() <= h * h / 24 + 70 * 2.0 ** -22 / h


def test_same_bits_every_time_and_under_capture(B):
    for M, C in ((30, 1000), (3, 100000)):
        x, lab = logits(M, C, torch.bfloat16)
        loss, dx = torch.empty(M, device="cuda"), torch.empty_like(x)
        B.fp_cross_entropy(x, lab, loss, dlogits=dx)
        first = loss.clone(), dx.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.fp_cross_entropy(x, lab, loss, dlogits=dx, stream=torch.cuda.current_stream())
        for _ in range(2):
            loss.zero_(), dx.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(loss, first[0]) and torch.equal(dx, first[1])


def test_no_rows_and_host_buffers(B):
    x = torch.empty(0, 10, device="cuda")
    B.fp_cross_entropy(x, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), dlogits=x)
    x, lab = logits(4, 8, torch.float32)
    import ctypes
    for field in ("d_labels", "d_loss", "d_logits", "d_dlogits", "d_row_grad"):
        loss = torch.empty(4, device="cuda")
        a = B.fp_cross_entropy_args(4, 8, 0, 8, -100, 0.0, 1.0, x.data_ptr(), lab.data_ptr(), None, loss.data_ptr(), None, 8, 8)
        host = torch.zeros(64, dtype=torch.int64).pin_memory()
        setattr(a, field, host.data_ptr())
        assert B.lib().fp_cross_entropy(ctypes.addressof(a), None) == B.FP_ERR_ARG


def test_offsets_beyond_32_bits(B):
    M, C = 17000, 131072
    x = torch.empty(M, C, device="cuda", dtype=torch.bfloat16).normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    lab = torch.arange(M, device="cuda") * 7 % C
    loss = torch.empty(M, device="cuda")
    last = x[-3:].clone()
    B.fp_cross_entropy(x, lab, loss, dlogits=x)
    X = last.double()
    want = -torch.log_softmax(X, 1).gather(1, lab[-3:, None])[:, 0]
    r = (C / 16 + 60) * 2.0 ** -22
    assert ((loss[-3:].double() - want).abs() <= r + 2.0 ** -20 * (X.abs().amax(1) + want)).all()
    p = torch.softmax(X, 1)
    p[torch.arange(3, device="cuda"), lab[-3:]] -= 1
    assert ((x[-3:].double() - p).abs() <= (2 * r + 2.0 ** -8) * p.abs() + 2.0 ** -126).all()
