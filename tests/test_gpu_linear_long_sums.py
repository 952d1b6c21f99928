"""Products with long sums, term by term: every block of 64 terms is added once, and no other one's.

All values are small whole numbers, so that products and sums are exact in 32 bits (below 2^24, and cutting a sum loses nothing): a result equals the exact one
rounded to its type, and a block of the sum that is lost, doubled or another row's shows.  (A bound on the rounding of a sum of random values
grows with its length and soon passes what a block contributes.)
"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def whole(gen, M, N, dtype=BF16, top=2):
    return torch.randint(-top, top + 1, (M, N), generator=gen, device="cuda", dtype=torch.int8).to(dtype)


def product(a, b, piece=8192):
    """a' b of whole numbers, exact: sums of `piece` terms at once stay below 2^24 in 32 bits, theirs in 64."""
    z = torch.zeros(a.shape[1], b.shape[1], dtype=torch.float64, device="cuda")
    for i in range(0, a.shape[0], piece):
        z += (a[i:i + piece].float().t() @ b[i:i + piece].float()).double()
    return z


@pytest.mark.parametrize("M,N,K", [(1, 300, 20000), (16, 136, 70000), (100, 1000, 33000), (300, 264, 40000), (700, 1030, 16384), (2304, 2560, 16500)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_forward(B, M, N, K, out):
    gen = torch.Generator(device="cuda").manual_seed(K)
    x, w = whole(gen, M, K), whole(gen, N, K)
    y = torch.empty(M, N, device="cuda", dtype=out)
    work = torch.empty(B.fp_linear_workspace(x, w, y), dtype=torch.uint8, device="cuda")
    B.fp_linear_forward(x, w, y, work=work)
    assert torch.equal(y, product(x.t(), w.t()).to(out))


@pytest.mark.parametrize("M,N,K", [(16384, 10, 64), (70000, 100, 256), (33000, 264, 136), (40000, 700, 1030), (16500, 2304, 2560),      # long sums of dw
                                   (64, 20000, 200), (300, 33000, 264), (2304, 16500, 2560)])                                          # of dx
@pytest.mark.parametrize("out", [BF16, F32])
def test_gradients(B, M, N, K, out):
    gen = torch.Generator(device="cuda").manual_seed(M + N)
    dy, x, w = whole(gen, M, N), whole(gen, M, K), whole(gen, N, K)
    dx, dw, db = torch.empty(M, K, device="cuda", dtype=BF16), torch.empty(N, K, device="cuda", dtype=out), torch.empty(N, device="cuda", dtype=out)
    for pre in (None, whole(gen, M, N)):
        kw = dict(dx=dx, dw=dw, db=db, pre=pre, act=B.FP_ACT_NONE if pre is None else B.FP_ACT_RELU)
        work = torch.empty(B.fp_linear_backward_workspace(dy, x, w, **kw), dtype=torch.uint8, device="cuda")
        B.fp_linear_backward(dy, x, w, work=work, **kw)
        d = dy if pre is None else dy * (pre > 0)
        assert torch.equal(dx, product(d.t(), w).to(BF16))
        assert torch.equal(dw, product(d, x).to(out))
        assert torch.equal(db, d.sum(0, dtype=torch.float64).to(out))


def test_offsets_beyond_32_bits(B):
    """A batch whose outputs, and a layer whose weights, pass 2^31 elements: all of the forward and all of the gradients of the first, the
    forward and the inputs' gradient of the second."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    M, N, K = 70000, 33000, 32
    x, w = whole(gen, M, K), whole(gen, N, K)
    y = torch.empty(M, N, device="cuda", dtype=BF16)
    B.fp_linear_forward(x, w, y)
    for i in range(0, M, 10000):
        assert torch.equal(y[i:i + 10000], (x[i:i + 10000].float() @ w.float().t()).to(BF16))
    dy = y.clamp_(-2, 2)                                 # whole numbers of two bits, and its own pre: relu of it
    dx, dw = torch.empty(M, K, device="cuda", dtype=BF16), torch.empty(N, K, device="cuda")
    kw = dict(dx=dx, dw=dw, pre=y, act=B.FP_ACT_RELU)
    work = torch.empty(B.fp_linear_backward_workspace(dy, x, w, **kw), dtype=torch.uint8, device="cuda")
    B.fp_linear_backward(dy, x, w, work=work, **kw)
    want = torch.zeros(N, K, dtype=torch.float64, device="cuda")
    for i in range(0, M, 5000):
        d = dy[i:i + 5000].clamp(min=0)
        want += (d.float().t() @ x[i:i + 5000].float()).double()
        assert torch.equal(dx[i:i + 5000], product(d.t(), w).to(BF16))
    assert torch.equal(dw, want.float())
    del x, w, y, dy, dx, dw, work, want, d
    M, N, K = 9, 70000, 33000
    x, w = whole(gen, M, K), whole(gen, N, K)
    y = torch.empty(M, N, device="cuda")
    B.fp_linear_forward(x, w, y)
    for i in range(0, N, 10000):
        assert torch.equal(y[:, i:i + 10000], product(x.t(), w[i:i + 10000].t()).float())
    dy = whole(gen, M, N)
    dx = torch.empty(M, K, device="cuda", dtype=BF16)
    B.fp_linear_backward(dy, None, w, dx=dx)
    assert torch.equal(dx, product(dy.t(), w).to(BF16))
