"""Fully connected layers and their gradients against 64-bit sums.

Tolerances.  A product of two 16-bit values is exact in 32 bits; a sum of K of them on the tensor cores, which may cut instead
of rounding, is off by at most 2^-23 of the running sum a term, so by K 2^-23 S with S the sum of the terms' magnitudes.
Bias and residual are two roundings more.  An activation passes an error on with its largest slope (gelu: 1.13) and adds its own evaluation, 2^-20
of the value (exponential, division, erf: some ulp each) and, for the cancellation of 1 + erf near -1, 2^-22 of |z|.  The result is rounded by half a step of
its type, 2^-25 at least in f16, whose small values are subnormal.
"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = "bfloat16", "float16", "float32"
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def act64(name, z):
    if name == "relu":
        return torch.relu(z)                             # (whose derivative at 0 is 0; that of clamp is 1)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(name, z):
    z = z.clone().requires_grad_()
    g, = torch.autograd.grad(act64(name, z).sum(), z) if name != "none" else (torch.ones_like(z),)
    return g.detach()


def half_step(dtype, y):
    return torch.finfo(dtype).eps / 2 * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)


def rows(gen, M, N, dtype, pad=0, offset=0, scale=1.0):
    """M x N values, rows `pad` elements apart, the first one `offset` elements into its buffer."""
    flat = (torch.randn(offset + M * (N + pad), generator=gen, device="cuda") * scale).to(dtype)
    return flat[offset:].view(M, N + pad)[:, :N]


def guarded(M, N, dtype, pad=0, offset=0):
    """An output of NaN in a larger buffer, and a function that says whether all around it is untouched."""
    flat = torch.full((offset + M * (N + pad) + 16,), float("nan"), device="cuda", dtype=dtype)
    t = flat[offset:offset + M * (N + pad)].view(M, N + pad)[:, :N]

    def untouched():
        own = torch.zeros_like(flat, dtype=torch.bool)
        own[offset:offset + M * (N + pad)].view(M, N + pad)[:, :N] = True
        return bool(flat[~own].isnan().all())
    return t, untouched


def forward_case(B, M, N, K, dtype=BF16, act="none", out=None, bias=F32, res=None, pre=False, pad=0, offset=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 31 * M + 7 * N + K)
    dt, ot = getattr(torch, dtype), getattr(torch, out or dtype)
    x, w = rows(gen, M, K, dt, pad, offset), rows(gen, N, K, dt, pad, offset, K ** -0.5)
    b = torch.randn(N, generator=gen, device="cuda").to(getattr(torch, bias)) if bias else None
    r = rows(gen, M, N, dt, pad, offset) if res else None
    y, y_ok = guarded(M, N, ot, pad, offset)
    p, p_ok = guarded(M, N, dt, pad, offset) if pre else (None, lambda: True)
    kw = dict(bias=b, res=r, pre=p, act=ACTS.index(act), res_first=res == "before")
    work = torch.empty(B.fp_linear_workspace(x, w, y, **kw), dtype=torch.uint8, device="cuda")
    B.fp_linear_forward(x, w, y, work=work, **kw)
    assert B.fp_linear_status() == B.FP_OK
    z = x.double() @ w.double().t()
    S = x.double().abs() @ w.double().abs().t()
    err = K * 2.0 ** -23 * S
    if b is not None:
        z, S = z + b.double(), S + b.double().abs()
    if res == "before":
        z, S = z + r.double(), S + r.double().abs()
    err = err + 2 * 2.0 ** -24 * S
    if pre:
        assert ((p.double() - z).abs() <= err + half_step(dt, z)).all() and p_ok()
    if act != "none":
        v = act64(act, z)
        err = 1.13 * err + 2.0 ** -20 * v.abs() + 2.0 ** -22 * z.abs()
        z = v
    if res == "after":
        z = z + r.double()
        err = err + 2.0 ** -24 * (z.abs() + err)
    assert ((y.double() - z).abs() <= err + half_step(ot, z)).all()
    assert y_ok()


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 1000, 2048), (2, 3, 5), (16, 128, 64), (17, 129, 65), (33, 257, 200), (64, 10, 4096), (65, 96, 8),
                                   (128, 128, 128), (129, 127, 63), (300, 520, 1000), (256, 256, 64), (1000, 777, 192), (4, 8192, 512), (2049, 16, 72)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_sizes(B, M, N, K, dtype):
    forward_case(B, M, N, K, dtype)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("res", [None, "after", "before"])
@pytest.mark.parametrize("M", [5, 200, 700])
def test_epilogues(B, act, res, M):
    forward_case(B, M, 136, 72, act=act, res=res, pre=True)
    forward_case(B, M, 131, 72, dtype=F16, act=act, res=res, pre=True, bias=F16, pad=3)


@pytest.mark.parametrize("M,N,K", [(3, 50, 70), (130, 200, 130), (600, 300, 257)])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (8, 0), (4, 4), (3, 7)])
def test_strides_and_alignment(B, M, N, K, pad, offset):
    forward_case(B, M, N, K, act="silu", res="after", pre=True, pad=pad, offset=offset)
    forward_case(B, M, N, K, dtype=F16, out=F32, bias=None, pad=pad, offset=offset)


@pytest.mark.parametrize("M", [1, 90, 400, 3000])
def test_float_outputs_and_long_sums(B, M):
    forward_case(B, M, 264, 8192, out=F32)
    forward_case(B, M, 264, 8200, dtype=F16, out=F32, res="before", act="relu")


def test_many_tiles(B):
    """More tiles than the GPU takes at once, and ragged ones at every end."""
    forward_case(B, 2500, 5000, 136, act="gelu", pre=True)


@pytest.mark.parametrize("M,N,K,act,out", [(2100, 2050, 520, "none", F32), (2304, 2048, 2304, "gelu", BF16), (9000, 72, 2200, "silu", F32), (136, 9000, 4100, "relu", BF16),
                                           (4097, 515, 1030, "gelu_tanh", F32)])
@pytest.mark.parametrize("pad", [0, 1])
def test_gradients_of_many_tiles(B, M, N, K, act, out, pad):
    backward_case(B, M, N, K, act=act, out=out, pad=pad)


def test_epilogues_of_many_tiles(B):
    for res in (None, "after", "before"):
        forward_case(B, 2100, 2310, 72, act="gelu", res=res, pre=True)
        forward_case(B, 2100, 2311, 200, dtype=F16, out=F32, act="silu", res=res, pre=True, bias=F16, pad=3)
    backward_case(B, 2100, 2052, 2049, act="relu", out=BF16, accumulate=True, dz=True)


def test_no_rows(B):
    x, w, y = (torch.empty(s, device="cuda", dtype=torch.bfloat16) for s in ((0, 16), (8, 16), (0, 8)))
    B.fp_linear_forward(x, w, y)
    dw, db = torch.full((8, 16), 3.0, device="cuda"), torch.full((8,), 3.0, device="cuda")
    B.fp_linear_backward(y, x, w, dx=x, dw=dw, db=db, accumulate=True)
    assert (dw == 3).all() and (db == 3).all()
    wide = torch.full((8, 20), 3.0, device="cuda")
    B.fp_linear_backward(y, x, w, dx=x, dw=wide[:, :16], db=db)
    assert (wide[:, :16] == 0).all() and (wide[:, 16:] == 3).all() and (db == 0).all()


@pytest.mark.parametrize("M", [7, 200, 900])
def test_what_is_not_finite_stays_in_its_row_and_column(B, M):
    """No value of one row, column or padding reaches another; a sum that meets an infinity or NaN has it by IEEE rules."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    K, N = 100, 150
    x, w = rows(gen, M, K, torch.bfloat16, 4), rows(gen, N, K, torch.bfloat16, 4)
    x.as_strided((M, 4), (K + 4, 1), K).fill_(float("nan"))             # behind the rows' ends
    w.as_strided((N, 4), (K + 4, 1), K).fill_(float("inf"))
    y, clean = (torch.empty(M, N, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    work = torch.empty(B.fp_linear_workspace(x, w, y), dtype=torch.uint8, device="cuda")
    B.fp_linear_forward(x, w, clean, work=work)
    assert clean.isfinite().all()
    x[2, 5], x[4, 99], w[9, 0] = float("nan"), float("inf"), float("-inf")
    B.fp_linear_forward(x, w, y, work=work)
    want = x.double() @ w.double().t()
    assert (y.isfinite() == want.isfinite()).all() and (y.isnan() == want.isnan()).all()
    ok = want.isfinite()
    assert (y[ok] == clean[ok]).all()


@pytest.mark.parametrize("act", ACTS)
def test_activations_of_extreme_values(B, act):
    """Through a 1 x 1 identity: the largest values, zeros, infinities and NaN give what the formula gives in 64 bits (or its limit)."""
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3e38, -3e38, 88.0, -88.0, 10.0, -10.0, 1e10, -1e10, float("nan"), float("inf")], device="cuda")
    x = v.to(torch.bfloat16)[:, None].contiguous()
    one = torch.ones(1, 1, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(len(v), 1, device="cuda")
    work = torch.empty(B.fp_linear_workspace(x, one, y), dtype=torch.uint8, device="cuda")
    B.fp_linear_forward(x, one, y, act=ACTS.index(act), work=work)
    z = x.double()
    want = act64(act, z)
    ok = want.isfinite()
    assert (y.isnan() == want.isnan()).all() and (y[want.isinf()] == want[want.isinf()].float()).all()
    assert ((y.double() - want).abs()[ok] <= (2.0 ** -19 * want.abs() + 2.0 ** -21 * z.abs().clamp(max=100) + 1e-37)[ok]).all()
    # and the derivative
    dz = torch.empty_like(x)
    B.fp_linear_backward(torch.ones_like(x), None, None, dz=dz, pre=x if act != "none" else None, act=ACTS.index(act))
    fine = x[:12]
    want = slope64(act, fine.double())
    want = torch.where(want.isnan(), (fine > 0).double(), want)          # (inf times 0 in the reference itself)
    assert ((dz[:12].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20).all()


def backward_case(B, M, N, K, dtype=BF16, act="none", out=F32, pad=0, offset=0, dz=False, accumulate=False, want="xwb"):
    gen = torch.Generator(device="cuda").manual_seed(17 * M + 5 * N + K)
    dt, ot = getattr(torch, dtype), getattr(torch, out)
    dy, x, w = rows(gen, M, N, dt, pad, offset), rows(gen, M, K, dt, pad, offset), rows(gen, N, K, dt, pad, offset, K ** -0.5)
    pre = rows(gen, M, N, dt, pad, offset) if act != "none" else None
    dx, dx_ok = guarded(M, K, dt, pad, offset) if "x" in want else (None, lambda: True)
    dw, dw_ok = guarded(N, K, ot, pad, offset) if "w" in want else (None, lambda: True)
    db = torch.full((N,), float("nan"), device="cuda", dtype=ot) if "b" in want else None
    z, z_ok = guarded(M, N, dt, pad, offset) if dz else (None, lambda: True)
    dw0 = db0 = 0.0
    if accumulate:
        dw.copy_(torch.randn(N, K, generator=gen, device="cuda")), db.copy_(torch.randn(N, generator=gen, device="cuda"))
        dw0, db0 = dw.double(), db.double()
    kw = dict(dx=dx, dw=dw, db=db, dz=z, pre=pre, act=ACTS.index(act), accumulate=accumulate)
    xs, ws = (x if "w" in want else None), (w if "x" in want else None)
    work = torch.empty(B.fp_linear_backward_workspace(dy, xs, ws, **kw), dtype=torch.uint8, device="cuda")
    B.fp_linear_backward(dy, xs, ws, work=work, **kw)
    assert B.fp_linear_status() == B.FP_OK
    d = dy.double()
    # the slope: evaluated in 32 bits (2^-20 of values of at most 1.13, plus 2^-22 |z| of the cancellation), then one product
    e = torch.zeros_like(d)
    if act != "none":
        s = slope64(act, pre.double())
        e = d.abs() * (2.0 ** -20 * (1 + s.abs()) + 2.0 ** -22 * pre.double().abs())
        d = d * s
    db_err = e.sum(0) + M * 2.0 ** -24 * d.abs().sum(0)
    if dz:
        assert ((z.double() - d).abs() <= e + half_step(dt, d)).all() and z_ok()
    if act != "none":
        e = e + half_step(dt, d)                         # the products take dz rounded
    D = d.abs() + e
    if "x" in want:
        v, err = d @ w.double(), e @ w.double().abs() + N * 2.0 ** -23 * (D @ w.double().abs())
        assert ((dx.double() - v).abs() <= err + half_step(dt, v.abs() + err)).all() and dx_ok()
    if "w" in want:
        v, err = d.t() @ x.double(), e.t() @ x.double().abs() + M * 2.0 ** -23 * (D.t() @ x.double().abs())
        v, err = v + dw0, err + 2.0 ** -24 * (v.abs() + err)
        assert ((dw.double() - v).abs() <= err + half_step(ot, v.abs() + err)).all() and dw_ok()
    if "b" in want:
        v = d.sum(0) + db0
        err = db_err + 2.0 ** -24 * v.abs()
        assert ((db.double() - v).abs() <= err + half_step(ot, v.abs() + err)).all()


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 1000, 512), (2, 3, 5), (64, 10, 64), (100, 64, 16), (128, 128, 128), (129, 130, 131), (256, 1000, 2048),
                                   (700, 96, 200), (1000, 257, 65), (33, 2000, 24)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gradient_sizes(B, M, N, K, dtype):
    backward_case(B, M, N, K, dtype)
    backward_case(B, M, N, K, dtype, act="gelu", out=dtype)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (8, 4), (5, 3)])
def test_gradient_activations_and_strides(B, act, pad, offset):
    backward_case(B, 150, 140, 90, act=act, pad=pad, offset=offset, dz=True)
    backward_case(B, 40, 72, 136, dtype=F16, act=act, out=F16, pad=pad, offset=offset)


@pytest.mark.parametrize("want", ["x", "w", "b", "xb", "wb", "xw"])
@pytest.mark.parametrize("M", [20, 500])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_single_gradients(B, want, M, act):
    backward_case(B, M, 88, 200, act=act, want=want)


@pytest.mark.parametrize("out", [F32, BF16])
def test_gradients_are_added_to_what_is_there(B, out):
    backward_case(B, 300, 140, 75, act="relu", out=out, accumulate=True)


def test_gradient_in_place_of_its_input(B):
    gen = torch.Generator(device="cuda").manual_seed(3)
    dy, pre, w = rows(gen, 60, 100, torch.bfloat16), rows(gen, 60, 100, torch.bfloat16), rows(gen, 100, 40, torch.bfloat16)
    kw = dict(pre=pre, act=B.FP_ACT_SILU)
    outs = []
    for dz in (torch.empty_like(dy), dy):
        dx = torch.empty(60, 40, device="cuda", dtype=torch.bfloat16)
        work = torch.empty(B.fp_linear_backward_workspace(dy, None, w, dx=dx, dz=dz, **kw), dtype=torch.uint8, device="cuda")
        B.fp_linear_backward(dy, None, w, dx=dx, dz=dz, work=work, **kw)
        outs.append((dx, dz))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_residual_in_place_of_the_output(B):
    gen = torch.Generator(device="cuda").manual_seed(4)
    for M in (9, 300):
        x, w, r = rows(gen, M, 64, torch.bfloat16), rows(gen, 72, 64, torch.bfloat16), rows(gen, M, 72, torch.bfloat16)
        y = torch.empty_like(r)
        B.fp_linear_forward(x, w, y, res=r, act=B.FP_ACT_RELU)
        B.fp_linear_forward(x, w, r, res=r, act=B.FP_ACT_RELU)
        assert torch.equal(y, r)


def test_gradient_against_differences(B):
    """The layer's own outputs moved by +-h along a direction give the gradient's product with it: with f32 outputs the difference
    of two sums is known to about K 2^-23 of their terms each, the cubic term is h^2 times the third derivative (< 2)."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    M, N, K, h = 24, 40, 64, 2.0 ** -5
    x = (torch.randint(-64, 65, (M, K), generator=gen, device="cuda") / 64).to(torch.bfloat16)     # x +- h v is exact in bf16
    v = torch.randint(-1, 2, (M, K), generator=gen, device="cuda").to(torch.bfloat16)
    w = rows(gen, N, K, torch.bfloat16, scale=K ** -0.5)
    dy = torch.ones(M, N, device="cuda", dtype=torch.bfloat16)
    y = [torch.empty(M, N, device="cuda") for _ in range(2)]
    pre, plain = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), torch.empty(M, N, device="cuda")
    for s, t in zip((1, -1), y):
        B.fp_linear_forward((x.float() + s * h * v.float()).to(torch.bfloat16), w, t, act=B.FP_ACT_GELU)
    B.fp_linear_forward(x, w, plain, pre=pre, act=B.FP_ACT_GELU)
    dx = torch.empty(M, K, device="cuda", dtype=torch.bfloat16)
    work = torch.empty(B.fp_linear_backward_workspace(dy, None, w, dx=dx, pre=pre, act=B.FP_ACT_GELU), dtype=torch.uint8, device="cuda")
    B.fp_linear_backward(dy, None, w, dx=dx, pre=pre, act=B.FP_ACT_GELU, work=work)
    got = (dx.double() * v.double()).sum(1)
    want = ((y[0].double() - y[1].double()) / (2 * h)).sum(1)
    wv = (v.double().abs() @ w.double().abs().t())
    direction = (v.double() @ w.double().t()).abs()
    # bf16 roundings of pre (slope' < 1.2), dz and dx; truncation of the difference; the two sums' errors over 2 h
    tol = (direction * (1.2 * 2.0 ** -8 * pre.double().abs() + 1.13 * 2.0 ** -8) + h * h / 3 * direction ** 3).sum(1) + \
        2.0 ** -8 * (dx.double().abs() * v.double().abs()).sum(1) + N * K * 2.0 ** -23 / h + 2.0 ** -20 * wv.sum(1)
    assert ((got - want).abs() <= tol).all()


def test_same_bits_every_time_and_under_capture(B):
    """Captured and replayed on a side stream, with other calls in between, the results keep their bits."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    M, N, K = 200, 264, 520
    x, w, dy, pre = (rows(gen, *s, torch.bfloat16) for s in ((M, K), (N, K), (M, N), (M, N)))
    y, dx = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda", dtype=torch.bfloat16)
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    kw = dict(dx=dx, dw=dw, db=db, pre=pre, act=B.FP_ACT_GELU)
    work = torch.empty(B.fp_linear_backward_workspace(dy, x, w, **kw), dtype=torch.uint8, device="cuda")

    def both(stream):
        B.fp_linear_forward(x, w, y, stream=stream)
        B.fp_linear_backward(dy, x, w, work=work, stream=stream, **kw)
    both(torch.cuda.current_stream())
    first = [t.clone() for t in (y, dx, dw, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(torch.cuda.current_stream())
    for _ in range(3):
        for t in (y, dx, dw, db):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (y, dx, dw, db)))


@pytest.mark.parametrize("M,N", [(4, 300), (100, 300), (300, 520), (2304, 2560)])
def test_sums_in_32_bits_are_not_cut_short(B, M, N):
    """The tensor cores cut a sum toward zero at every 16 terms, by 2^-23 of it at most.  A 32-bit result is summed in runs of 512 terms
    (1024 where tensor memory holds no more runs): 64 cuts, so it is too small by 64 * 2^-23 of itself at most, not by 1024 * 2^-23 as 16384 terms in one run
    could be (measured: 1.6e-5).  That is where every cut takes a whole unit of a sum of its final size; a cut takes half a unit on average,
    of sums that grow up to that size: a quarter.  The runs' rounded sums have no direction."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    K = 16384
    x, w = rows(gen, M, K, torch.bfloat16), rows(gen, N, K, torch.bfloat16, scale=K ** -0.5)
    y = torch.empty(M, N, device="cuda")
    B.fp_linear_forward(x, w, y)
    z = x.double() @ w.double().t()
    short = -((y.double() - z) * z.sign()).mean() / z.abs().mean()
    assert short <= 64 * 2.0 ** -23 / 4 and (y.double() - z).norm() <= 64 * 2.0 ** -23 / 4 * z.norm()


@pytest.mark.parametrize("M,N,K", [(3000, 10, 200), (5000, 16, 136), (2500, 100, 65), (9000, 3, 33), (700, 128, 64)])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_gradients_of_narrow_layers(B, M, N, K, act):
    backward_case(B, M, N, K, act=act, dz=True)
    backward_case(B, M, N, K, dtype=F16, act=act, out=F16, want="xwb")


# Column sums by the last product's launch (no activation, few tiles) and by one of their own, on both sides of each limit.
@pytest.mark.parametrize("M,N,K,pad", [(1, 300, 64, 0), (64, 1003, 520, 5), (129, 131, 200, 5), (256, 1000, 2048, 0), (300, 2048, 1000, 0), (2048, 264, 128, 0),
                                       (2049, 264, 128, 0), (1500, 9000, 64, 0), (1500, 9600, 64, 0), (640, 128, 4096, 8)])
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("want", ["xwb", "wb", "xb"])
def test_column_sums_beside_the_products(B, M, N, K, pad, dtype, out, want):
    backward_case(B, M, N, K, dtype=dtype, out=out, pad=pad, accumulate=want == "xwb", want=want)


def test_calls_that_follow_each_other_share_their_scratch(B):
    """Twenty layers one after the other through one scratch buffer, each reading what the one before has written: launches that overlap
    keep their order."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    for M, N in ((3, 65), (70, 129), (300, 131), (2000, 2051)):
        w = [rows(gen, N, N, torch.bfloat16, pad=1, scale=N ** -0.5) for _ in range(4)]
        x0 = rows(gen, M, N, torch.bfloat16, pad=1)
        bufs = [torch.empty(M, N, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        work = torch.empty(B.fp_linear_workspace(x0, w[0], bufs[0]) + B.fp_linear_workspace(bufs[0], w[0], bufs[1]), dtype=torch.uint8, device="cuda")

        def run(wait):
            x = x0
            for i in range(20):
                y = bufs[i % 2]
                B.fp_linear_forward(x, w[i % 4], y, act=B.FP_ACT_SILU, res=x0, work=work)
                if wait:
                    torch.cuda.synchronize()
                x = y
            dx, dw = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), torch.empty(N, N, device="cuda")
            for i in range(6):
                kw = dict(dx=dx, dw=dw, db=None, pre=x0, act=B.FP_ACT_SILU)
                scratch = back if i % 2 else back2
                B.fp_linear_backward(x, x0, w[i % 4], work=scratch, **kw)
                B.fp_linear_forward(dx, w[0], x, work=work)
                if wait:
                    torch.cuda.synchronize()
            return x.clone(), dx.clone(), dw.clone()
        need = B.fp_linear_backward_workspace(bufs[1], x0, w[0], dx=bufs[0], dw=torch.empty(N, N, device="cuda"), pre=x0, act=B.FP_ACT_SILU)
        back, back2 = (torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2))
        first = run(True)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, run(False)))


def test_calls_of_every_form_on_two_streams(B):
    """Single rows, small, split and large products queued on two streams at once give what they give alone."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    cases = []
    for M, N, K in ((1, 1000, 2048), (40, 512, 4096), (300, 300, 4096), (1000, 777, 520), (2304, 2304, 512), (2, 8192, 512)):
        x, w = rows(gen, M, K, torch.bfloat16), rows(gen, N, K, torch.bfloat16, scale=K ** -0.5)
        y = torch.empty(M, N, device="cuda")
        B.fp_linear_forward(x, w, y)
        cases.append((x, w, y, y.clone()))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(c[2]) for c in cases] for _ in streams]
    torch.cuda.synchronize()
    for i in range(30):
        for k, st in enumerate(streams):
            j = (i * (k + 1) + k) % len(cases)
            B.fp_linear_forward(cases[j][0], cases[j][1], outs[k][j], stream=st)
    torch.cuda.synchronize()
    for k in range(2):
        for i in range(30):
            j = (i * (k + 1) + k) % len(cases)
            assert torch.equal(outs[k][j], cases[j][3])
    assert B.fp_linear_status() == B.FP_OK


def test_scratch_that_is_too_small_or_not_on_the_device_is_refused(B):
    x, w, y = (torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((200, 15), (8, 15), (200, 8)))
    need = B.fp_linear_workspace(x, w, y)
    assert need > 0
    for work in (None, torch.empty(need - 1, dtype=torch.uint8, device="cuda")):
        with pytest.raises(B.FpError) as e:
            B.fp_linear_forward(x, w, y, work=work)
        assert e.value.status == B.FP_ERR_BOUNDS
    for work in (torch.empty(need + 256, dtype=torch.uint8, device="cuda")[8:], torch.empty(need, dtype=torch.uint8).pin_memory()):
        with pytest.raises(B.FpError) as e:
            B.fp_linear_forward(x, w, y, work=work)
        assert e.value.status == B.FP_ERR_ARG


def test_host_buffers_are_refused(B):
    import ctypes
    x, w, y = (torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((16, 16), (8, 16), (16, 8)))
    host = torch.zeros(4096, dtype=torch.uint8).pin_memory()
    for field in ("d_x", "d_w", "d_y", "d_res", "d_pre", "d_bias"):
        a = B._linear_args(x, w, y, None, None, None, 0, False)
        a.ld_res = a.ld_pre = 8
        setattr(a, field, host.data_ptr())
        assert B.lib().fp_linear_forward(ctypes.addressof(a), None, 0, None) == B.FP_ERR_ARG
        assert b"current device" in B.lib().fp_last_error()


def test_offsets_beyond_32_bits(B):
    """A batch whose outputs, and a layer whose weights, pass 2^31 elements: the rows at both ends."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    for M, N, K in ((70000, 33000, 32), (9, 70000, 33000)):
        x, w = rows(gen, M, K, torch.bfloat16), torch.randn(N, K, generator=gen, device="cuda", dtype=torch.bfloat16)
        y = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
        B.fp_linear_forward(x, w, y)
        for part in (slice(0, 4), slice(M - 5, M)):
            for cols in (slice(0, 300), slice(N - 300, N)):
                z, S = x[part].double() @ w[cols].double().t(), x[part].double().abs() @ w[cols].double().abs().t()
                assert ((y[part, cols].double() - z).abs() <= K * 2.0 ** -23 * S + half_step(torch.bfloat16, z)).all()
        # and back: dz of that size, through scratch of that size
        dx, dw = torch.empty(M, K, device="cuda", dtype=torch.bfloat16), torch.empty(N, K, device="cuda", dtype=torch.bfloat16)
        kw = dict(dx=dx, dw=dw, pre=y, act=B.FP_ACT_RELU)
        work = torch.empty(B.fp_linear_backward_workspace(y, x, w, **kw), dtype=torch.uint8, device="cuda")
        B.fp_linear_backward(y, x, w, work=work, **kw)
        d = y[M - 3:].double().clamp(min=0)
        z, S = torch.zeros(3, K, dtype=torch.float64, device="cuda"), torch.zeros(3, K, dtype=torch.float64, device="cuda")
        for a in range(0, N, 10000):
            z += d[:, a:a + 10000] @ w[a:a + 10000].double()
            S += d[:, a:a + 10000] @ w[a:a + 10000].double().abs()
        assert ((dx[M - 3:].double() - z).abs() <= N * 2.0 ** -23 * S + half_step(torch.bfloat16, z)).all()
        d = y[:, N - 3:].double().clamp(min=0)
        z, S = d.t() @ x.double(), d.t() @ x.double().abs()
        assert ((dw[N - 3:].double() - z).abs() <= M * 2.0 ** -23 * S + half_step(torch.bfloat16, z)).all()
        del x, w, y, dx, dw, work
