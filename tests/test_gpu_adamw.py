"""AdamW steps over many tensors against 64-bit arithmetic.

Tolerances.  m and v are two products and a sum in 32 bits: each off by 3 * 2^-24 of its terms' magnitudes.  The step's quotient
takes m (that error), sqrt v (half of v's relative error, 2^-23, and its own rounding), a sum, an approximate division (2 ulp) and three
scalars rounded to 32 bits: 2^-20 of it, and, where m's terms cancel, their error over the divisor; p is then rounded to its type.
8-bit states: a value is off by half a step of e4m3, 2^-4 of it, and half the smallest code, 2^-10 of the scale (a positive root of
v by up to the whole of it, 2^-9); the scale by 2^-22 of it.
"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
BLOCK = 256
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def place(t, offset):
    """A copy that starts `offset` elements into its buffer, and the buffer (the rest of it holds 77)."""
    flat = torch.full((offset + t.numel() + 9,), 77, device="cuda").to(t.dtype)
    flat[offset:offset + t.numel()] = t
    return flat[offset:offset + t.numel()], flat


def make(n, p_dtype, g_dtype, bits, gen, offset=0, rows=0):
    def rn():
        return torch.randn(n, generator=gen, device="cuda")
    size = torch.exp(rn() - 5)
    t, flats = {}, {}
    vals = dict(p=(rn() * 0.1).to(p_dtype), g=(rn() * size).to(g_dtype))
    m, r = rn() * size * 0.3, torch.exp(rn() * 0.5) * size
    if bits == 32:
        vals.update(m=m, v=r * r)
    else:
        blocks = -(-n // BLOCK)
        for k, x in (("m", m), ("v", r)):
            pad = torch.zeros(blocks * BLOCK, device="cuda")
            pad[:n] = x
            scale = (pad.view(-1, BLOCK).abs().amax(1) / 448).clamp(min=1e-30)
            vals[k] = (pad.view(-1, BLOCK) / scale[:, None]).reshape(-1)[:n].to(torch.float8_e4m3fn).view(torch.uint8)
            vals[k + "_scale"] = scale
    if rows:
        vals["mask"] = (torch.rand(rows, generator=gen, device="cuda") > 0.4).to(torch.uint8)
    for k, x in vals.items():
        t[k], flats[k] = place(x, offset)
    return t, flats


def codes(t, k):
    n = t["p"].numel()
    return t[k].view(torch.float8_e4m3fn).double() * t[k + "_scale"].double().repeat_interleave(BLOCK)[:n]


def moments64(t):
    return (codes(t, "m"), codes(t, "v") ** 2) if "m_scale" in t else (t["m"].double(), t["v"].double())


def step64(t, h):
    """p, m, v after a step, the errors of m and v (32 bits), and that of p before it is rounded."""
    m0, v0 = moments64(t)
    g = t["g"].double() * h.get("grad_scale", 1.0)
    b1, b2, lr, wd, eps = h.get("beta1", 0.9), h.get("beta2", 0.999), h["lr"], h.get("weight_decay", 0.01), h.get("eps", 1e-8)
    m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
    me, ve = 3 * 2.0 ** -23 * (b1 * m0.abs() + (1 - b1) * g.abs()) + 1e-44, 5 * 2.0 ** -23 * v + 1e-44
    c1, c2 = 1 - b1 ** h["step"], 1 - b2 ** h["step"]
    div = (v / c2).sqrt() + eps
    upd, pe = lr / c1 * m / div, lr / c1 * me / div
    p0 = t["p"].double()
    p = p0 * (1 - lr * wd) - upd
    pe = pe + 2.0 ** -20 * upd.abs() + 2.0 ** -22 * p0.abs()
    if "mask" in t:
        keep = t["mask"].double().repeat_interleave(-(-t["p"].numel() // t["mask"].numel()))[:t["p"].numel()]
        p, m, v, me, ve, pe = (x * keep for x in (p, m, v, me, ve, pe))
    return p, m, v, me, ve, pe


def check(B, ts, h, **extra):
    """One step over the tensors of ts (pairs of make), and what it did to each."""
    want = [step64(t, h) for t, _ in ts]
    B.fp_adamw_step(B.fp_adamw_tensors([t for t, _ in ts]), **{**h, **extra})
    torch.cuda.synchronize()
    for (t, flats), (p, m, v, me, ve, pe) in zip(ts, want):
        step = torch.finfo(t["p"].dtype).eps / 2 * (p.abs() + pe) + (2.0 ** -25 if t["p"].dtype == F16 else 0)
        assert ((t["p"].double() - p).abs() <= pe + step).all()
        if "m_scale" not in t:
            assert ((t["m"].double() - m).abs() <= me).all() and ((t["v"].double() - v).abs() <= ve).all()
        else:
            n = p.numel()
            for k, x, e in (("m", m, me), ("v", v.sqrt(), ve.sqrt() * 0 + 2.0 ** -21 * v.sqrt())):
                pad = torch.zeros(-(-n // BLOCK) * BLOCK, dtype=torch.float64, device="cuda")
                pad[:n] = x.abs()
                top = pad.view(-1, BLOCK).amax(1) / 448
                pad[:n] = e
                slack = pad.view(-1, BLOCK).amax(1) / 448
                scale = t[k + "_scale"].double()
                assert ((scale - top).abs() <= 2.0 ** -22 * top + slack + 2.0 ** -126).all()
                s = scale.repeat_interleave(BLOCK)[:n]
                assert ((codes(t, k) - x).abs() <= (x.abs() + e) * 2.0 ** -4 * (1 + 2.0 ** -20) + e + s * 2.0 ** (-9 if k == "v" else -10) + 1e-36).all()
                if k == "v":
                    assert ((codes(t, "v") > 0) == ((x > 0) & (s > 0))).all()
        for k, f in flats.items():
            own = t[k].numel()
            at = (t[k].data_ptr() - f.data_ptr()) // f.element_size()
            assert (f[:at].float() == 77).all() and (f[at + own:].float() == 77).all()
        if "mask" in t:
            gone = t["mask"].repeat_interleave(-(-t["p"].numel() // t["mask"].numel()))[:t["p"].numel()] == 0
            assert (t["p"][gone] == 0).all() and (moments64(t)[0][gone] == 0).all() and (moments64(t)[1][gone] == 0).all()


H = dict(lr=1e-2, step=7)
SIZES = [1, 2, 3, 4, 5, 31, 64, 255, 256, 257, 511, 1000, 2048, 4095, 4096, 4097, 8200, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F32, F16), (F32, BF16), (F16, F32), (F16, BF16), (BF16, F16)])
def test_sizes_and_types(B, bits, p, g):
    gen = torch.Generator(device="cuda").manual_seed(1)
    check(B, [make(n, p, g, bits, gen) for n in SIZES], H)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 2, 3, 4, 7, 8])
def test_alignment(B, bits, offset):
    gen = torch.Generator(device="cuda").manual_seed(2)
    check(B, [make(n, d, d, bits, gen, offset) for n in (1, 100, 256, 4500) for d in (F32, BF16)], H)


@pytest.mark.parametrize("bits", [32, 8])
def test_masks(B, bits):
    gen = torch.Generator(device="cuda").manual_seed(3)
    ts = [make(r * c, F32, F32, bits, gen, rows=r) for r, c in ((1, 1), (5, 1), (64, 27), (16, 144), (3, 5000), (1000, 9), (7, 257), (300, 4))]
    ts[4][0]["mask"][:] = 0                              # nothing of a tensor stays
    for t, _ in ts:                                      # and what is pruned need not be finite
        gone = (t["mask"] == 0).repeat_interleave(t["p"].numel() // t["mask"].numel())
        t["g"][gone] = float("nan")
    want = [{k: x.clone() for k, x in t.items()} for t, _ in ts]
    for w in want:
        w["g"] = torch.nan_to_num(w["g"])
    check_masked(B, ts, want)


def check_masked(B, ts, clean):
    """As check, with the expected values from tensors whose gradients were made finite."""
    B.fp_adamw_step(B.fp_adamw_tensors(clean), **H)
    B.fp_adamw_step(B.fp_adamw_tensors([t for t, _ in ts]), **H)
    torch.cuda.synchronize()
    for (t, _), w in zip(ts, clean):
        for k in ("p", "m", "v", "m_scale", "v_scale"):
            assert k not in t or torch.equal(t[k], w[k])
        gone = (t["mask"] == 0).repeat_interleave(t["p"].numel() // t["mask"].numel())
        assert (t["p"][gone] == 0).all() and (moments64(t)[0][gone] == 0).all() and (moments64(t)[1][gone] == 0).all()
        assert (t["p"][~gone] != 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_masks_against_the_formula(B, bits):
    gen = torch.Generator(device="cuda").manual_seed(4)
    check(B, [make(r * c, F32, F32, bits, gen, rows=r) for r, c in ((64, 27), (16, 144), (3, 5000), (1000, 9))], H)


@pytest.mark.parametrize("h", [dict(lr=1e-3, step=1), dict(lr=1e-3, step=1000000), dict(lr=0.5, step=3, weight_decay=0.5, beta1=0.0, beta2=0.5, eps=1e-3),
                               dict(lr=1e-3, step=2, grad_scale=1.0 / 1024), dict(lr=0.0, step=5, weight_decay=0.0)])
@pytest.mark.parametrize("bits", [32, 8])
def test_hyper_parameters(B, bits, h):
    gen = torch.Generator(device="cuda").manual_seed(5)
    check(B, [make(n, F32, F32, bits, gen) for n in (5, 300, 5000)], h)


def test_more_tensors_than_a_launch_takes(B):
    gen = torch.Generator(device="cuda").manual_seed(6)
    ts = [make(1 + (37 * i) % 700, (F32, BF16)[i % 3 == 0], F32, (32, 8)[i % 2], gen) for i in range(1700)]
    check(B, ts, H)


def test_nothing_to_do(B):
    B.fp_adamw_step(B.fp_adamw_tensors([]), lr=1.0)
    e = torch.empty(0, device="cuda")
    B.fp_adamw_step(B.fp_adamw_tensors([dict(p=e, g=e, m=e, v=e)]), lr=1.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_values_at_the_edge(B, bits):
    """Zero gradients and states, and gradients whose squares leave 32 bits: zeros stay zero (p only decays), a block of zeros has scale 0."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    t, flats = make(1024, F32, F32, bits, gen)
    t["g"][:] = 0
    t["m"][:256], t["v"][:256] = 0, 0
    p0 = t["p"].clone()
    check(B, [(t, flats)], H)
    assert (t["p"][:256] - p0[:256] * (1 - 1e-2 * 0.01)).abs().max() <= 2.0 ** -24
    if bits == 8:
        assert t["m_scale"][0] == 0 and t["v_scale"][0] == 0
    t, _ = make(512, F32, F32, bits, gen)
    t["g"][:256] = 1e30                                  # v overflows: a step of m / inf = 0, as the formula in 32 bits has it
    before = t["p"].clone()
    B.fp_adamw_step(B.fp_adamw_tensors([t]), lr=1e-2, weight_decay=0.0)
    assert torch.equal(t["p"][:256], before[:256])
    assert t["p"].isfinite().all() and not torch.equal(t["p"][256:], before[256:])


def test_a_gradient_that_is_not_finite_stays_in_its_element_or_block(B):
    for bits in (32, 8):
        gen = torch.Generator(device="cuda").manual_seed(8)
        t, _ = make(1024, F32, F32, bits, gen)
        w = {k: x.clone() for k, x in t.items()}
        t["g"][300] = float("nan")
        for x in (t, w):
            B.fp_adamw_step(B.fp_adamw_tensors([x]), **H)
        assert t["p"][300].isnan()
        other = torch.arange(1024, device="cuda") != 300
        assert torch.equal(t["p"][other], w["p"][other])
        far = (torch.arange(1024, device="cuda") // 256) != 1
        for a, b in zip(moments64(t), moments64(w)):
            assert torch.equal(a[far], b[far])


def test_8_bit_states_are_what_the_formula_in_32_bits_rounds_to(B):
    """The states' 32-bit values before rounding are sums in a stated order, so that the codes of m can be told bit by bit."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    t, _ = make(256 * 40, F32, BF16, 8, gen)
    g = t["g"].float()
    got = []
    for k in ("m", "v"):
        x = t[k].view(torch.float8_e4m3fn).float() * t[k + "_scale"].repeat_interleave(BLOCK)
        x = x * 0.9 + g * (1 - 0.9) if k == "m" else torch.sqrt(x * x * 0.999 + g * (1 - 0.999) * g)
        scale = x.view(-1, BLOCK).abs().amax(1) * (1.0 / 448)
        q = (x.view(-1, BLOCK) * torch.reciprocal(scale)[:, None]).reshape(-1)
        if k == "v":
            q = torch.where(x > 0, q.clamp(min=2.0 ** -9), q)
        got += [q.to(torch.float8_e4m3fn).view(torch.uint8), scale]
    B.fp_adamw_step(B.fp_adamw_tensors([t]), **H)
    assert torch.equal(t["m"], got[0]) and torch.equal(t["m_scale"], got[1])
    # v's root is off by 2^-22 of itself: the scale by as much and a rounding, a code where the value lies within 2^-20 of a border
    assert ((t["v_scale"] - got[3]).abs() <= 2.0 ** -21 * got[3]).all()
    differ = t["v"] != got[2]
    here, there = (c.view(torch.float8_e4m3fn).double()[differ] for c in (t["v"], got[2]))
    border = (here + there) / 2
    assert ((t["v"].int() - got[2].int()).abs() <= 1).all() and ((q.double()[differ] - border).abs() <= 2.0 ** -20 * border).all()


def test_device_scalars_and_capture(B):
    """A captured step replayed with the step count, rate and gradient scale that device memory holds then."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    for bits in (32, 8):
        a = [make(n, F32, F32, bits, gen) for n in (7, 500, 5000)]
        b = [{k: x.clone() for k, x in t.items()} for t, _ in a]
        lr, scale, step = torch.tensor([0.0], device="cuda"), torch.tensor([0.0], device="cuda"), torch.tensor([0], device="cuda")
        table, plain = B.fp_adamw_tensors([t for t, _ in a]), B.fp_adamw_tensors(b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.fp_adamw_step(table, 123.0, step=99, grad_scale=55.0, d_lr=lr, d_grad_scale=scale, d_step=step, stream=torch.cuda.current_stream())
        for i in range(1, 4):
            rate = float(torch.tensor(1e-2 / i))
            lr.fill_(rate), scale.fill_(0.5), step.fill_(i)
            graph.replay()
            B.fp_adamw_step(plain, rate, step=i, grad_scale=0.5)
            torch.cuda.synchronize()
            for (t, _), w in zip(a, b):
                for k in t:
                    # the device's powers of beta may differ from the host's in their last bits
                    x, y = t[k].float(), w[k].float()
                    assert ((x - y).abs() <= (2.0 ** -22 * y.abs() + 2.0 ** -20 * rate if k == "p" else 0.0 * y)).all()


def test_host_buffers_are_refused(B):
    gen = torch.Generator(device="cuda").manual_seed(11)
    t, _ = make(300, F32, F32, 8, gen, rows=3)
    host = torch.zeros(4096, dtype=torch.uint8).pin_memory()
    for field in ("d_p", "d_g", "d_m", "d_v", "d_m_scale", "d_v_scale", "d_mask"):
        table = B.fp_adamw_tensors([t])
        setattr(table.array[0], field, host.data_ptr())
        with pytest.raises(B.FpError) as e:
            B.fp_adamw_step(table, lr=1.0)
        assert e.value.status == B.FP_ERR_ARG


def test_offsets_beyond_32_bits(B):
    """One tensor of more than 2^31 elements: its last blocks are what the formula makes of them, alone and masked."""
    n = (1 << 31) + 12345
    for masked in (False, True):
        gen = torch.Generator(device="cuda").manual_seed(13)
        tail, _ = make(16 * BLOCK + 12345 % BLOCK, BF16, BF16, 8, gen)
        k, blocks = tail["p"].numel(), -(-n // BLOCK)
        at = n - k
        assert at % BLOCK == 0
        t = dict(p=torch.zeros(n, device="cuda", dtype=BF16), g=torch.zeros(n, device="cuda", dtype=BF16), m=torch.zeros(n, device="cuda", dtype=torch.uint8),
                 v=torch.zeros(n, device="cuda", dtype=torch.uint8), m_scale=torch.zeros(blocks, device="cuda"), v_scale=torch.zeros(blocks, device="cuda"))
        for key in ("p", "g", "m", "v"):
            t[key][at:] = tail[key]
        for key in ("m_scale", "v_scale"):
            t[key][at // BLOCK:] = tail[key]
        if masked:                                       # an entry an element; every third of the last is pruned
            t["mask"] = torch.ones(n, device="cuda", dtype=torch.uint8)
            t["mask"][at::3] = 0
            tail["mask"] = t["mask"][at:].clone()
        B.fp_adamw_step(B.fp_adamw_tensors([t]), **H)
        B.fp_adamw_step(B.fp_adamw_tensors([tail]), **H)
        torch.cuda.synchronize()
        for key in ("p", "m", "v"):
            assert torch.equal(t[key][at:], tail[key])
        for key in ("m_scale", "v_scale"):
            assert torch.equal(t[key][at // BLOCK:], tail[key])
        assert not t["p"][:1 << 20].any() and not t["m_scale"][:1 << 12].any()
        del t
