"""The training-step calls as a program uses them: a pruned two-layer classifier is trained for a few steps - layers, loss, gradients, AdamW,
filters ranked and masked by the library, masked steps - and every step is compared with the same step in 64 bits from the same
weights.

Tolerances.  A rounding to bf16 is off by r = 2^-8 of the value.  h is rounded, so logits are off by t = r sum |h| |w1|, the loss by 2t, p by
2.5 t p (e^2t - 1 for t < 0.2); the logits' gradient is that and a rounding; dx of the upper layer is a product with it and a rounding;
the slope is taken of a rounded pre (|gelu''| < 0.8, gelu' < 1.13) and dz0 rounded.  Each error goes on linearly through the products' magnitudes; 5 %
covers second orders and the 32-bit sums.
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


class Step:
    """One training step's calls on buffers that are made once, so that it can be captured."""

    def __init__(self, B, n, d, hidden, classes, bits, gen):
        self.B, bf = B, torch.bfloat16
        new = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)   # noqa: E731
        self.x, self.lab = torch.randn(n, d, generator=gen, device="cuda").to(bf), torch.randint(0, classes, (n,), generator=gen, device="cuda")
        self.W = [torch.randn(hidden, d, generator=gen, device="cuda") * d ** -0.5, torch.randn(classes, hidden, generator=gen, device="cuda") * hidden ** -0.5]
        self.b = [new(hidden), new(classes)]
        self.w16 = [w.to(bf) for w in self.W]
        self.h, self.pre, self.logits, self.loss = new(n, hidden, dt=bf), new(n, hidden, dt=bf), new(n, classes), new(n)
        self.dlogits, self.d16, self.dh = new(n, classes), new(n, classes, dt=bf), new(n, hidden, dt=bf)
        self.dW, self.db = [new(hidden, d), new(classes, hidden)], [new(hidden), new(classes)]
        self.rank, self.mask = new(hidden, dt=torch.int32), torch.ones(hidden, device="cuda", dtype=torch.uint8)
        self.lr, self.t = torch.full((1,), 1e-2, device="cuda"), torch.zeros(1, device="cuda", dtype=torch.int64)
        ts = []
        for p, g, mask in zip(self.W + self.b, self.dW + self.db, (self.mask, None, self.mask, None)):
            k, blocks = p.numel(), -(-p.numel() // B.FP_ADAMW_BLOCK)
            t = dict(p=p, g=g, mask=mask)
            if bits == 8:
                t.update(m=new(k, dt=torch.uint8), v=new(k, dt=torch.uint8), m_scale=new(blocks), v_scale=new(blocks))
            else:
                t.update(m=new(k), v=new(k))
            ts.append(t)
        self.table = B.fp_adamw_tensors(ts)
        back1 = B.fp_linear_backward_workspace(self.d16, self.h, self.w16[1], dx=self.dh, dw=self.dW[1], db=self.db[1])
        back0 = B.fp_linear_backward_workspace(self.dh, self.x, None, dw=self.dW[0], db=self.db[0], pre=self.pre, act=B.FP_ACT_GELU)
        fwd = max(B.fp_linear_workspace(self.x, self.w16[0], self.h), B.fp_linear_workspace(self.h, self.w16[1], self.logits))
        self.work = torch.empty(max(back0, back1, fwd), dtype=torch.uint8, device="cuda")

    def gradients(self):
        B, s = self.B, torch.cuda.current_stream()
        for a, w in zip(self.w16, self.W):
            a.copy_(w)
        B.fp_linear_forward(self.x, self.w16[0], self.h, bias=self.b[0], pre=self.pre, act=B.FP_ACT_GELU, work=self.work, stream=s)
        B.fp_linear_forward(self.h, self.w16[1], self.logits, bias=self.b[1], work=self.work, stream=s)
        B.fp_cross_entropy(self.logits, self.lab, self.loss, dlogits=self.dlogits, label_smoothing=0.1, grad_scale=1.0 / len(self.lab), stream=s)
        self.d16.copy_(self.dlogits)
        B.fp_linear_backward(self.d16, self.h, self.w16[1], dx=self.dh, dw=self.dW[1], db=self.db[1], work=self.work, stream=s)
        B.fp_linear_backward(self.dh, self.x, None, dw=self.dW[0], db=self.db[0], pre=self.pre, act=B.FP_ACT_GELU, work=self.work, stream=s)

    def select(self, q):
        self.B.fp_rank_filters_static(self.W[0], self.W[0].shape[0], self.W[0].shape[1], self.B.FP_NORM_L2, q, self.rank, self.mask,
                                      stream=torch.cuda.current_stream())

    def update(self):
        self.t.add_(1)
        self.B.fp_adamw_step(self.table, 0.0, d_lr=self.lr, d_step=self.t, stream=torch.cuda.current_stream())

    def run(self):
        self.gradients()
        self.update()


def check_gradients(s):
    """The step's gradients against autograd in 64 bits, from the weights as the layers read them."""
    w = [a.double().requires_grad_() for a in s.w16]
    b = [a.double().requires_grad_() for a in s.b]
    z0 = s.x.double() @ w[0].t() + b[0]
    h = z0 * torch.special.ndtr(z0)
    logp = torch.log_softmax(h @ w[1].t() + b[1], 1)
    n, C = logp.shape
    q = torch.full_like(logp, 0.1 / C)
    q[torch.arange(n, device="cuda"), s.lab] += 0.9
    loss = -(q * logp).sum(1)
    loss.mean().backward()
    p = logp.exp().detach()
    r = 2.0 ** -8
    H, w1, x, p, z0 = h.detach().abs(), w[1].detach().abs(), s.x.double().abs(), logp.exp().detach(), z0.detach().abs()
    t = r * (H @ w1.t()).amax(1, keepdim=True)
    assert ((s.loss.double() - loss.detach()).abs() <= 1.05 * 2 * t[:, 0]).all()
    D, E = (p - q).abs() / n, (2.5 * t * p + r * (p - q).abs()) / n
    G, GE = D @ w1, E @ w1 + r * (D @ w1)
    ZE = 1.13 * GE + 0.8 * r * z0 * (G + GE) + 1.13 * r * (G + GE)
    for got, want, bound in ((s.dW[1], w[1].grad, E.t() @ H + r * (D.t() @ H)), (s.db[1], b[1].grad, E.sum(0)),
                             (s.dW[0], w[0].grad, ZE.t() @ x), (s.db[0], b[0].grad, ZE.sum(0))):
        assert ((got.double() - want).abs() <= 1.05 * bound).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n,d,hidden,classes", [(64, 100, 96, 10), (256, 512, 260, 1000), (33, 75, 50, 7)])
def test_training_a_pruned_classifier(B, bits, n, d, hidden, classes):
    gen = torch.Generator(device="cuda").manual_seed(n)
    s = Step(B, n, d, hidden, classes, bits, gen)
    for i in range(6):
        if i == 3:                                       # prune the weakest hidden units, and keep them out
            s.select(hidden // 3)
        s.gradients()
        if i in (0, 5):
            check_gradients(s)
        s.update()
        if i >= 3:
            gone = s.mask == 0
            assert int(gone.sum()) == hidden // 3
            assert (s.W[0][gone] == 0).all() and (s.b[0][gone] == 0).all() and (s.W[0][~gone] != 0).any(1).all()
    assert B.fp_linear_status() == B.FP_OK
    assert s.t.item() == 6 and all(w.isfinite().all() for w in s.W)


def test_a_captured_step_is_the_eager_one(B):
    outs = []
    for captured in (False, True):
        gen = torch.Generator(device="cuda").manual_seed(1)
        s = Step(B, 100, 90, 70, 12, 8, gen)
        s.select(20)
        s.run()                                          # (a first step outside the capture)
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                s.run()
        for _ in range(4):
            graph.replay() if captured else s.run()
        torch.cuda.synchronize()
        outs.append([t.clone() for t in s.W + s.b + [s.loss]])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_two_programs_on_two_streams(B):
    """Two trainings queued at the same time on streams of their own, each with its scratch, do not touch each other."""
    def train(streams):
        steps = [Step(B, 120, 200, 150, 30, 32, torch.Generator(device="cuda").manual_seed(k)) for k in range(2)]
        torch.cuda.synchronize()
        for _ in range(10):
            for s, st in zip(steps, streams):
                with torch.cuda.stream(st):
                    s.run()
        torch.cuda.synchronize()
        return [t for s in steps for t in s.W + s.b]
    alone = train([torch.cuda.current_stream()] * 2)
    both = train([torch.cuda.Stream(), torch.cuda.Stream()])
    assert all(torch.equal(a, b) for a, b in zip(alone, both))
