"""What the speed of the training-step operators is measured on: the calls with which a program retrains a (pruned) network.

A case is a dict of plain values:

    kind      "linear"  y = act(x w' + bias) + res, or act(x w' + bias + res): a fully connected layer
              "grads"   its gradients: dz = dy * act'(pre), dx = dz w, dw = dz' x, db = column sums of dz
              "loss"    softmax cross-entropy of a batch of logits, and its gradient
              "adamw"   one AdamW step over all tensors of a network
    M, N, K   linear, grads: rows (images or tokens), outputs, inputs
    dtype     of the inputs and, where nothing else is said, of the outputs: "bf16", "f16" or "f32"
    act       "none", "relu", "gelu" (with erf), "gelu_tanh", "silu"
    pad       elements between the end of a row of x, w, dy, pre, res or the logits and the start of the next one
    out       linear: dtype of y; grads: of dw and db
    res       linear: "none", "after" or "before" the activation; keep_pre: what the activation is taken of is written too
    rows, classes, smoothing, ignored (share of rows without a label), labels ("i32", "i64")    loss
    net       adamw: "resnet20", "resnet50" or "drawn" (`count` tensors up to `largest` elements, by `shapes`)
    grad, state  adamw: dtype of the gradients; "f32", or "f8" for states of 8 bits in blocks of 256
    pruned    adamw: share of the filters of every tensor with more than one that a mask holds at zero
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
BLOCK = 256                  # elements of a tensor that share one scale of an 8-bit state
TOP, TINY = 448.0, 2.0 ** -9  # largest and smallest positive value of the 8-bit type
HYPER = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "step": 1000}
INV_SQRT_2, INV_SQRT_2PI, SQRT_2_PI = math.sqrt(0.5), 1.0 / math.sqrt(2.0 * math.pi), math.sqrt(2.0 / math.pi)


def _linear(M, N, K, dtype="bf16", act="none", out=None, res="none", keep_pre=False, pad=0):
    return {"kind": "linear", "M": M, "N": N, "K": K, "dtype": dtype, "act": act, "out": out or dtype, "res": res,
            "keep_pre": keep_pre, "pad": pad}


def _grads(M, N, K, dtype="bf16", act="none", out=None, pad=0):
    return {"kind": "grads", "M": M, "N": N, "K": K, "dtype": dtype, "act": act, "out": out or dtype, "pad": pad}


def _loss(rows, classes, dtype="f32", smoothing=0.0, ignored=0.0, labels="i64", pad=0):
    return {"kind": "loss", "rows": rows, "classes": classes, "dtype": dtype, "smoothing": smoothing, "ignored": ignored,
            "labels": labels, "pad": pad}


def _adamw(net, dtype="f32", grad="f32", state="f32", pruned=0.0, count=0, largest=0, shapes=0):
    return {"kind": "adamw", "net": net, "dtype": dtype, "grad": grad, "state": state, "pruned": pruned, "count": count,
            "largest": largest, "shapes": shapes}


def listed():
    return [
        # the classifier of a bottleneck network on one image: single-request latency
        dict(_linear(1, 1000, 2048, out="f32"), name="linear_1x1000x2048"),
        # a decoding step of sixteen sequences through a wide layer: the weights' bytes are the whole cost
        dict(_linear(16, 16384, 4096, act="gelu_tanh"), name="linear_16x16384x4096"),
        # a ragged batch through an odd-sized layer whose rows are not aligned, with a residual
        dict(_linear(1003, 777, 2050, dtype="f16", act="silu", res="after", pad=1), name="linear_1003x777x2050_f16"),
        # a large training batch through a wide layer that keeps what its backward pass needs
        dict(_linear(8192, 16384, 4096, act="gelu", keep_pre=True), name="linear_8192x16384x4096"),
        # the classifier's gradients for a batch of 256 images, in 32 bits for the optimizer
        dict(_grads(256, 1000, 2048, out="f32"), name="grads_256x1000x2048"),
        # the wide layer's gradients
        dict(_grads(8192, 16384, 4096, act="gelu"), name="grads_8192x16384x4096"),
        # the loss of a batch of 256 images over 1000 classes, labels smoothed
        dict(_loss(256, 1000, smoothing=0.1), name="loss_256x1000"),
        # few rows over very many classes
        dict(_loss(4, 131072, dtype="f16", labels="i32"), name="loss_4x131072_f16"),
        # a large batch over many classes, some rows without a label
        dict(_loss(8192, 32000, dtype="bf16", ignored=0.1), name="loss_8192x32000_bf16"),
        # the smallest network of the library, 59 tensors: launches and latency
        dict(_adamw("resnet20"), name="adamw_resnet20"),
        # the library's largest, 161 tensors, while 40 % of the filters are held at zero
        dict(_adamw("resnet50", pruned=0.4), name="adamw_resnet50_pruned"),
        # a large model whose states would not fit in 32 bits
        dict(_adamw("drawn", dtype="bf16", grad="bf16", state="f8", count=24, largest=1 << 26, shapes=7), name="adamw_large_f8"),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "grads", "loss", "adamw"))
    if kind in ("linear", "grads"):
        M, N, K = _between(rng, 1, 8192), _between(rng, 10, 16384), _between(rng, 16, 8192)
        K = max(16, min(K, 8192 * 16384 * 4096 // (M * N)))
        if rng.random() < 0.5:       # most layers' widths are round, batches need not be
            N, K = -(-N // 64) * 64, -(-K // 64) * 64
            while M * N * K > 8192 * 16384 * 4096:
                K -= 64
        dtype, act, pad = rng.choice(("bf16", "f16")), rng.choice(sorted(ACTS)), rng.choice((0, 0, 0, 1, 8))
        if kind == "grads":
            return _grads(M, N, K, dtype, act, rng.choice((dtype, "f32")) if act == "none" else dtype, pad)
        return _linear(M, N, K, dtype, act, rng.choice((dtype, dtype, "f32")), rng.choice(("none", "after", "before")),
                       rng.random() < 0.3, pad)
    if kind == "loss":
        classes = _between(rng, 2, 150000)
        rows = _between(rng, 1, max(1, min(65536, 8192 * 32000 // (2 * classes))))
        return _loss(rows, classes, rng.choice(("f32", "bf16", "f16")), rng.choice((0.0, 0.1)), rng.choice((0.0, 0.1)),
                     rng.choice(("i32", "i64")), rng.choice((0, 0, 1, 8)))
    dtype = rng.choice(("f32", "bf16", "f16"))
    return _adamw("drawn", dtype, rng.choice((dtype, "f32")), rng.choice(("f32", "f8")), rng.choice((0.0, 0.0, 0.3)),
                  rng.randint(1, 200), _between(rng, 64, 1 << 20), rng.randrange(1 << 30))


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _resnet20():
    """(filters, weights per filter) of every tensor: convolutions, the two vectors of each batch norm, the classifier."""
    convs = [(16, 27)] + [(w, 9 * (v if b == 0 and half == 0 else w)) for v, w in ((16, 16), (16, 32), (32, 64))
                          for b in range(3) for half in range(2)]
    return [t for c in convs for t in (c, (1, c[0]), (1, c[0]))] + [(10, 64), (1, 10)]


def _resnet50():
    def block(cin, w, first):
        return [(w, cin), (w, 9 * w), (4 * w, w)] + ([(4 * w, cin)] if first else [])
    convs = [(64, 147)] + [c for w, before, n in ((64, 64, 3), (128, 256, 4), (256, 512, 6), (512, 1024, 3))
                           for b in range(n) for c in block(before if b == 0 else 4 * w, w, b == 0)]
    return [t for c in convs for t in (c, (1, c[0]), (1, c[0]))] + [(1000, 2048), (1, 1000)]


def _drawn(case):
    rng = random.Random(case["shapes"])
    sizes = [_between(rng, 16, case["largest"]) for _ in range(case["count"] - 1)] + [case["largest"]]
    rows = [_between(rng, 1, max(1, n // 8)) for n in sizes]
    return [(r, max(1, n // r)) for n, r in zip(sizes, rows)]


def _shapes(case):
    return {"resnet20": _resnet20, "resnet50": _resnet50}[case["net"]]() if case["net"] != "drawn" else _drawn(case)


def _rows(gen, M, N, dtype, pad, scale=1.0):
    """M rows of N normal values of `dtype`, each row `pad` elements behind the end of the one before it."""
    t = torch.randn(M, N + pad, generator=gen, device="cuda").mul_(scale).to(DTYPES[dtype])
    return t[:, :N]


def _to_f8(x, floor):
    """Blocks (rows of x) as values of the 8-bit type and one scale each; with floor, no positive value becomes zero."""
    scale = x.abs().amax(dim=1, keepdim=True) * (1.0 / TOP)
    some = scale >= 2.0 ** -126
    scale = torch.where(some, scale, torch.zeros_like(scale))
    q = x * torch.where(some, torch.reciprocal(scale), torch.zeros_like(scale))
    if floor:
        q = torch.where(x > 0, torch.clamp(q, min=TINY), q)
    return q.to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["kind"] in ("linear", "grads"):
        M, N, K, dtype, pad = (case[k] for k in ("M", "N", "K", "dtype", "pad"))
        out = DTYPES[case["out"]]
        s["x"] = _rows(gen, M, K, dtype, pad)
        s["w"] = _rows(gen, N, K, dtype, pad, math.sqrt(2.0 / K))
        if case["kind"] == "linear":
            s["bias"] = torch.randn(N, generator=gen, device="cuda") * 0.1
            s["r"] = _rows(gen, M, N, dtype, pad) if case["res"] != "none" else None
            s["y"] = torch.empty(M, N, device="cuda", dtype=out)
            s["pre"] = torch.empty(M, N, device="cuda", dtype=DTYPES[dtype]) if case["keep_pre"] else None
        else:
            s["dy"] = _rows(gen, M, N, dtype, pad, 1.0 / M)
            s["pre"] = _rows(gen, M, N, dtype, pad) if case["act"] != "none" else None
            s["dx"] = torch.empty(M, K, device="cuda", dtype=DTYPES[dtype])
            s["dw"] = torch.empty(N, K, device="cuda", dtype=out)
            s["db"] = torch.empty(N, device="cuda", dtype=out)
    elif case["kind"] == "loss":
        rows, classes = case["rows"], case["classes"]
        s["logits"] = _rows(gen, rows, classes, case["dtype"], case["pad"], 3.0)
        lab = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
        drop = torch.rand(rows, generator=gen, device="cuda") < case["ignored"]
        s["target"] = torch.where(drop, torch.full_like(lab, -100), lab).to(torch.int32 if case["labels"] == "i32" else torch.int64)
        s["loss"] = torch.empty(rows, device="cuda")
        s["dlogits"] = torch.empty(rows, classes, device="cuda", dtype=DTYPES[case["dtype"]])
    else:
        shapes = _shapes(case)
        spans = [-(-r * c // BLOCK) * BLOCK for r, c in shapes]   # one flat buffer, every tensor from a block's start on
        n, starts = sum(spans), [0]
        for v in spans:
            starts.append(starts[-1] + v)
        keep, row0 = [], 0
        inside = torch.zeros(n, dtype=torch.bool, device="cuda")
        s["row_of"] = torch.zeros(n if case["pruned"] else 0, dtype=torch.int64, device="cuda")
        for (r, c), at in zip(shapes, starts):
            inside[at:at + r * c] = True
            if case["pruned"]:
                s["row_of"][at:at + r * c] = torch.arange(row0, row0 + r, device="cuda").repeat_interleave(c)
                keep.append(torch.rand(r, generator=gen, device="cuda") >= (case["pruned"] if r > 1 else 0.0))
                row0 += r
        s["keep"] = torch.cat(keep).to(torch.uint8) if keep else None
        s["shapes"], s["starts"] = shapes, starts[:-1]
        # gradients of many sizes: a common one for each block, another for each element
        size = torch.exp(torch.randn(n // BLOCK, 1, generator=gen, device="cuda") - 7.0)
        def normal():
            return torch.randn(n // BLOCK, BLOCK, generator=gen, device="cuda")
        def only(t, dtype):
            return torch.where(inside, t.reshape(-1), torch.zeros((), device="cuda")).to(dtype)
        s["p"] = only(normal() * 0.05, DTYPES[case["dtype"]])
        s["g"] = only(normal() * size, DTYPES[case["grad"]])
        m, r = only(normal() * size * 0.3, torch.float32), only(torch.exp(normal() * 0.7) * size, torch.float32)
        del inside, size
        if case["state"] == "f8":
            (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = (_to_f8(t.view(-1, BLOCK), f) for t, f in ((m, False), (r, True)))
        else:
            s["m"], s["v"] = m, r * r
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def _act(name, z):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * INV_SQRT_2))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(SQRT_2_PI * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * INV_SQRT_2)) + z * torch.exp(-0.5 * z * z) * INV_SQRT_2PI
    if name == "gelu_tanh":
        t = torch.tanh(SQRT_2_PI * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * SQRT_2_PI * (1.0 + 3 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _plain_linear(s):
    z = s["x"].float() @ s["w"].float().t() + s["bias"]
    if s["res"] == "before":
        z = z + s["r"].float()
    y = _act(s["act"], z)
    if s["res"] == "after":
        y = y + s["r"].float()
    return {"y": y.to(s["y"].dtype), "pre": z.to(s["pre"].dtype) if s["keep_pre"] else None}


def _plain_grads(s):
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_grad(s["act"], s["pre"].float())
    return {"dx": (dz @ s["w"].float()).to(s["dx"].dtype), "dw": (dz.t() @ s["x"].float()).to(s["dw"].dtype),
            "db": dz.sum(dim=0).to(s["db"].dtype)}


def _plain_loss(s):
    x, C, eps = s["logits"].float(), s["classes"], s["smoothing"]
    x = x - x.amax(dim=1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(dim=1, keepdim=True)
    there = s["target"] != -100
    at = torch.where(there, s["target"], torch.zeros_like(s["target"])).to(torch.int64)[:, None]
    log_total = torch.log(total[:, 0])
    loss = log_total - (1.0 - eps) * x.gather(1, at)[:, 0] - (eps / C * x.sum(dim=1) if eps else 0.0)
    grad = e / total - eps / C
    grad.scatter_add_(1, at, torch.full_like(at, -(1.0 - eps), dtype=torch.float32))
    grad = torch.where(there[:, None], grad * (1.0 / s["rows"]), torch.zeros_like(grad))
    return {"loss": torch.where(there, loss, torch.zeros_like(loss)), "dlogits": grad.to(s["dlogits"].dtype)}


def _plain_adamw(s):
    h, f8 = HYPER, s["state"] == "f8"
    g = s["g"].float()
    if f8:
        m, r = ((s[k].float() * s[k + "_scale"]).reshape(-1) for k in ("m", "v"))
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * h["beta1"] + g * (1.0 - h["beta1"])
    v = v * h["beta2"] + g * (1.0 - h["beta2"]) * g
    r = torch.sqrt(v)
    c1, c2 = 1.0 - h["beta1"] ** h["step"], 1.0 - h["beta2"] ** h["step"]
    p = s["p"].float() * (1.0 - h["lr"] * h["weight_decay"]) - (m / (r * (1.0 / math.sqrt(c2)) + h["eps"])) * (h["lr"] / c1)
    if s["keep"] is not None:
        keep = s["keep"][s["row_of"]].bool()
        p, m, v, r = (torch.where(keep, t, torch.zeros((), device="cuda")) for t in (p, m, v, r))
    s["p"].copy_(p)
    if f8:
        (m8, ms), (v8, vs) = (_to_f8(t.view(-1, BLOCK), f) for t, f in ((m, False), (r, True)))
        s["m"].copy_(m8), s["m_scale"].copy_(ms), s["v"].copy_(v8), s["v_scale"].copy_(vs)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    return _states(s)


def _states(s):
    return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale") if k in s}


def _own_linear(fp, s):
    if "work" not in s:      # the workspace that a program keeps for the layer
        s["work"] = torch.empty(fp.fp_linear_workspace(s["x"], s["w"], s["y"]), dtype=torch.uint8, device="cuda")
    fp.fp_linear_forward(s["x"], s["w"], s["y"], bias=s["bias"], res=s["r"], pre=s["pre"], act=ACTS[s["act"]],
                         res_first=s["res"] == "before", work=s["work"], stream=torch.cuda.current_stream())
    return {"y": s["y"], "pre": s["pre"]}


def _own_grads(fp, s):
    if "work" not in s:
        s["work"] = torch.empty(fp.fp_linear_backward_workspace(s["dy"], s["x"], s["w"], dx=s["dx"], dw=s["dw"], db=s["db"],
                                                                pre=s["pre"], act=ACTS[s["act"]]), dtype=torch.uint8, device="cuda")
    fp.fp_linear_backward(s["dy"], s["x"], s["w"], dx=s["dx"], dw=s["dw"], db=s["db"], pre=s["pre"], act=ACTS[s["act"]],
                          work=s["work"], stream=torch.cuda.current_stream())
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_loss(fp, s):
    fp.fp_cross_entropy(s["logits"], s["target"], s["loss"], dlogits=s["dlogits"], label_smoothing=s["smoothing"],
                        ignore_index=-100, grad_scale=1.0 / s["rows"], stream=torch.cuda.current_stream())
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def _own_adamw(fp, s):
    if "table" not in s:     # the table of tensors that a program makes once for its network
        rows = [0]
        for r, _ in s["shapes"]:
            rows.append(rows[-1] + r)
        f8 = s["state"] == "f8"
        s["table"] = fp.fp_adamw_tensors([
            dict({k: s[k].view(-1)[at:at + r * c] for k in ("p", "g", "m", "v")},
                 **({k: s[k].view(-1)[at // BLOCK:(at + r * c + BLOCK - 1) // BLOCK] for k in ("m_scale", "v_scale")} if f8 else {}),
                 **({"mask": s["keep"][q:q + r]} if s["keep"] is not None else {}))
            for (r, c), at, q in zip(s["shapes"], s["starts"], rows)])
    fp.fp_adamw_step(s["table"], stream=torch.cuda.current_stream(), **HYPER)
    return _states(s)


def run(s):
    if own:
        from paper_2010_16165_b200 import binding as fp
        return {"linear": _own_linear, "grads": _own_grads, "loss": _own_loss, "adamw": _own_adamw}[s["kind"]](fp, s)
    return {"linear": _plain_linear, "grads": _plain_grads, "loss": _plain_loss, "adamw": _plain_adamw}[s["kind"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["kind"] in ("linear", "grads"):
        M, N, K, b, o = case["M"], case["N"], case["K"], size[case["dtype"]], size[case["out"]]
        if case["kind"] == "linear":
            return {"bytes": b * (M * K + N * K) + 4 * N + o * M * N + b * M * N * ((case["res"] != "none") + case["keep_pre"]),
                    "flops": 2.0 * M * N * K}
        return {"bytes": b * (M * N * (1 + (case["act"] != "none")) + 2 * M * K + N * K) + o * (N * K + N), "flops": 4.0 * M * N * K}
    if case["kind"] == "loss":
        n = case["rows"] * case["classes"]
        return {"bytes": 2 * size[case["dtype"]] * n + case["rows"] * (4 + (4 if case["labels"] == "i32" else 8)), "flops": 8.0 * n}
    shapes = _shapes(case)
    n, rows = sum(r * c for r, c in shapes), sum(r for r, _ in shapes)
    blocks = sum(-(-r * c // BLOCK) for r, c in shapes)
    states = 16 * n if case["state"] == "f32" else 4 * n + 16 * blocks
    return {"bytes": (2 * size[case["dtype"]] + size[case["grad"]]) * n + states + (rows if case["pruned"] else 0), "flops": 16.0 * n}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("linear", "grads"):
        x, w, act = s["x"].double(), s["w"].double(), case["act"]
        if case["kind"] == "linear":
            z = torch.einsum("mk,nk->mn", x, w).add_(s["bias"].double()[None, :])
            if case["res"] == "before":
                z += s["r"].double()
            y = {"none": lambda: z, "relu": lambda: z * (z > 0), "gelu": lambda: z * torch.special.ndtr(z),
                 "gelu_tanh": lambda: z * torch.sigmoid(2.0 * SQRT_2_PI * (z + 0.044715 * z ** 3)),
                 "silu": lambda: z * torch.sigmoid(z)}[act]()
            if case["res"] == "after":
                y = y + s["r"].double()
            return {"y": y, "pre": z if case["keep_pre"] else None}
        dz = s["dy"].double()
        if act != "none":
            z = s["pre"].double().requires_grad_()
            y = {"relu": lambda: z * (z > 0), "gelu": lambda: z * torch.special.ndtr(z),
                 "gelu_tanh": lambda: z * torch.sigmoid(2.0 * SQRT_2_PI * (z + 0.044715 * z ** 3)), "silu": lambda: z * torch.sigmoid(z)}[act]()
            dz, = torch.autograd.grad(y, z, dz)
        return {"dx": torch.einsum("mn,nk->mk", dz, w), "dw": torch.einsum("mn,mk->nk", dz, x), "db": torch.einsum("mn->n", dz)}
    if case["kind"] == "loss":
        loss, grad, C, eps = [], [], case["classes"], case["smoothing"]
        for at in range(0, case["rows"], 1024):
            logp = torch.log_softmax(s["logits"][at:at + 1024].double(), dim=1)
            lab = s["target"][at:at + 1024].long()
            there = (lab >= 0).double()
            q = torch.full_like(logp, eps / C)
            q[torch.arange(len(lab), device="cuda"), lab.clamp(min=0)] += 1.0 - eps
            loss.append(-(q * logp).sum(dim=1) * there)
            grad.append((logp.exp() - q) * there[:, None] / case["rows"])
        return {"loss": torch.cat(loss), "dlogits": torch.cat(grad)}
    h = HYPER
    c1, c2 = 1.0 - h["beta1"] ** h["step"], 1.0 - h["beta2"] ** h["step"]
    f8, n, got = case["state"] == "f8", s["p"].numel(), {}
    step = 1 << 24                   # a multiple of the block: the pieces are independent of each other
    for at in range(0, n, step):
        part = slice(at, min(n, at + step))
        blocks = slice(part.start // BLOCK, part.stop // BLOCK)
        p, g = s["p"][part].double(), s["g"][part].double()
        if f8:
            m = (s["m"][blocks].double() * s["m_scale"][blocks].double()).reshape(-1)
            v = (s["v"][blocks].double() * s["v_scale"][blocks].double()).square().reshape(-1)
        else:
            m, v = s["m"][part].double(), s["v"][part].double()
        m = h["beta1"] * m + (1.0 - h["beta1"]) * g
        v = h["beta2"] * v + (1.0 - h["beta2"]) * g.square()
        p = p - h["lr"] * (h["weight_decay"] * p + (m / c1) / ((v / c2).sqrt() + h["eps"]))
        if s["keep"] is not None:
            kept = s["keep"].double()[s["row_of"][part]]
            p, m, v = p * kept, m * kept, v * kept
        out = {"p": p, "m": m, "v": v}
        if f8:
            for k, t in (("m", m.view(-1, BLOCK)), ("v", v.sqrt().view(-1, BLOCK))):
                scale = t.abs().amax(dim=1, keepdim=True) / TOP
                code = t / torch.where(scale > 0, scale, torch.ones_like(scale))
                if k == "v":
                    code = torch.where(t > 0, code.clamp(min=TINY), code)
                e = torch.floor(torch.log2(code.abs().clamp(min=2.0 ** -6)))   # three bits behind the leading one
                out[k], out[k + "_scale"] = (torch.round(code * 2.0 ** (3 - e)) * 2.0 ** (e - 3)).float(), scale
        for k, t in out.items():
            got.setdefault(k, []).append(t)
    return {k: torch.cat(t) for k, t in got.items()}
