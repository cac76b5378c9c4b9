"""Performance cases of a training step's other operators: root-mean-square norm with the residual's addition, the cross
entropy of a linear layer over many classes, and the orthogonalised update of a weight, as a program that trains or
serves a model of node features has them.

A case is a dict of plain values.  "op" is rms, ce or orth; "train" says whether a pass is forward and backward
(outputs and all gradients) or forward only; "dtype" is that of activations and parameters.

  rms    rows x C; "residual": x is added to it first and the sum is an output, too; "eight": the normalised rows leave
         in e4m3 with a scale each (serving only)
  ce     rows x d times d x V, the cross entropy against a target class per row; "labelled" is the share of rows that have
         one (the others: -1), "bias" whether the layer has one, "reduction" mean or none
  orth   B matrices of r x c: five Newton-Schulz steps towards the nearest matrix with orthonormal rows or columns

Where `own` is false the operators are computed in their plain form: elementary torch operations in 32
bits, rounded once at the end.
"""
import math

import torch

own = False

EPS = 1e-6
STEPS = 5
COEFFICIENTS = (3.4445, -4.775, 2.0315)


def listed():
    return [
        # serving one token: a row between two layers of a wide model, its result for a product in 8 bits; latency counts
        dict(name="rms_row_4096_e4m3", op="rms", rows=1, C=4096, residual=True, eight=True, dtype="bfloat16", train=False),
        # every node normalised between two layers of a training step
        dict(name="rms_nodes_262144_c128", op="rms", rows=262144, C=128, residual=True, eight=False, dtype="float32", train=True),
        # a training step of a wide model
        dict(name="rms_tokens_8192_c4096", op="rms", rows=8192, C=4096, residual=True, eight=False, dtype="bfloat16", train=True),
        # raw input features: a number of channels that is no multiple of 4, no residual
        dict(name="rms_input_30011_c602", op="rms", rows=30011, C=602, residual=False, eight=False, dtype="float32", train=True),
        # a mini-batch of node classification: latency counts
        dict(name="ce_61_64_v41", op="ce", rows=61, d=64, V=41, labelled=1.0, bias=True, reduction="mean", dtype="float32",
             train=True),
        # node classification on a whole graph, half of its nodes labelled
        dict(name="ce_262144_128_v41", op="ce", rows=262144, d=128, V=41, labelled=0.5, bias=True, reduction="mean",
             dtype="float32", train=True),
        # odd sizes throughout: entities of a catalogue as classes
        dict(name="ce_1531_602_v9973", op="ce", rows=1531, d=602, V=9973, labelled=1.0, bias=False, reduction="none",
             dtype="float32", train=True),
        # tokens of a vocabulary
        dict(name="ce_4096_2048_v65536", op="ce", rows=4096, d=2048, V=65536, labelled=1.0, bias=False, reduction="mean",
             dtype="bfloat16", train=True),
        # the weight of a narrow layer; latency counts
        dict(name="orth_64_256", op="orth", B=1, r=64, c=256, dtype="float32"),
        # a tall weight with odd sizes: raw input features to hidden ones
        dict(name="orth_1187_602", op="orth", B=1, r=1187, c=602, dtype="float32"),
        # the like weights of 12 blocks together
        dict(name="orth_12_256_1024", op="orth", B=12, r=256, c=1024, dtype="bfloat16"),
        # a weight of a wide model's feed-forward block
        dict(name="orth_2048_8192", op="orth", B=1, r=2048, c=8192, dtype="bfloat16"),
    ]


# ------------------------------------------------------------------------------------------------
# drawn cases
# ------------------------------------------------------------------------------------------------
MAX_ELEMENTS = 6.0e7          # of a norm's input
MAX_LOGITS = 2.7e8
MAX_CE_FLOPS = {"float32": 1.0e12, "bfloat16": 3.3e12}
MAX_ORTH_FLOPS = {"float32": 3.0e11, "bfloat16": 7.0e11}


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_rms(rng):
    eight = rng.random() < 0.3
    C = round(_log(rng, 16, 16384))
    if rng.random() < 0.7:                                   # most widths are whole pieces of 8
        C = max(16, C // 8 * 8)
    rows = max(1, min(1000000, round(_log(rng, C, MAX_ELEMENTS / (4 if eight else 1)) / C)))
    return dict(op="rms", rows=rows, C=C, residual=rng.random() < 0.7, eight=eight, dtype=rng.choice(["float32", "bfloat16"]),
                train=not eight and rng.random() < 0.7)


def _draw_ce(rng):
    dtype = rng.choice(["float32", "bfloat16"])
    train = rng.random() < 0.7
    while True:
        rows, d, V = round(_log(rng, 1, 300000)), round(_log(rng, 16, 4096)), round(_log(rng, 4, 150000))
        if rng.random() < 0.6:
            d = max(16, d // 8 * 8)
        if (6.0 if train else 2.0) * rows * d * V <= MAX_CE_FLOPS[dtype] and rows * V <= MAX_LOGITS and rows * d <= 1e8:
            return dict(op="ce", rows=rows, d=d, V=V, labelled=rng.choice([1.0, 1.0, 0.5, 0.1]) if rows >= 64 else 1.0,
                        bias=rng.random() < 0.4, reduction=rng.choice(["mean", "none"]), dtype=dtype, train=train)


def _draw_orth(rng):
    dtype = rng.choice(["float32", "bfloat16"])
    while True:
        r, c = round(_log(rng, 16, 4096)), round(_log(rng, 16, 8192))
        if rng.random() < 0.6:
            r, c = max(16, r // 8 * 8), max(16, c // 8 * 8)
        B = rng.choice([1, 1, 1, round(_log(rng, 2, 48))])
        case = dict(op="orth", B=B, r=r, c=c, dtype=dtype)
        if max(r, c) <= 8 * min(r, c) and work(case)["flops"] <= MAX_ORTH_FLOPS[dtype] and B * r * c <= 4e7:
            return case


def draw(rng):
    """One more case of the same ranges."""
    return rng.choice([_draw_rms, _draw_ce, _draw_orth])(rng)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _type(case):
    return getattr(torch, case["dtype"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _type(case)

    def normal(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).to(dt)

    st = dict(case)
    leaves = ()
    if case["op"] == "rms":
        rows, C = case["rows"], case["C"]
        st["x"] = normal(rows, C)
        st["residual"] = normal(rows, C, scale=2.0) if case["residual"] else None     # a sum of many layers' results
        st["w"] = normal(C, scale=0.2, shift=1.0)
        if case["train"]:
            st["dy"] = normal(rows, C)
            st["dsum"] = normal(rows, C) if case["residual"] else None
        leaves = ("x", "residual", "w") if case["residual"] else ("x", "w")
    elif case["op"] == "ce":
        T, d, V = case["rows"], case["d"], case["V"]
        st["x"] = normal(T, d)
        st["w"] = normal(d, V, scale=2.0 * d ** -0.5)        # logits of two units, as after some training
        st["bias"] = normal(V, scale=0.3) if case["bias"] else None
        target = torch.randint(0, V, (T,), generator=g, device="cuda")
        without = torch.rand(T, generator=g, device="cuda") >= case["labelled"]
        st["target"] = torch.where(without, -1, target)
        st["dloss"] = torch.rand(T, generator=g, device="cuda") / T if case["reduction"] == "none" else None
        leaves = ("x", "w", "bias") if case["bias"] else ("x", "w")
    else:
        B, r, c = case["B"], case["r"], case["c"]
        # a momentum of gradients: a few strong directions and noise
        k = max(2, min(r, c) // 8)
        strong = torch.randn(B, r, k, generator=g, device="cuda") @ torch.randn(B, k, c, generator=g, device="cuda")
        st["update"] = (1e-3 * (strong / math.sqrt(k) + 0.3 * torch.randn(B, r, c, generator=g, device="cuda"))).to(dt)
        if B == 1:
            st["update"] = st["update"][0]
    if case.get("train"):
        for name in leaves:
            st[name] = st[name].detach().requires_grad_(True)
    return st


# ------------------------------------------------------------------------------------------------
# the plain form
# ------------------------------------------------------------------------------------------------
def _rms_plain(st):
    dt = st["x"].dtype
    x, w = st["x"].float(), st["w"].float()
    out = {}
    if st["residual"] is not None:
        # what is normalised is the sum as the next layers get it
        out["sum"] = (x + st["residual"].float()).to(dt)
        x = out["sum"].float()
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    xh = x * r
    y = xh * w
    if st["eight"]:
        scale = y.abs().amax(1) / 448.0
        out["scale"] = scale
        out["q"] = (y / torch.where(scale > 0, scale, 1.0)[:, None]).to(torch.float8_e4m3fn)
        return out
    out["y"] = y.to(dt)
    if not st["train"]:
        return out
    dy = st["dy"].float()
    e = dy * w
    dx = r * (e - xh * (e * xh).mean(1, keepdim=True))
    if st["residual"] is not None:
        dx = dx + st["dsum"].float()
        out["dresidual"] = dx.to(dt)
    out["dx"] = dx.to(dt)
    out["dw"] = (dy * xh).sum(0).to(dt)
    return out


def _ce_plain(st):
    dt = st["x"].dtype
    x, w, target = st["x"].float(), st["w"].float(), st["target"]
    valid = target >= 0
    at = target.clamp(min=0)[:, None]
    z = x @ w
    if st["bias"] is not None:
        z += st["bias"].float()
    largest = z.amax(1, keepdim=True)
    zt = z.gather(1, at)
    q = z.sub_(largest).exp_()
    total = q.sum(1, keepdim=True)
    loss = torch.where(valid, (torch.log(total) + largest - zt)[:, 0], 0.0)
    count = valid.sum().clamp(min=1).float()
    mean = st["reduction"] == "mean"
    out = dict(loss=(loss.double().sum() / count).float() if mean else loss)
    if not st["train"]:
        return out
    dloss = torch.where(valid, 1.0 / count if mean else st["dloss"], 0.0)[:, None]
    q.mul_(dloss / total)
    q.scatter_add_(1, at, -dloss)
    out.update(dx=(q @ w.t()).to(dt), dw=(x.t() @ q).to(dt))
    if st["bias"] is not None:
        out["dbias"] = q.sum(0).to(dt)
    return out


def _orth_plain(st):
    a, b, c = COEFFICIENTS
    G = st["update"].float()
    tall = G.shape[-2] > G.shape[-1]
    X = G.transpose(-2, -1).contiguous() if tall else G
    X = X / (G.double().pow(2).sum((-2, -1), keepdim=True).sqrt() + 1e-7).float()
    for _ in range(STEPS):
        A = X @ X.transpose(-2, -1).contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return (X.transpose(-2, -1) if tall else X).to(st["update"].dtype).contiguous()


# ------------------------------------------------------------------------------------------------
# a pass
# ------------------------------------------------------------------------------------------------
def run(st):
    if not own:
        with torch.no_grad():
            return dict(rms=_rms_plain, ce=_ce_plain, orth=_orth_plain)[st["op"]](st)
    from paper_2202_08556_amd import layers, optim
    if st["op"] == "rms":
        x, w, residual = st["x"], st["w"], st["residual"]
        if st["eight"]:
            got = layers.rms_norm_e4m3(x, w, residual=residual, eps=EPS)
            return dict(zip(("q", "scale") if residual is None else ("q", "scale", "sum"), got))
        if residual is None:
            y = layers.rms_norm(x, w, eps=EPS)
            if not st["train"]:
                return dict(y=y)
            dx, dw = torch.autograd.grad(y, (x, w), st["dy"])
            return dict(y=y, dx=dx, dw=dw)
        y, s = layers.rms_norm(x, w, residual=residual, eps=EPS)
        if not st["train"]:
            return dict(y=y, sum=s)
        dx, dresidual, dw = torch.autograd.grad((y, s), (x, residual, w), (st["dy"], st["dsum"]))
        return dict(y=y, sum=s, dx=dx, dresidual=dresidual, dw=dw)
    if st["op"] == "ce":
        loss = layers.linear_cross_entropy(st["x"], st["w"], st["target"], bias=st["bias"], reduction=st["reduction"])
        if not st["train"]:
            return dict(loss=loss)
        if st["bias"] is None:
            dx, dw = torch.autograd.grad(loss, (st["x"], st["w"]), st["dloss"])
            return dict(loss=loss, dx=dx, dw=dw)
        dx, dw, dbias = torch.autograd.grad(loss, (st["x"], st["w"], st["bias"]), st["dloss"])
        return dict(loss=loss, dx=dx, dw=dw, dbias=dbias)
    return optim.orthogonalise(st["update"], steps=STEPS, coefficients=COEFFICIENTS)


def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "rms":
        n, res = case["rows"] * case["C"], bool(case["residual"])
        moved = n * size * (1 + 2 * res) + (n + 4 * case["rows"] if case["eight"] else n * size)
        if case["train"]:
            moved += n * size * (3 + res)                    # dy, the sum (or x) again, dsum; dx, which is dresidual, too
        return dict(bytes=moved + size * case["C"] * (2 if case["train"] else 1), flops=n * (16 if case["train"] else 6))
    if case["op"] == "ce":
        T, d, V = case["rows"] * case["labelled"], case["d"], case["V"]
        return dict(bytes=size * (T * d + d * V) * (2 if case["train"] else 1) + 12 * case["rows"],
                    flops=(6 if case["train"] else 2) * T * d * V)
    m, n = min(case["r"], case["c"]), max(case["r"], case["c"])
    # half of the symmetric products
    return dict(bytes=2 * size * case["B"] * m * n, flops=float(STEPS) * case["B"] * (3 * m * m * n + m * m * m))


# ------------------------------------------------------------------------------------------------
# 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The definitions in 64 bits, gradients by differentiation."""
    F = torch.nn.functional
    st = prepare(case, seed)
    dt = torch.float64
    train = case.get("train", False)

    def leaf(t):
        return t if t is None else t.detach().to(dt).requires_grad_(train)

    if case["op"] == "rms":
        x, w, residual = leaf(st["x"]), leaf(st["w"]), leaf(st["residual"])
        out = {}
        s = x
        if residual is not None:
            s = x + residual
            out["sum"] = s.detach()
            # the sum leaves in the type of x, and that is what is normalised
            s = s + (s.detach().to(st["x"].dtype).to(dt) - s.detach())
        y = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + EPS) * w
        if case["eight"]:
            scale = y.abs().amax(-1) / 448
            return dict(out, scale=scale, q=y / scale[:, None])
        out["y"] = y.detach()
        if not train:
            return out
        outs, grads = ((y,), (st["dy"].to(dt),)) if residual is None else ((y, s), (st["dy"].to(dt), st["dsum"].to(dt)))
        got = torch.autograd.grad(outs, (x, w) if residual is None else (x, w, residual), grads)
        return dict(out, **dict(zip(("dx", "dw", "dresidual"), got)))
    if case["op"] == "ce":
        x, w, bias = leaf(st["x"]), leaf(st["w"]), leaf(st["bias"])
        has = st["target"].ge(0).nonzero()[:, 0]
        z = torch.mm(x[has], w)
        if bias is not None:
            z = z + bias
        rows = -z.log_softmax(1).gather(1, st["target"][has, None])[:, 0]
        loss = torch.zeros(case["rows"], dtype=dt, device="cuda").index_copy(0, has, rows)
        if case["reduction"] == "mean":
            loss = loss.sum() / max(1, has.numel())
        if not train:
            return dict(loss=loss)
        names = ("dx", "dw") if bias is None else ("dx", "dw", "dbias")
        got = torch.autograd.grad(loss, (x, w) if bias is None else (x, w, bias),
                                  None if st["dloss"] is None else st["dloss"].to(dt))
        return dict(loss=loss.detach(), **dict(zip(names, got)))
    a, b, c = COEFFICIENTS
    X = st["update"].to(dt)
    flip = X.shape[-2] > X.shape[-1]
    if flip:
        X = X.mT.contiguous()
    X = X / (torch.linalg.vector_norm(X, dim=(-2, -1), keepdim=True) + 1e-7)
    # by the Gram matrix: X (a + b G + c G^2), G = X^T X on the smaller side
    for _ in range(STEPS):
        G = torch.matmul(X, X.mT.contiguous())
        P = torch.addmm(b * G, G, G, alpha=c) if G.dim() == 2 else torch.baddbmm(b * G, G, G, alpha=c)
        P = P + a * torch.eye(G.shape[-1], dtype=dt, device="cuda")
        X = torch.matmul(P, X)
    return X.mT.contiguous() if flip else X
