"""The ends of a language model and its matrix update, by which the speed of
the operators beside the aggregation step is measured:

  embed      scaled rows of a table for a list of tokens
  embed_grad the table's gradient: every row's sum over its tokens
  xent       softmax cross entropy over a vocabulary, from the last layer's
             outputs and the vocabulary's rows
  xent_grad  the same with both gradients
  orth       updates made orthogonal by Newton-Schulz products, for one matrix,
             a stack of equal ones or every layer of one of the networks in
             `workloads/tables.py`

Their plain form is elementary torch operations in 32 bits.  A token or target
below zero is padding: a row of zeros, no loss, no gradient.
"""
import math

import torch

from workloads import tables

own = False  # True: the calls a user makes of the framework's operators

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
NS = (3.4445, -4.7750, 2.0315)  # X <- a X + (b A + c A^2) X, A = X X^T
STEPS = 5
NETS = ("nin", "googlenet", "alexnet")
PAD = 0.02  # share of tokens and targets that are padding


def listed():
    return [
        # one token of a conversation: latency only
        {"name": "embed_one", "op": "embed", "tokens": 1, "rows": 65536, "dim": 2048, "dtype": "f16", "out": "f16"},
        # a training batch's tokens, widened for a network in 32 bits; odd sizes
        {"name": "embed_odd", "op": "embed", "tokens": 5001, "rows": 50001, "dim": 1001, "dtype": "bf16", "out": "f32"},
        # one worker's share of a large batch
        {"name": "embed_batch", "op": "embed", "tokens": 32768, "rows": 131072, "dim": 2048, "dtype": "f16",
         "out": "f16"},
        # a table of classes with a small batch: the framework's 1000 outputs
        {"name": "embed_grad_classes", "op": "embed_grad", "tokens": 256, "rows": 1000, "dim": 1001, "dtype": "f32",
         "out": "f32"},
        # one worker's gradient of a vocabulary's table, 16-bit activations into a 32-bit replica
        {"name": "embed_grad_batch", "op": "embed_grad", "tokens": 32768, "rows": 65536, "dim": 2048, "dtype": "f16",
         "out": "f32"},
        # scores of a few answers' tokens: the vocabulary is read once
        {"name": "xent_few", "op": "xent", "tokens": 24, "rows": 65536, "dim": 2048, "dtype": "bf16"},
        # a small model's step with odd sizes throughout
        {"name": "xent_grad_odd", "op": "xent_grad", "tokens": 1003, "rows": 50001, "dim": 520, "dtype": "bf16"},
        # one worker's share of a large batch over a large vocabulary
        {"name": "xent_grad_batch", "op": "xent_grad", "tokens": 8192, "rows": 131072, "dim": 2048, "dtype": "f16"},
        # the first layer of NiN, the smallest update there is: 96 filters of 363 weights
        {"name": "orth_conv1", "op": "orth", "net": "", "count": 1, "rows": 96, "cols": 363, "dtype": "f32",
         "out": "bf16"},
        # every layer of GoogLeNet: 58 matrices, hardly two alike
        {"name": "orth_googlenet", "op": "orth", "net": "googlenet", "count": 0, "rows": 0, "cols": 0, "dtype": "f32",
         "out": "bf16"},
        # AlexNet's seventh layer, kept in 32 bits throughout
        {"name": "orth_fc7_f32", "op": "orth", "net": "", "count": 1, "rows": 4096, "cols": 4096, "dtype": "f32",
         "out": "f32"},
        # every layer of AlexNet, 4096 x 9216 the largest
        {"name": "orth_alexnet", "op": "orth", "net": "alexnet", "count": 0, "rows": 0, "cols": 0, "dtype": "f32",
         "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "xent", "xent_grad", "orth", "orth"))
    most = max((work(c) for c in listed()), key=lambda w: w["flops"])["flops"]
    while True:
        if op == "orth":
            case = {"op": op, "net": rng.choice(("", "", "", "") + NETS), "count": _log(rng, 1, 32),
                    "rows": _log(rng, 16, 4096), "cols": _log(rng, 16, 8192), "dtype": rng.choice(tuple(DTYPES)),
                    "out": rng.choice(("bf16", "bf16", "f16", "f32"))}
            if case["net"]:
                case.update(count=0, rows=0, cols=0)
        else:
            case = {"op": op, "tokens": _log(rng, 1, 32768 if op.startswith("embed") else 8192),
                    "rows": _log(rng, 1000, 131072), "dim": _log(rng, 64, 4096),
                    "dtype": rng.choice(("f16", "bf16") if op.startswith("xent") else tuple(DTYPES))}
            if op == "embed":
                case["out"] = rng.choice((case["dtype"], case["dtype"], "f32"))
            if op == "embed_grad":
                case["out"] = rng.choice(("f32", "f32", "f16"))
            if rng.random() < 0.6:  # a model's width is mostly a multiple of 64, but not always
                case["dim"] = max(64, case["dim"] // 64 * 64)
        if work(case)["flops"] <= most:
            return case


def _shapes(case):
    """(rows, columns) of every matrix of an orth case."""
    if case["net"]:
        return [(layer.out_ch, layer.fan_in) for layer in tables.get(case["net"]).layers]
    return [(case["rows"], case["cols"])] * case["count"]


def _matrices(case):
    """(offset, rows, columns) of every matrix of an orth case in one vector,
    each on a multiple of 64 elements, and the vector's length."""
    got, at = [], 0
    for r, c in _shapes(case):
        got.append((at, r, c))
        at += -(-r * c // 64) * 64
    return got, at


def _tokens(n, rows, g, dev):
    """Tokens of which a few make up most of the text, some of them padding."""
    u = torch.rand(n, generator=g, device=dev)
    t = (rows ** u - 1).clamp_(0, rows - 1).long()  # density falling as 1 / (token + 1)
    return torch.where(torch.rand(n, generator=g, device=dev) < PAD, -1, t)


def _inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if case["op"] == "orth":
        mats, total = _matrices(case)
        grad = torch.zeros(total, device=dev)
        for at, r, c in mats:  # a few strong directions in noise
            k = min(16, r, c)
            m = normal(r, k) * (0.7 ** torch.arange(k, device=dev)) @ normal(k, c) + 0.2 * normal(r, c)
            grad[at:at + r * c] = 1e-3 * m.reshape(-1)
        return {"grad": grad.to(dtype)}
    n, rows, dim = case["tokens"], case["rows"], case["dim"]
    tokens = _tokens(n, rows, g, dev)
    if case["op"] == "embed":
        return {"tokens": tokens, "table": (0.02 * normal(rows, dim)).to(dtype)}
    if case["op"] == "embed_grad":
        return {"tokens": tokens, "dy": (1e-2 * normal(n, dim)).to(dtype)}
    # outputs that lean toward their target's row, as a model's in training do
    w = normal(rows, dim) * dim ** -0.5
    x = normal(n, dim) + 2.0 * w[tokens.clamp(min=0)]
    return {"tokens": tokens, "w": w.to(dtype), "x": x.to(dtype)}


def prepare(case, seed):
    s = dict(_inputs(case, seed), op=case["op"], case=case)
    dev = s["tokens" if "tokens" in s else "grad"].device
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "embed":
        s["scale"] = case["dim"] ** 0.5
        s["out"] = torch.zeros((case["tokens"], case["dim"]), dtype=DTYPES[case["out"]], device=dev)
    elif case["op"] == "embed_grad":
        s["scale"] = case["dim"] ** 0.5
        s["out"] = torch.zeros((case["rows"], case["dim"]), dtype=DTYPES[case["out"]], device=dev)
    elif case["op"] == "orth":
        s["mats"] = _matrices(case)[0]
        s["out"] = torch.zeros(s["grad"].numel(), dtype=DTYPES[case["out"]], device=dev)
    else:
        s["loss"] = torch.zeros(case["tokens"], device=dev)
        if case["op"] == "xent_grad":
            s["dx"] = torch.zeros((case["tokens"], case["dim"]), dtype=dtype, device=dev)
            s["dw"] = torch.zeros((case["rows"], case["dim"]), dtype=dtype, device=dev)
    if own:
        import paper_1511_00175_amd as fc
        if case["op"] in ("embed", "embed_grad"):
            s["plan"] = fc.Embedding(case["rows"], case["dim"], case["tokens"])
        elif case["op"] == "orth":
            s["plan"] = fc.Muon(s["mats"], dtype=case["out"], steps=STEPS)
        else:
            s["plan"] = fc.CrossEntropy(case["rows"], case["dim"], case["tokens"], case["dtype"])
    return s


def _plain_embed(s):
    keep = s["tokens"] >= 0
    rows = s["table"][s["tokens"].clamp(min=0)].float() * s["scale"]
    s["out"].copy_(torch.where(keep[:, None], rows, 0.0))
    return {"out": s["out"]}


def _plain_embed_grad(s):
    keep = s["tokens"] >= 0
    dy = torch.where(keep[:, None], s["dy"].float() * s["scale"], 0.0)
    total = torch.zeros(s["out"].shape, device=dy.device)
    total.index_add_(0, s["tokens"].clamp(min=0), dy)
    s["out"].copy_(total)
    return {"out": s["out"]}


def _plain_xent(s):
    keep, t = s["tokens"] >= 0, s["tokens"].clamp(min=0)
    x, w = s["x"].float(), s["w"].float()
    p = x @ w.t()
    at = torch.arange(len(t), device=t.device)
    target = p[at, t]
    top = p.amax(1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    loss = torch.log(total[:, 0]) + top[:, 0] - target
    s["loss"].copy_(torch.where(keep, loss, 0.0))
    if s["op"] == "xent":
        return {"loss": s["loss"]}
    p.div_(total)
    p[at, t] -= 1.0
    p.mul_(keep[:, None])
    s["dx"].copy_(p @ w)
    s["dw"].copy_(p.t() @ x)
    return {"loss": s["loss"], "dx": s["dx"], "dw": s["dw"]}


def _newton_schulz(x):
    """A stack of matrices (count, rows, columns), made orthogonal."""
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / x.square().sum((1, 2), keepdim=True).sqrt()
    a, b, c = NS
    for _ in range(STEPS):
        m = x @ x.transpose(1, 2)
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.transpose(1, 2) if tall else x


def _plain_orth(s):
    g, out = s["grad"].float(), s["out"]
    alike = {}  # matrices of one shape go through the products together
    for at, r, c in s["mats"]:
        alike.setdefault((r, c), []).append(at)
    for (r, c), places in alike.items():
        x = _newton_schulz(torch.stack([g[at:at + r * c].view(r, c) for at in places]))
        for at, m in zip(places, x):
            out[at:at + r * c] = m.reshape(-1)
    return {"out": out}


def _own(s):
    op, plan = s["op"], s["plan"]
    if op == "embed":
        plan.lookup(s["table"], s["tokens"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "embed_grad":
        plan.grad(s["dy"], s["tokens"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "xent":
        plan.loss(s["x"], s["w"], s["tokens"], s["loss"])
        return {"loss": s["loss"]}
    if op == "xent_grad":
        plan.loss_grad(s["x"], s["w"], s["tokens"], s["loss"], s["dx"], s["dw"])
        return {"loss": s["loss"], "dx": s["dx"], "dw": s["dw"]}
    plan.orthogonalize(s["grad"], s["out"])
    return {"out": s["out"]}


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "xent": _plain_xent, "xent_grad": _plain_xent,
            "orth": _plain_orth}[state["op"]](state)


def work(case):
    size = BYTES[case["dtype"]]
    if case["op"] == "orth":
        flops = bytes_ = 0
        for r, c in _shapes(case):
            s, l = min(r, c), max(r, c)
            # half of X X^T and of A A (both symmetric), all of B X
            flops += STEPS * (s * s * l + s * s * s + 2 * s * s * l)
            bytes_ += r * c * (size + BYTES[case["out"]])
        return {"bytes": bytes_, "flops": flops}
    n, rows, dim = case["tokens"], case["rows"], case["dim"]
    if case["op"] == "embed":
        return {"bytes": min(n, rows) * dim * size + n * dim * BYTES[case["out"]] + 8 * n, "flops": n * dim}
    if case["op"] == "embed_grad":
        return {"bytes": n * dim * size + rows * dim * BYTES[case["out"]] + 8 * n, "flops": n * dim}
    io, one = (n + rows) * dim * size, 2 * n * rows * dim
    if case["op"] == "xent":
        return {"bytes": io + 12 * n, "flops": one}
    return {"bytes": 2 * io + 12 * n, "flops": 3 * one}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    s = _inputs(case, seed)
    if case["op"] == "orth":
        grad = s["grad"].double()
        out = torch.zeros_like(grad)
        for at, r, c in _matrices(case)[0]:
            m = grad[at:at + r * c].view(r, c)
            m = m / torch.linalg.norm(m)
            side = m if r <= c else m.t()  # the products are over the longer axis
            eye = torch.eye(min(r, c), dtype=torch.float64, device=m.device)
            for _ in range(STEPS):
                gram = side @ side.t()
                side = (NS[0] * eye + gram @ (NS[1] * eye + NS[2] * gram)) @ side
            out[at:at + r * c] = (side if r <= c else side.t()).reshape(-1)
        return {"out": out}
    n, rows, dim = case["tokens"], case["rows"], case["dim"]
    real = torch.nonzero(s["tokens"] >= 0)[:, 0]
    tokens = s["tokens"][real]
    dev = tokens.device
    if case["op"] == "embed":
        out = torch.zeros((n, dim), dtype=torch.float64, device=dev)
        out[real] = s["table"].double()[tokens] * dim ** 0.5
        return {"out": out}
    if case["op"] == "embed_grad":
        out = torch.zeros((rows, dim), dtype=torch.float64, device=dev)
        out.scatter_add_(0, tokens[:, None].expand(-1, dim), s["dy"][real].double() * dim ** 0.5)
        return {"out": out}
    x, w = s["x"].double(), s["w"].double()
    loss = torch.zeros(n, dtype=torch.float64, device=dev)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for a in range(0, len(real), 1024):  # targets at a time
        i, t = real[a:a + 1024], tokens[a:a + 1024]
        logp = torch.log_softmax(x[i] @ w.t(), 1)
        loss[i] = -logp.gather(1, t[:, None])[:, 0]
        if case["op"] == "xent_grad":
            d = logp.exp_()
            d.scatter_add_(1, t[:, None], torch.full_like(d[:, :1], -1.0))
            dx[i] = d @ w
            dw += d.t() @ x[i]
    return {"loss": loss, "dx": dx, "dw": dw} if case["op"] == "xent_grad" else {"loss": loss}
