"""The operators at the two ends of a training step that the compressed step stands in, as a user's program calls them, and
their plain forms: the loss of a linear output layer over its classes (forward alone, and forward with every gradient) with no
logits kept, and the orthogonalisation of a model's matrices by Newton-Schulz products, before they are packed into a worker's row.

`own` chooses the side: plain torch operations in float32, or the package's own operators on the same state."""
import math
import random

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
IGNORE = -100
ALIGN = 128                         # elements: matrices start where an allocator would start them
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
MOST = 4096 * 65536 * 2048          # the largest listed loss: rows * classes * features


# ---- the workloads' matrices ---------------------------------------------------------------------------------------------

def _cifar(blocks):
    """The convolutions of ResNet-(6 blocks + 2) on 32x32 images as [out, in * 9]: 20 layers at blocks = 3, 56 at blocks = 9."""
    out, cin = [(16, 27)], 16
    for c in (16, 32, 64):
        for _ in range(blocks):
            out += [(c, cin * 9), (c, c * 9)]
            cin = c
    return out


def _encoder(layers, hidden):
    """The projections of a transformer encoder's layers; embeddings and vectors are not orthogonalised."""
    return ([(hidden, hidden)] * 4 + [(4 * hidden, hidden), (hidden, 4 * hidden)]) * layers


def _matrices(case):
    if case["model"] == "cifar":
        return _cifar(case["blocks"])
    if case["model"] == "encoder":
        return _encoder(case["layers"], case["hidden"])
    return [(case["m"], case["n"])] * case["count"]


# ---- cases ---------------------------------------------------------------------------------------------------------------

def listed():
    def loss(name, op, n, d, v, dtype, bias=False, ignored=0.0, reduction="mean", wide=0):
        return dict(name=name, op=op, n=n, d=d, v=v, dtype=dtype, bias=bias, ignored=ignored, reduction=reduction, wide=wide)

    def ortho(name, model, dtype, result, rows=1, **more):
        return dict(name=name, op="ortho", model=model, dtype=dtype, result=result, rows=rows, **more)
    return [
        # The classifier of the small model on one worker's batch, without mixed precision: latency counts.
        loss("loss 128x64x10 f32 bias", "loss", 128, 64, 10, "float32", bias=True),
        # The encoder's held-out loss of every position of 8 sequences.
        loss("loss 4096x768x30522 bf16", "loss", 4096, 768, 30522, "bfloat16", reduction="none"),
        # The ImageNet-sized model's classifier, one worker's batch of 32, float32: loss and gradients.
        loss("train 32x2048x1000 f32 bias", "train", 32, 2048, 1000, "float32", bias=True),
        # Odd in every size, a slice of a wider tensor, one position in ten of a padded batch has no target.
        loss("train 1021x515x5003 f16 slice", "train", 1021, 515, 5003, "float16", bias=True, ignored=0.1, wide=37),
        # Masked training of the encoder: 32 sequences of 512, 15 % of the positions have a target.
        loss("train 16384x768x30522 masked", "train", 16384, 768, 30522, "bfloat16", ignored=0.85),
        # The same head where every position has one.
        loss("train 8192x768x30522 bf16", "train", 8192, 768, 30522, "bfloat16"),
        # A wide model's head: the largest of these calls.
        loss("train 4096x2048x65536 bf16", "train", 4096, 2048, 65536, "bfloat16"),
        # One convolution's gradient: latency counts.
        ortho("ortho 64x576 f32", "one", "float32", "bfloat16", m=64, n=576, count=1),
        # Four workers' convolutions of ResNet-20 in full precision.
        ortho("ortho resnet20 x4 f32", "cifar", "float32", "float32", rows=4, blocks=3),
        # Every projection of the 12-layer encoder, one worker.
        ortho("ortho encoder bf16", "encoder", "bfloat16", "bfloat16", layers=12, hidden=768),
        # Odd sizes, taller than wide.
        ortho("ortho 3 x 1001x333 f16", "one", "float16", "float16", m=1001, n=333, count=3),
        # One matrix of a wide model.
        ortho("ortho 4096x4096 bf16", "one", "bfloat16", "bfloat16", m=4096, n=4096, count=1),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "train", "train", "ortho", "ortho"])
    if op != "ortho":
        while True:
            n, d, v = _between(rng, 1, 16384), _between(rng, 16, 4096), _between(rng, 10, 131072)
            if n * d * v <= MOST // 4 and n * v <= 1 << 29:
                break
        if rng.random() < 0.5:
            d = -(-d // 64) * 64
        return {"op": op, "n": n, "d": d, "v": v, "dtype": rng.choice(["float32", "bfloat16", "bfloat16", "float16"]),
                "bias": rng.random() < 0.4, "ignored": rng.choice([0.0, 0.0, 0.1, 0.85]),
                "reduction": rng.choice(["mean", "mean", "sum", "none"]), "wide": rng.choice([0, 0, 0, 8, 37])}
    case = {"op": op, "dtype": rng.choice(["float32", "bfloat16", "float16"])}
    case["result"] = rng.choice([case["dtype"], "bfloat16"])
    model = rng.choice(["cifar", "encoder", "one", "one"])
    if model == "cifar":
        return case | {"model": model, "blocks": rng.randint(1, 9), "rows": rng.randint(1, 8)}
    if model == "encoder":
        hidden = _between(rng, 48, 767)
        return case | {"model": model, "layers": rng.randint(1, 12), "hidden": hidden, "rows": rng.randint(1, 2)}
    while True:
        m, n, count = _between(rng, 4, 4096), _between(rng, 4, 4096), _between(rng, 1, 24)
        if min(m, n) ** 2 * max(m, n) * count <= 4096 ** 3 // 4:
            return case | {"model": model, "m": m, "n": n, "count": count, "rows": 1}


# ---- states --------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) & 0x7FFFFFFF)


def _prepare_loss(case, seed):
    gen = _gen(seed)
    n, d, v, dt = case["n"], case["d"], case["v"], DTYPES[case["dtype"]]
    # normalised hidden states against rows of about unit length: logits of a standard deviation of 1.5; `wide` more features
    # beside the ones that are read
    weight = (torch.randn((v, d), device="cuda", generator=gen) * (1.5 / math.sqrt(d))).to(dt)
    x = torch.randn((n, d + case["wide"]), device="cuda", generator=gen)[:, :d]
    # classes come with very different frequencies, and a trained model has an idea of the right one
    u = torch.rand(n, device="cuda", generator=gen)
    target = ((v + 1.0) ** u - 1).long().clamp(0, v - 1)
    x = (x + 2.0 * weight[target].float()).to(dt)
    if case["wide"]:
        x = torch.cat([x, x.new_zeros((n, case["wide"]))], 1)[:, :d]
    target[torch.rand(n, device="cuda", generator=gen) < case["ignored"]] = IGNORE
    target[0] = v // 2                  # a batch without any target has no mean
    state = {"case": case, "x": x, "weight": weight, "target": target, "bias": None}
    if case["bias"]:
        state["bias"] = (0.3 * torch.randn(v, device="cuda", generator=gen)).to(dt)
    if case["op"] == "train":
        state["dloss"] = torch.rand(n, device="cuda", generator=gen) + 0.5 if case["reduction"] == "none" else torch.ones((), device="cuda")
    return state


def _prepare_ortho(case, seed):
    gen, host, dt = _gen(seed), random.Random(seed), DTYPES[case["dtype"]]
    shapes = _matrices(case)

    def gradient(m, n):
        # a few directions that many examples share, over noise, at a layer's own scale
        r = min(4, m, n)
        low = torch.randn((m, r), device="cuda", generator=gen) @ torch.randn((r, n), device="cuda", generator=gen)
        return ((0.5 * low + torch.randn((m, n), device="cuda", generator=gen)) * 10.0 ** host.uniform(-4.0, -1.0)).to(dt)
    room = [-(-m * n // ALIGN) * ALIGN for m, n in shapes]
    # the results lie in one buffer a row, as a worker's matrices do that are packed next
    flat = torch.zeros((case["rows"], sum(room)), dtype=DTYPES[case["result"]], device="cuda")
    out = [[v[:m * n].view(m, n) for v, (m, n) in zip(row.split(room), shapes)] for row in flat]
    state = {"case": case, "rows": [[gradient(m, n) for m, n in shapes] for _ in range(case["rows"])], "flat": flat, "out": out}
    if own:
        # the plan of the parameter list (shapes, tables and workspace), made once for a model
        from paper_2008_05823_b200 import orthogonal
        state["plan"] = orthogonal.Orthogonalizer(shapes, dt, num_rows=case["rows"], coefficients=COEFFICIENTS, eps=EPS,
                                                  result_dtypes=DTYPES[case["result"]])
    return state


def prepare(case, seed):
    return _prepare_ortho(case, seed) if case["op"] == "ortho" else _prepare_loss(case, seed)


# ---- one pass ------------------------------------------------------------------------------------------------------------

def _reduced(case, rows, count):
    return rows if case["reduction"] == "none" else rows.sum() if case["reduction"] == "sum" else rows.sum() / count


def _plain_loss(state):
    case, target = state["case"], state["target"]
    x, weight = state["x"].float(), state["weight"].float()
    logits = x @ weight.t()
    if case["bias"]:
        logits += state["bias"].float()
    valid = target != IGNORE
    at = torch.where(valid, target, 0)[:, None]
    top = logits.amax(1, keepdim=True)
    picked = logits.gather(1, at) - top
    e = torch.exp(logits.sub_(top), out=logits)
    total = e.sum(1, keepdim=True)
    rows = torch.where(valid, (torch.log(total) - picked)[:, 0], 0.0)
    count = valid.sum()
    out = {"loss": _reduced(case, rows, count)}
    if case["op"] == "loss":
        return out
    p = e.div_(total)
    p.scatter_add_(1, at, p.new_full((), -1.0).expand_as(at))
    g = state["dloss"] / count if case["reduction"] == "mean" else state["dloss"]
    p.mul_(torch.where(valid, g, 0.0)[:, None])
    out["dx"] = (p @ weight).to(state["x"].dtype)
    out["dweight"] = (p.t() @ x).to(state["weight"].dtype)
    if case["bias"]:
        out["dbias"] = p.sum(0).to(state["bias"].dtype)
    return out


def _own_loss(state):
    from paper_2008_05823_b200 import cross_entropy as ce
    case, x, weight, target, bias = state["case"], state["x"], state["weight"], state["target"], state["bias"]
    loss, lse, count = ce.linear_cross_entropy_forward(x, weight, target, bias, IGNORE, case["reduction"])
    if case["op"] == "loss":
        return {"loss": loss}
    dx, dweight, dbias = ce.linear_cross_entropy_backward(state["dloss"], x, weight, target, lse, count, bias, IGNORE, case["reduction"])
    out = {"loss": loss, "dx": dx, "dweight": dweight}
    if case["bias"]:
        out["dbias"] = dbias
    return out


def _polar(x, steps=5):
    """The Newton-Schulz iteration of a batch of matrices, in the type that x has."""
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    a, b, c = COEFFICIENTS
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(steps):
        s = x @ x.transpose(1, 2)
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.transpose(1, 2) if tall else x


def _by_shape(rows):
    """{shape: its places (row, matrix)}: matrices of one shape go through the products together."""
    places = {}
    for k, row in enumerate(rows):
        for j, t in enumerate(row):
            places.setdefault(tuple(t.shape), []).append((k, j))
    return places


def _plain_ortho(state):
    rows, to = state["rows"], DTYPES[state["case"]["result"]]
    for places in _by_shape(rows).values():
        y = _polar(torch.stack([rows[k][j].float() for k, j in places])).to(to)
        torch._foreach_copy_([state["out"][k][j] for k, j in places], list(y.unbind()))
    return {"flat": state["flat"]}


def _own_ortho(state):
    state["plan"](state["rows"], state["out"])
    return {"flat": state["flat"]}


def run(state):
    if state["case"]["op"] == "ortho":
        return _own_ortho(state) if own else _plain_ortho(state)
    return _own_loss(state) if own else _plain_loss(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "ortho":
        shapes = _matrices(case) * case["rows"]
        e = sum(m * n for m, n in shapes)
        # s = x x' and s s have half of their products by symmetry
        flops = 5 * sum(3 * min(m, n) ** 2 * max(m, n) + min(m, n) ** 3 for m, n in shapes)
        return {"bytes": e * (BYTES[case["dtype"]] + BYTES[case["result"]]), "flops": flops}
    n, d, v, b = (case["n"], case["d"], case["v"], BYTES[case["dtype"]])
    n_used = max(1, round(n * (1 - case["ignored"])))
    bias = v * b if case["bias"] else 0
    if case["op"] == "loss":
        return {"bytes": (n_used + v) * d * b + bias + 8 * n + 4 * (n if case["reduction"] == "none" else 1), "flops": 2 * n_used * d * v}
    # with nothing kept from the forward pass but the sums, the logits are made twice
    return {"bytes": (n_used + n + 2 * v) * d * b + 2 * bias + 8 * n, "flops": 8 * n_used * d * v}


# ---- the same from the definition, in 64 bits --------------------------------------------------------------------------------

def _exact_loss(state):
    case = state["case"]
    x, w, target = state["x"].double(), state["weight"].double(), state["target"]
    used = (target != IGNORE).nonzero()[:, 0]
    rows = torch.zeros(len(target), dtype=torch.float64, device="cuda")
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), w.new_zeros(len(w))
    for part in used.split(1024):
        z = x[part] @ w.t() + (state["bias"].double() if case["bias"] else 0.0)
        rows[part] = torch.logsumexp(z, 1) - z.gather(1, target[part, None])[:, 0]
        if case["op"] == "train":
            q = torch.softmax(z, 1)
            q[torch.arange(len(part), device="cuda"), target[part]] -= 1
            q *= (state["dloss"].double()[part, None] if case["reduction"] == "none" else
                  state["dloss"].double() / (len(used) if case["reduction"] == "mean" else 1))
            dx[part] = q @ w
            dw += q.t() @ x[part]
            db += q.sum(0)
    loss = {"none": rows, "sum": rows.sum(), "mean": rows.sum() / len(used)}[case["reduction"]]
    if case["op"] == "loss":
        return {"loss": loss}
    return {"loss": loss, "dx": dx, "dweight": dw} | ({"dbias": db} if case["bias"] else {})


def _exact_ortho(state):
    def one(g):
        g = g.double()
        a, b, c = COEFFICIENTS
        u, s, vt = torch.linalg.svd(g, full_matrices=False)
        s = s / (torch.linalg.matrix_norm(g) + EPS)
        for _ in range(5):                              # the iteration acts on the singular values alone
            s = a * s + b * s ** 3 + c * s ** 5
        return (u * s) @ vt
    flat = torch.zeros_like(state["flat"], dtype=torch.float64)
    for row, given in zip(flat, state["rows"]):
        at = 0
        for t in given:
            row[at:at + t.numel()] = one(t).reshape(-1)
            at += -(-t.numel() // ALIGN) * ALIGN
    return {"flat": flat}


def exact(case, seed):
    if case["op"] == "ortho":
        if sum(min(m, n) ** 2 * max(m, n) for m, n in _matrices(case)) * case["rows"] > 2e10 or len(_matrices(case)) * case["rows"] > 400:
            return None
        return _exact_ortho(_prepare_ortho(case, seed))
    return _exact_loss(_prepare_loss(case, seed))
