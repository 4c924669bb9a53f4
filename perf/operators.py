"""Performance cases of the training operators on either side of the codec, called as a training program calls them.

Before the codec: layer norm's forward and backward pass, whose weight gradients are those of each user apart and go to
that user's row of the gradient buffer.  After it: the PS makes an update of the average - every matrix of the flat
model vector is orthogonalised by Newton-Schulz products, with momentum and weight decay around that.  A case's fields:

  op        "orthogonalize": out = scale NS(g) for every matrix of a flat vector;
            "muon": m = beta m + g, u = g + beta m, w = w (1 - eta decay) - eta scale NS(u), all of them fp32;
            "norm": y, mean, rstd of every row;  "norm_backward": dx, and dweight, dbias of every user
  matrices  "64x128*2,10x33": rows x columns * how many, one behind the other in the flat vector
  type      of g and out, or of x, y, dy and dx: "fp32", "bf16" or "fp16".  Weights and their gradients are fp32
  steps     Newton-Schulz steps, with the coefficients of Muon's quintic
  users, rows, cols    users of that many rows each;  pad: rows lie cols + pad elements apart
  affine    whether the norm has a weight and a bias

Gradients of matrices are sums of a few outer products with falling weights and of noise, as a batch's gradient is.
"""
import math

import torch

own = False

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
BETA, ETA, DECAY = 0.95, 0.02, 0.01
NORM_EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one small layer: a call's latency
        dict(name="ortho_one_small", op="orthogonalize", type="bf16", matrices="64x64", steps=5),
        # layers of odd shapes in one call: a classifier's, a wide and a narrow one, a single row
        dict(name="ortho_odd", op="orthogonalize", type="bf16", matrices="1000x2048,257x1023,33x4097,1x777", steps=5),
        # four tall matrices, fp32 as the codec's average is
        dict(name="ortho_tall_fp32", op="orthogonalize", type="fp32", matrices="2048x512*4", steps=5),
        # one large square layer
        dict(name="ortho_square", op="orthogonalize", type="bf16", matrices="4096x4096", steps=5),
        # the update of a network of 20 thousand elements
        dict(name="muon_small", op="muon", type="fp32", matrices="64x64*2,128x64,10x128", steps=5),
        # the update of some 25 million elements: projections and the two layers of the blocks between them
        dict(name="muon_blocks", op="muon", type="fp32", matrices="1024x1024*8,4096x1024*2,1024x4096*2", steps=5),
        # the fully connected part of a network of 138 million elements
        dict(name="muon_large", op="muon", type="fp32", matrices="4096x25088,4096x4096,1000x4096", steps=5),
        # a few rows: a call's latency
        dict(name="norm_few_rows", op="norm", type="bf16", users=1, rows=8, cols=1024, pad=0, affine=True),
        # a batch of a large model's activations
        dict(name="norm_batch", op="norm", type="bf16", users=1, rows=16384, cols=4096, pad=0, affine=True),
        # the backward pass of a few rows
        dict(name="norm_backward_few_rows", op="norm_backward", type="bf16", users=2, rows=8, cols=512, pad=0, affine=True),
        # eight users' batches with a weight gradient each, fp32, rows of an odd length
        dict(name="norm_backward_users", op="norm_backward", type="fp32", users=8, rows=1024, cols=1001, pad=3, affine=True),
        # the backward pass of a large batch
        dict(name="norm_backward_batch", op="norm_backward", type="bf16", users=1, rows=16384, cols=8192, pad=0, affine=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["orthogonalize", "muon", "norm", "norm_backward"])
    if op in ("norm", "norm_backward"):
        cols = _log(rng, 16, 16384)
        users = rng.choice([1, 1, 2, 3, 8, 16])
        rows = max(1, _log(rng, 1, min(32768, 6e7 / cols)) // users)
        return dict(op=op, type=rng.choice(["fp32", "bf16", "bf16", "fp16"]), users=users, rows=rows, cols=cols,
                    pad=rng.choice([0, 0, 8, 24, 5]), affine=rng.random() < 0.9)
    groups, left = [], 4e11
    for _ in range(rng.choice([1, 1, 2, 3, 4])):
        rows, cols, count = _log(rng, 2, 4096), _log(rng, 2, 8192), rng.choice([1, 1, 1, 2, 4])
        need = count * _step_flops(rows, cols)
        if need <= left:
            groups.append("%dx%d*%d" % (rows, cols, count))
            left -= need
    if not groups:
        groups.append("%dx%d*1" % (_log(rng, 2, 1024), _log(rng, 2, 2048)))
    return dict(op=op, type="fp32" if op == "muon" else rng.choice(["fp32", "bf16", "bf16", "fp16"]),
                matrices=",".join(groups), steps=rng.choice([5, 5, 5, 3, 6]))


def _groups(case):
    """(rows, columns, how many) of every group of a case's matrices."""
    out = []
    for text in case["matrices"].split(","):
        shape, _, count = text.partition("*")
        rows, cols = shape.split("x")
        out.append((int(rows), int(cols), int(count or 1)))
    return out


def _scale(rows, cols):
    return math.sqrt(max(1.0, rows / cols))


def _matrix_gradients(groups, gen, dev):
    """A flat fp32 vector of all matrices: eight outer products with falling weights, and noise of half their size."""
    parts = []
    for rows, cols, count in groups:
        r = min(8, rows, cols)
        weight = torch.arange(1, r + 1, device=dev, dtype=torch.float32).pow(-1.0)
        left = torch.randn((count, rows, r), generator=gen, device=dev) * weight
        g = left @ torch.randn((count, r, cols), generator=gen, device=dev)
        g += 0.5 * torch.randn((count, rows, cols), generator=gen, device=dev)
        size = torch.empty((count, 1, 1), device=dev).uniform_(math.log(1e-4), math.log(1e-2), generator=gen).exp_()
        parts.append((g * size).reshape(-1))
    return torch.cat(parts)


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = TYPES[case["type"]]
    if case["op"] in ("orthogonalize", "muon"):
        groups = _groups(case)
        s = dict(g=_matrix_gradients(groups, gen, dev).to(t))
        if case["op"] == "muon":
            s["momentum"] = 3 * s["g"] + 6 * _matrix_gradients(groups, gen, dev)
            s["model"] = torch.cat([torch.randn(n * r * c, generator=gen, device=dev) / math.sqrt(c) for r, c, n in groups])
        return s
    users, rows, cols = case["users"], case["rows"], case["cols"]

    def rows_of(scale):
        whole = torch.randn((users, rows, cols + case["pad"]), generator=gen, device=dev)
        return (whole * scale).to(t)[:, :, :cols]

    # a row's own mean and size, and some columns far larger than the others
    size = torch.empty((users, rows, 1), device=dev).uniform_(0.5, 2.0, generator=gen)
    x = rows_of(size)
    x += (0.5 * torch.randn((users, rows, 1), generator=gen, device=dev)).to(t)
    x[:, :, ::61] *= 4
    s = dict(x=x, weight=None, bias=None)
    if case["affine"]:
        s["weight"] = 1 + 0.2 * torch.randn(cols, generator=gen, device=dev)
        s["bias"] = 0.1 * torch.randn(cols, generator=gen, device=dev)
    if case["op"] == "norm_backward":
        s["dy"] = rows_of(1e-2)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["op"] in ("orthogonalize", "muon"):
        s["groups"] = _groups(case)
    if case["op"] == "norm_backward":   # what the forward pass left
        x = s["x"].float()
        mean = x.mean(dim=2)
        s["mean"] = mean
        s["rstd"] = torch.rsqrt((x - mean[:, :, None]).square().mean(dim=2) + NORM_EPS)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The plan, the workspace and the output buffers that a program keeps."""
    from paper_2204_08211_amd import binding as B
    case = s["case"]
    if case["op"] in ("orthogonalize", "muon"):
        matrices, offset = [], 0
        for rows, cols, count in s["groups"]:
            for _ in range(count):
                matrices.append((offset, rows, cols))
                offset += rows * cols
        s["plan"] = B.MatrixPlan(matrices, dtype=TYPES[case["type"]], scales=[_scale(r, c) for _, r, c in matrices])
        s["workspace"] = torch.empty(s["plan"].workspace_bytes, dtype=torch.uint8, device="cuda:0")
        if case["op"] == "orthogonalize":
            s["out"] = torch.empty_like(s["g"])
        return
    shape = (case["users"], case["rows"], case["cols"])
    if case["op"] == "norm":
        s["y"] = torch.empty(shape, dtype=s["x"].dtype, device="cuda:0")
        s["mean"] = torch.empty(shape[:2], device="cuda:0")
        s["rstd"] = torch.empty(shape[:2], device="cuda:0")
    else:
        s["dx"] = torch.empty(shape, dtype=s["x"].dtype, device="cuda:0")
        if case["affine"]:   # a row of the gradient buffer holds both, the weight's and behind it the bias's
            s["grad"] = torch.zeros((case["users"], 2 * case["cols"]), device="cuda:0")
        s["workspace"] = torch.empty(B.co3_layernorm_backward_workspace_bytes(*shape), dtype=torch.uint8, device="cuda:0")


def _run_own(s):
    from paper_2204_08211_amd import binding as B
    case = s["case"]
    if case["op"] == "orthogonalize":
        B.co3_orthogonalize(s["plan"], s["g"], s["out"], steps=case["steps"], workspace=s["workspace"])
        return dict(out=s["out"])
    if case["op"] == "muon":
        B.co3_muon_update(s["plan"], s["g"], s["momentum"], s["model"], eta=ETA, beta=BETA, weight_decay=DECAY,
                          steps=case["steps"], workspace=s["workspace"])
        return dict(momentum=s["momentum"], model=s["model"])
    if case["op"] == "norm":
        B.co3_layernorm(s["x"], s["weight"], s["bias"], eps=NORM_EPS, y=s["y"], mean=s["mean"], rstd=s["rstd"])
        return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
    cols = case["cols"]
    dweight, dbias = (s["grad"][:, :cols], s["grad"][:, cols:]) if case["affine"] else (None, None)
    B.co3_layernorm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], dx=s["dx"], dweight=dweight, dbias=dbias,
                             workspace=s["workspace"])
    return dict(dx=s["dx"], dweight=dweight, dbias=dbias)


def _newton_schulz(g, steps):
    """[count, rows, cols] fp32: the plain iteration, on the transposed matrices where they are tall."""
    a, b, c = COEFFICIENTS
    x = g.mT.contiguous() if g.shape[1] > g.shape[2] else g
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(steps):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if g.shape[1] > g.shape[2] else x


def _orthogonalized(flat, groups, steps):
    """The scaled iteration of every group of equal matrices of a flat vector."""
    parts, offset = [], 0
    for rows, cols, count in groups:
        g = flat[offset:offset + rows * cols * count].view(count, rows, cols)
        parts.append((_scale(rows, cols) * _newton_schulz(g, steps)).reshape(-1))
        offset += rows * cols * count
    return torch.cat(parts)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "orthogonalize":
        return dict(out=_orthogonalized(state["g"].float(), state["groups"], case["steps"]).to(state["g"].dtype))
    if case["op"] == "muon":
        g, m, w = state["g"], state["momentum"], state["model"]
        m.mul_(BETA).add_(g)
        update = _orthogonalized(g + BETA * m, state["groups"], case["steps"])
        w.mul_(1 - ETA * DECAY).sub_(ETA * update)
        return dict(momentum=m, model=w)
    x = state["x"].float()
    weight, bias = state["weight"], state["bias"]
    if case["op"] == "norm":
        mean = x.mean(dim=2)
        centred = x - mean[:, :, None]
        rstd = torch.rsqrt(centred.square().mean(dim=2) + NORM_EPS)
        y = centred * rstd[:, :, None]
        if case["affine"]:
            y = y * weight + bias
        return dict(y=y.to(state["x"].dtype), mean=mean, rstd=rstd)
    dy, rstd = state["dy"].float(), state["rstd"][:, :, None]
    xhat = (x - state["mean"][:, :, None]) * rstd
    t = dy * weight if case["affine"] else dy
    dx = rstd * (t - t.mean(dim=2, keepdim=True) - xhat * (t * xhat).mean(dim=2, keepdim=True))
    out = dict(dx=dx.to(state["x"].dtype), dweight=None, dbias=None)
    if case["affine"]:
        out.update(dweight=(dy * xhat).sum(dim=1), dbias=dy.sum(dim=1))
    return out


def exact(case, seed):
    """The definitions in 64 bits.  The iteration in Horner's form, X times a polynomial of the smaller Gram matrix."""
    s = _inputs(case, seed)
    if case["op"] in ("orthogonalize", "muon"):
        u = s["g"].double()
        if case["op"] == "muon":
            m = BETA * s["momentum"].double() + u
            u = u + BETA * m
        parts, offset = [], 0
        a, b, c = COEFFICIENTS
        for rows, cols, count in _groups(case):
            for _ in range(count):
                x = u[offset:offset + rows * cols].view(rows, cols)
                x = x / (torch.linalg.vector_norm(x) + EPS)
                eye = torch.eye(min(rows, cols), dtype=torch.float64, device=x.device)
                for _ in range(case["steps"]):
                    if rows <= cols:
                        k = torch.mm(x, x.t())
                        x = torch.mm(a * eye + torch.mm(k, b * eye + c * k), x)
                    else:
                        k = torch.mm(x.t(), x)
                        x = torch.mm(x, a * eye + torch.mm(k, b * eye + c * k))
                parts.append((_scale(rows, cols) * x).reshape(-1))
                offset += rows * cols
        o = torch.cat(parts)
        if case["op"] == "orthogonalize":
            return dict(out=o)
        return dict(momentum=m, model=s["model"].double() * (1 - ETA * DECAY) - ETA * o)
    x = s["x"].double()
    weight = s["weight"].double() if case["affine"] else torch.ones((), dtype=torch.float64, device=x.device)
    mean = x.sum(dim=2, keepdim=True) / case["cols"]
    var = (x - mean).pow(2).sum(dim=2, keepdim=True) / case["cols"]
    rstd = (var + NORM_EPS) ** -0.5
    z = (x - mean) * rstd
    if case["op"] == "norm":
        y = z * weight + (s["bias"].double() if case["affine"] else 0.0)
        return dict(y=y, mean=mean[:, :, 0], rstd=rstd[:, :, 0])
    dy = s["dy"].double()
    p = dy * weight
    dx = (p - (p.sum(dim=2, keepdim=True) + z * (p * z).sum(dim=2, keepdim=True)) / case["cols"]) * rstd
    if not case["affine"]:
        return dict(dx=dx, dweight=None, dbias=None)
    return dict(dx=dx, dweight=(dy * z).sum(dim=1), dbias=dy.sum(dim=1))


def _step_flops(rows, cols):
    """One Newton-Schulz step: X X^T and its square are symmetric, (b A + c A^2) X is a whole product."""
    m, n = min(rows, cols), max(rows, cols)
    return m * m * n + m * m * m + 2 * m * m * n


def work(case):
    size = 4 if case["type"] == "fp32" else 2
    if case["op"] in ("orthogonalize", "muon"):
        groups = _groups(case)
        elements = sum(r * c * n for r, c, n in groups)
        flops = case["steps"] * sum(n * _step_flops(r, c) for r, c, n in groups)
        return dict(bytes=elements * (20 if case["op"] == "muon" else 2 * size), flops=flops)
    rows, cols, users = case["users"] * case["rows"], case["cols"], case["users"]
    if case["op"] == "norm":
        return dict(bytes=2 * rows * cols * size + 8 * rows + (8 * cols if case["affine"] else 0), flops=8 * rows * cols)
    return dict(bytes=3 * rows * cols * size + 8 * rows + ((4 + 8 * users) * cols if case["affine"] else 0), flops=14 * rows * cols)
