"""Performance cases of a training step in 8 bits before the codec, called as a user's training program calls them.

Activations are kept, and products are made, in e4m3 numbers with a power of two as the scale of each block of 128 columns, of 128
rows or of a single row.  A convolutional network's norms are group norms with an activation, channels last.  The weight gradients of
every user apart go to that user's row of the gradient buffer.  A case's fields:

  op        "checkpoint": x to 8 bits, as the forward pass keeps it, and back to its type, as a backward pass asks for it;
            "product": out = op(a) op(b) of tensors in 8 bits, form "nn", "nt" (b transposed) or "tn" (a transposed);
            "linear_backward": dy to 8 bits, dx = dy w and, for every user, dw = dy^T x from the x that was kept in 8 bits;
            "groupnorm": y, mean, rstd;  "groupnorm_backward": dx, and dweight, dbias of every user, from x or from x kept in 8 bits
  type      of x, y, dy and dx, and of a product's result: "fp32", "bf16" or "fp16".  Weights' gradients are fp32
  users     a batch of so many; in a product "shared" says that all have the same b
  block_rows    rows of a block of a product's a: 128 or 1
  rows, cols, outs    a linear layer's rows of a user, its inputs and its outputs;  m, n, k    a product's sizes
  samples, pixels, channels, groups    of a group norm, samples of each user;  kept    whether x is in 8 bits
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 128
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one small layer's activations: a call's latency
        dict(name="checkpoint_small", op="checkpoint", type="bf16", users=1, rows=64, cols=257),
        # what four users keep of a wide layer
        dict(name="checkpoint_users", op="checkpoint", type="bf16", users=4, rows=4096, cols=4096),
        # one row through a layer: reading the weights is all there is
        dict(name="product_one_row", op="product", type="bf16", form="nt", users=1, shared=True, block_rows=1, m=1, n=4096, k=4096),
        # odd sizes, a gradient through a layer whose sum runs across the weights' rows
        dict(name="product_odd", op="product", type="fp32", form="nn", users=1, shared=True, block_rows=128, m=1000, n=517, k=1001),
        # a large layer's forward pass
        dict(name="product_large", op="product", type="bf16", form="nt", users=1, shared=True, block_rows=1, m=8192, n=4096, k=4096),
        # the backward pass of a small layer, eight users with a weight gradient each
        dict(name="linear_backward_users", op="linear_backward", type="bf16", users=8, rows=500, cols=1024, outs=1000),
        # the backward pass of a large layer
        dict(name="linear_backward_large", op="linear_backward", type="bf16", users=4, rows=4096, cols=4096, outs=4096),
        # two small images: a call's latency
        dict(name="groupnorm_small", op="groupnorm", type="bf16", act="silu", users=1, samples=2, pixels=64, channels=64, groups=8),
        # a batch of images of 32 x 32
        dict(name="groupnorm_batch", op="groupnorm", type="bf16", act="silu", users=1, samples=256, pixels=1024, channels=256, groups=32),
        # eight users' images, fp32, groups of an odd number of channels
        dict(name="groupnorm_backward_users", op="groupnorm_backward", type="fp32", act="relu", users=8, samples=16, pixels=1024, channels=60,
             groups=4, kept=False),
        # four users' images, x kept in 8 bits
        dict(name="groupnorm_backward_kept", op="groupnorm_backward", type="bf16", act="silu", users=4, samples=32, pixels=1024, channels=256,
             groups=32, kept=True),
        # a few large images
        dict(name="groupnorm_backward_large", op="groupnorm_backward", type="bf16", act="silu", users=1, samples=4, pixels=16384, channels=512,
             groups=32, kept=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["checkpoint", "product", "product", "linear_backward", "groupnorm", "groupnorm_backward", "groupnorm_backward"])
    kind = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if op == "checkpoint":
        cols, users = _log(rng, 16, 8192), rng.choice([1, 1, 2, 5, 16])
        return dict(op=op, type=kind, users=users, rows=max(1, _log(rng, 1, min(65536, 6e7 / cols)) // users), cols=cols)
    if op == "product":
        form, users = rng.choice(["nn", "nt", "nt", "tn"]), rng.choice([1, 1, 1, 3, 8])
        n, k = _log(rng, 16, 8192), _log(rng, 16, 8192)
        m = max(1, _log(rng, 1, min(32768, 1e11 / (n * k))) // users)
        return dict(op=op, type=kind, form=form, users=users, shared=form != "tn" and rng.random() < 0.7,
                    block_rows=128 if form == "tn" else rng.choice([1, 128]), m=m, n=n, k=k)
    if op == "linear_backward":
        cols, outs, users = _log(rng, 16, 8192), _log(rng, 16, 8192), rng.choice([1, 2, 4, 8, 16])
        return dict(op=op, type=kind, users=users, rows=max(1, _log(rng, 1, min(32768, 1e11 / (cols * outs))) // users), cols=cols, outs=outs)
    groups, width = _log(rng, 1, 64), _log(rng, 1, 64)
    channels, pixels = groups * width, _log(rng, 1, 16384)
    users = rng.choice([1, 1, 2, 4, 8])
    case = dict(op=op, type=kind, act=rng.choice(["silu", "relu", "none"]), users=users,
                samples=max(1, _log(rng, 1, min(4096, 6e7 / (channels * pixels))) // users), pixels=pixels, channels=channels, groups=groups)
    if op == "groupnorm_backward":
        case["kept"] = rng.random() < 0.4
    return case


def _ceil(n, d):
    return -(-n // d)


def _tiles(x, block_rows):
    """[users, block rows, rows of a block, block columns, 128] of x [users, rows, cols], filled up with zeros."""
    users, rows, cols = x.shape
    up = (_ceil(rows, block_rows), _ceil(cols, BLOCK))
    x = torch.nn.functional.pad(x, (0, up[1] * BLOCK - cols, 0, up[0] * block_rows - rows))
    return x.view(users, up[0], block_rows, up[1], BLOCK)


def _to_8_bits(x, block_rows):
    """e4m3 values [users, rows, cols] and the scales' exponents [users, block rows, block columns] of fp32 x: the least power of two
    by which a block's largest value is at most 448."""
    tiles = _tiles(x, block_rows)
    mantissa, exponent = torch.frexp(tiles.abs().amax(dim=(2, 4)))
    scale = torch.where(mantissa == 0, 0, (exponent - 9 + (mantissa > 0.875)).clamp(min=-126))
    inverse = ((127 - scale) << 23).to(torch.int32).view(torch.float32)
    values = (tiles * inverse[:, :, None, :, None]).to(torch.float8_e4m3fn)
    return values.reshape(x.shape[0], tiles.shape[1] * block_rows, -1)[:, :x.shape[1], :x.shape[2]], scale


def _from_8_bits(values, scale, block_rows):
    """fp32 of what _to_8_bits gives."""
    rows, cols = values.shape[1:]
    power = ((scale + 127) << 23).to(torch.int32).view(torch.float32)
    return values.to(torch.float32) * power.repeat_interleave(block_rows, dim=1).repeat_interleave(BLOCK, dim=2)[:, :rows, :cols]


def _stored(x, block_rows=BLOCK):
    """What a program keeps of x: the values' bytes, rows 16 bytes aligned and filled up with zeros, and the scales' bytes, those of a
    column of blocks next to each other, 16 bytes aligned and filled up too."""
    values, scale = _to_8_bits(x.float(), block_rows)
    users, rows, cols = x.shape
    whole = torch.zeros((users, rows, _ceil(cols, 16) * 16), dtype=torch.uint8, device=x.device)
    whole[:, :, :cols] = values.contiguous().view(torch.uint8)
    scales = torch.nn.functional.pad((scale + 127).to(torch.uint8).mT, (0, -scale.shape[1] % 16)).contiguous()
    return dict(values=whole, scales=scales, cols=cols, block_rows=block_rows)


def _numbers(kept):
    """fp32 of what _stored gives."""
    values = kept["values"][:, :, :kept["cols"]].contiguous().view(torch.float8_e4m3fn)
    scale = kept["scales"][:, :, :_ceil(values.shape[1], kept["block_rows"])].mT.int() - 127
    return _from_8_bits(values, scale, kept["block_rows"])


def _activations(gen, dev, users, rows, cols):
    """Rows of sizes of their own, some columns far larger than the others, and about a third of zeros."""
    x = torch.randn((users, rows, cols), generator=gen, device=dev)
    x *= torch.empty((users, rows, 1), device=dev).uniform_(0.3, 3.0, generator=gen)
    x[:, :, ::61] *= 8
    return x.clamp_(min=-0.4).add_(0.4)


def _gradients(gen, dev, users, rows, cols):
    size = torch.empty((users, rows, 1), device=dev).uniform_(math.log(1e-5), math.log(1e-2), generator=gen).exp_()
    return torch.randn((users, rows, cols), generator=gen, device=dev) * size


def _weights(gen, dev, users, rows, cols):
    return torch.randn((users, rows, cols), generator=gen, device=dev) / math.sqrt(cols)


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t, users, op = TYPES[case["type"]], case["users"], case["op"]
    if op == "checkpoint":
        return dict(x=_activations(gen, dev, users, case["rows"], case["cols"]).to(t))
    if op == "product":
        m, n, k, form = case["m"], case["n"], case["k"], case["form"]
        shared = 1 if case["shared"] else users
        if form == "tn":
            return dict(a=_stored(_gradients(gen, dev, users, k, m)), b=_stored(_activations(gen, dev, shared, k, n)))
        b = _weights(gen, dev, shared, n, k) if form == "nt" else _weights(gen, dev, shared, k, n)
        return dict(a=_stored(_activations(gen, dev, users, m, k), case["block_rows"]), b=_stored(b))
    if op == "linear_backward":
        rows, cols, outs = case["rows"], case["cols"], case["outs"]
        return dict(dy=_gradients(gen, dev, users, rows, outs).to(t), x=_stored(_activations(gen, dev, users, rows, cols)),
                    w=_stored(_weights(gen, dev, 1, outs, cols)))
    count, pixels, channels = users * case["samples"], case["pixels"], case["channels"]
    x = torch.randn((count, pixels, channels), generator=gen, device=dev)
    x *= torch.empty((count, 1, channels), device=dev).uniform_(0.5, 2.0, generator=gen)
    x += torch.randn((count, 1, channels), generator=gen, device=dev)
    s = dict(x=x.to(t), weight=1 + 0.2 * torch.randn(channels, generator=gen, device=dev), bias=0.2 * torch.randn(channels, generator=gen, device=dev))
    if op == "groupnorm_backward":
        s["dy"] = (1e-2 * torch.randn((count, pixels, channels), generator=gen, device=dev)).to(t)
        grouped = s["x"].double().view(count, pixels, case["groups"], -1)   # what the forward pass left
        s["mean"] = grouped.mean(dim=(1, 3)).float()
        s["rstd"] = (grouped.var(dim=(1, 3), unbiased=False) + EPS).rsqrt().float()
        if case["kept"]:
            s["x"] = _stored(s["x"].view(users, -1, channels))
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The workspaces and the output buffers that a program keeps, and what it kept in 8 bits as the calls take it."""
    from paper_2204_08211_amd import binding as B
    case, t, dev = s["case"], TYPES[s["case"]["type"]], "cuda:0"
    users, op = case["users"], case["op"]
    for name in ("a", "b", "w", "x"):
        if isinstance(s.get(name), dict):
            k = s[name]
            s[name] = B.Blocks8(k["values"], k["scales"], k["cols"], block_rows=k["block_rows"])
    if op == "checkpoint":
        s["kept"] = B.Blocks8.empty(users, case["rows"], case["cols"], device=dev)
        s["back"] = torch.empty_like(s["x"])
    elif op == "product":
        s["out"] = torch.empty((users, case["m"], case["n"]), dtype=t, device=dev)
        s["ta"], s["tb"] = case["form"] == "tn", case["form"] == "nt"
        s["workspace"] = torch.empty(B.co3_matmul8_workspace_bytes(s["a"], s["b"], transpose_a=s["ta"], transpose_b=s["tb"]), dtype=torch.uint8, device=dev)
    elif op == "linear_backward":
        s["dy8"] = B.Blocks8.empty(users, case["rows"], case["outs"], device=dev)
        s["dx"] = torch.empty((users, case["rows"], case["cols"]), dtype=t, device=dev)
        s["dw"] = torch.empty((users, case["outs"], case["cols"]), device=dev)
        s["workspace"] = torch.empty(max(B.co3_matmul8_workspace_bytes(s["dy8"], s["w"]), B.co3_matmul8_workspace_bytes(s["dy8"], s["x"], transpose_a=True)),
                                     dtype=torch.uint8, device=dev)
    else:
        s["act"] = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU}[case["act"]]
        count, channels, groups = users * case["samples"], case["channels"], case["groups"]
        shape = (count, case["pixels"], channels)
        if op == "groupnorm":
            s["y"] = torch.empty(shape, dtype=t, device=dev)
            s["mean"], s["rstd"] = torch.empty((count, groups), device=dev), torch.empty((count, groups), device=dev)
            need = B.co3_groupnorm_workspace_bytes(*shape, groups, t)
        else:
            s["dx"] = torch.empty(shape, dtype=t, device=dev)
            s["grad"] = torch.zeros((users, 2 * channels), device=dev)   # a row of the gradient buffer holds both, the weight's and behind it the bias's
            need = B.co3_groupnorm_backward_workspace_bytes(users, *shape, groups, t)
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=dev)


def _run_own(s):
    from paper_2204_08211_amd import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "checkpoint":
        B.co3_quantize8(s["x"], out=s["kept"])
        return dict(back=B.co3_dequantize8(s["kept"], out=s["back"]))
    if op == "product":
        return dict(out=B.co3_matmul8(s["a"], s["b"], out=s["out"], transpose_a=s["ta"], transpose_b=s["tb"], workspace=s["workspace"]))
    if op == "linear_backward":
        B.co3_quantize8(s["dy"], out=s["dy8"])
        B.co3_matmul8(s["dy8"], s["w"], out=s["dx"], workspace=s["workspace"])
        B.co3_matmul8(s["dy8"], s["x"], out=s["dw"], transpose_a=True, workspace=s["workspace"])
        return dict(dx=s["dx"], dw=s["dw"])
    if op == "groupnorm":
        B.co3_groupnorm(s["x"], case["groups"], s["weight"], s["bias"], eps=EPS, activation=s["act"], y=s["y"], mean=s["mean"], rstd=s["rstd"],
                        workspace=s["workspace"])
        return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
    c = case["channels"]
    dweight, dbias = s["grad"][:, :c], s["grad"][:, c:]
    B.co3_groupnorm_backward(s["dy"], s["x"], case["groups"], s["weight"], s["bias"], s["mean"], s["rstd"], activation=s["act"], users=case["users"],
                             dx=s["dx"], dweight=dweight, dbias=dbias, workspace=s["workspace"])
    return dict(dx=s["dx"], dweight=dweight, dbias=dbias)


def run(state):
    if own:
        return _run_own(state)
    case, op = state["case"], state["case"]["op"]
    t = TYPES[case["type"]]
    if op == "checkpoint":
        most = torch.finfo(t).max
        return dict(back=_from_8_bits(*_to_8_bits(state["x"].float(), BLOCK), BLOCK).clamp(-most, most).to(t))
    if op == "product":
        a, b = _numbers(state["a"]), _numbers(state["b"])
        a, b = a.mT if case["form"] == "tn" else a, b.mT if case["form"] == "nt" else b
        return dict(out=torch.matmul(a, b[0] if case["shared"] else b).to(t))
    if op == "linear_backward":
        dy = _from_8_bits(*_to_8_bits(state["dy"].float(), BLOCK), BLOCK)
        return dict(dx=torch.matmul(dy, _numbers(state["w"])[0]).to(t), dw=torch.matmul(dy.mT, _numbers(state["x"])))
    count, pixels, channels, groups = case["users"] * case["samples"], case["pixels"], case["channels"], case["groups"]
    weight, bias = state["weight"].view(groups, -1), state["bias"].view(groups, -1)
    if op == "groupnorm":
        x = state["x"].float().view(count, pixels, groups, -1)
        mean = x.mean(dim=(1, 3))
        centred = x - mean[:, None, :, None]
        rstd = torch.rsqrt(centred.square().mean(dim=(1, 3)) + EPS)
        z = centred * rstd[:, None, :, None] * weight + bias
        if case["act"] == "relu":
            z = z.clamp(min=0)
        elif case["act"] == "silu":
            z = z / (1 + torch.exp(-z))
        return dict(y=z.view(count, pixels, channels).to(t), mean=mean, rstd=rstd)
    x = (_numbers(state["x"]) if case["kept"] else state["x"].float()).view(count, pixels, groups, -1)
    rstd = state["rstd"][:, None, :, None]
    xhat = (x - state["mean"][:, None, :, None]) * rstd
    dz = state["dy"].float().view(count, pixels, groups, -1)
    if case["act"] == "relu":
        dz = dz * (xhat * weight + bias > 0)
    elif case["act"] == "silu":
        z = xhat * weight + bias
        sigma = 1 / (1 + torch.exp(-z))
        dz = dz * sigma * (1 + z * (1 - sigma))
    t_ = dz * weight
    dx = rstd * (t_ - t_.mean(dim=(1, 3), keepdim=True) - xhat * (t_ * xhat).mean(dim=(1, 3), keepdim=True))
    sums = (case["users"], case["samples"] * pixels, channels)
    return dict(dx=dx.view(count, pixels, channels).to(t), dweight=(dz * xhat).view(sums).sum(dim=1), dbias=dz.view(sums).sum(dim=1))


def _exact_numbers(values, scales, block_rows):
    """Numbers in 64 bits of bytes: sign, four bits of an exponent, three of a fraction; times a power of two for each block."""
    v = values.long()
    field, fraction = (v >> 3) & 15, (v & 7).double()
    size = torch.where(field == 0, fraction * 2.0 ** -9, (8 + fraction) * torch.pow(torch.full_like(fraction, 2.0), (field - 10).double()))
    size = torch.where(v >= 128, -size, size)
    row = torch.arange(v.shape[1], device=v.device) // block_rows
    col = torch.arange(v.shape[2], device=v.device) // BLOCK
    return size * torch.pow(2.0, scales.mT.double() - 127)[:, row][:, :, col]


def _exact_rounded(x):
    """x in 64 bits, rounded to a multiple of its binade's eighth (of 2^-6's below 2^-6) within its block's scale, ties to even."""
    out = torch.empty_like(x)
    for r in range(0, x.shape[1], BLOCK):
        rows = x[:, r:r + BLOCK]
        most = torch.nn.functional.pad(rows.abs().amax(dim=1), (0, -x.shape[2] % BLOCK)).view(x.shape[0], -1, BLOCK).amax(dim=2)
        e = torch.ceil(torch.log2(most.clamp(min=1e-300) / 448)).clamp(min=-126)
        e = torch.where(most > 448 * torch.exp2(e), e + 1, e)
        e = torch.where((most <= 224 * torch.exp2(e)) & (e > -126), e - 1, e)
        unit = torch.exp2(e).repeat_interleave(BLOCK, dim=1)[:, None, :x.shape[2]]
        v = rows / unit
        step = torch.exp2(torch.frexp(v)[1].clamp(min=-5).double() - 4)
        out[:, r:r + BLOCK] = torch.round(v / step) * step * unit
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op, users = case["op"], case["users"]
    if op == "checkpoint":
        most = torch.finfo(TYPES[case["type"]]).max
        return dict(back=_exact_rounded(s["x"].double()).clamp(-most, most))
    numbers = lambda k: _exact_numbers(k["values"][:, :, :k["cols"]], k["scales"], k["block_rows"])  # noqa: E731
    if op == "product":
        a, b, form = numbers(s["a"]), numbers(s["b"]), case["form"]
        out = [torch.mm(a[u].t() if form == "tn" else a[u], (lambda m: m.t() if form == "nt" else m)(b[0 if case["shared"] else u])) for u in range(users)]
        return dict(out=torch.stack(out))
    if op == "linear_backward":
        dy, x, w = _exact_rounded(s["dy"].double()), numbers(s["x"]), numbers(s["w"])[0]
        return dict(dx=torch.stack([torch.mm(d, w) for d in dy]), dw=torch.stack([torch.mm(d.t(), k) for d, k in zip(dy, x)]))
    count, pixels, channels, groups = users * case["samples"], case["pixels"], case["channels"], case["groups"]
    width = channels // groups
    weight, bias = s["weight"].double(), s["bias"].double()
    spread = lambda v: v.double().repeat_interleave(width, dim=1)[:, None, :]  # noqa: E731
    per_group = lambda v: v.sum(dim=1).view(count, groups, width).sum(dim=2) / (pixels * width)  # noqa: E731
    if op == "groupnorm":
        x = s["x"].double()
        mean = per_group(x)
        d = x - spread(mean)
        rstd = (per_group(d * d) + EPS) ** -0.5
        z = d * spread(rstd) * weight + bias
        y = torch.where(z > 0, z, 0.0) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z
        return dict(y=y, mean=mean, rstd=rstd)
    x = numbers(s["x"]).view(count, pixels, channels) if case["kept"] else s["x"].double()
    h = (x - spread(s["mean"])) * spread(s["rstd"])
    z, dz = h * weight + bias, s["dy"].double()
    if case["act"] == "relu":
        # whether a value next to 0 passes hangs on the last bit of an fp32 product and sum
        z32 = (x.float() - s["mean"].repeat_interleave(width, dim=1)[:, None, :]) * s["rstd"].repeat_interleave(width, dim=1)[:, None, :] * s["weight"] + s["bias"]
        dz = torch.where(z32 > 0, dz, 0.0)
    elif case["act"] == "silu":
        p = torch.sigmoid(z)
        dz = dz * (p + z * p * torch.sigmoid(-z))
    p = dz * weight
    dx = spread(s["rstd"]) * (p - spread(per_group(p)) - h * spread(per_group(p * h)))
    by_user = lambda v: v.view(users, -1, channels).sum(dim=1)  # noqa: E731
    return dict(dx=dx, dweight=by_user(dz * h), dbias=by_user(dz))


def work(case):
    size = 4 if case["type"] == "fp32" else 2
    op, users = case["op"], case["users"]
    if op == "checkpoint":     # x read, the checkpoint written; it read, x written
        elements = users * case["rows"] * case["cols"]
        return dict(bytes=elements * (2 * size + 2), flops=4 * elements)
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(bytes=users * m * k + (1 if case["shared"] else users) * n * k + users * m * n * size, flops=2 * users * m * n * k)
    if op == "linear_backward":
        rows, cols, outs = case["rows"], case["cols"], case["outs"]
        return dict(bytes=users * rows * (outs * size + cols + cols * size) + outs * cols + 4 * users * outs * cols, flops=4 * users * rows * cols * outs)
    elements = users * case["samples"] * case["pixels"] * case["channels"]
    rows, channels = 8 * users * case["samples"] * case["groups"], case["channels"]
    if op == "groupnorm":
        return dict(bytes=elements * 2 * size + rows + 8 * channels, flops=elements * 10)
    return dict(bytes=elements * (2 * size + (1 if case["kept"] else size)) + rows + (8 + 8 * users) * channels, flops=elements * 20)
