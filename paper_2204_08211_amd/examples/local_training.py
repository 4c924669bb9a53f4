#!/usr/bin/env python3
"""Algorithm 1 with what stands before and behind the codec: U users train a residual network with layer norms on their
own data, and the PS updates its matrices as Muon does.  One iteration, all of it on the device:

  users   forward and backward pass; layer norm's are co3_layernorm and co3_layernorm_backward, which writes every user's weight
          gradients into that user's row of the gradient buffer                        (line 7)
          co3_encode: error feedback, conversion, Huffman code                         (lines 8-10)
  PS      co3_ps_aggregate: decode and average                                         (lines 13-14)
          co3_muon_update: momentum, every matrix of the average orthogonalised, update of the model; the norms' weights take
          a plain step (--sgd: the matrices too)                                       (line 14)

The network is h <- h + W2 relu(W1 norm(h)) a few times and out = W norm(h), fitted to a fixed random network of the same kind.
With --images it is one for images, in 8 bits: h <- h + W n a few times and out = W n, n = silu(group norm(h)), at every pixel.  Its
products are co3_matmul8's, of tensors that co3_quantize8 makes; what the backward pass needs, h and n of every block, is kept as
such a tensor, a byte an element.
Prints the mean squared error and the bits per element sent.

    python -m paper_2204_08211_amd.examples.local_training [--users 4] [--width 256] [--blocks 3] [--iters 100] [--sgd STEP] [--images PIXELS]
"""
import argparse
import math

import torch

from paper_2204_08211_amd import binding as B


class Layout:
    """The layout of a model in its flat vector."""

    def __init__(self, shapes):
        self.at, offset = {}, 0
        for name, shape in shapes:
            self.at[name] = (offset, shape)
            offset += math.prod(shape)
        self.d = offset
        self.lengths = [math.prod(shape) for _, shape in shapes]
        self.matrices = [(o, *shape) for o, shape in self.at.values() if len(shape) == 2]
        self.vectors = torch.cat([torch.arange(o, o + shape[0]) for o, shape in self.at.values() if len(shape) == 1])

    def start(self, seed, device):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        w = torch.empty(self.d, device=device)
        for name, (o, shape) in self.at.items():
            part = self.part(w, name)
            if len(shape) == 2:
                part.copy_(torch.randn(shape, generator=gen, device=device) / math.sqrt(shape[1]))
            else:
                part.fill_(1.0 if name.startswith("weight") else 0.0)
        return w

    def part(self, flat, name):
        """A layer's part of the flat vector, or of every user's row."""
        o, shape = self.at[name]
        return flat[..., o:o + math.prod(shape)].unflatten(-1, shape) if len(shape) == 2 else flat[..., o:o + shape[0]]


class Network(Layout):
    """Both passes for all users at once."""

    def __init__(self, width, hidden, blocks, outputs):
        self.width, self.blocks = width, blocks
        shapes = []
        for k in range(blocks):
            shapes += [(f"weight{k}", (width,)), (f"bias{k}", (width,)), (f"up{k}", (hidden, width)), (f"down{k}", (width, hidden))]
        super().__init__(shapes + [("weight_out", (width,)), ("bias_out", (width,)), ("out", (outputs, width))])

    def forward(self, w, x):
        """Outputs for x [users, rows, width], and what the backward pass needs."""
        kept, h = [], x
        for k in range(self.blocks):
            n, mean, rstd = B.co3_layernorm(h, self.part(w, f"weight{k}"), self.part(w, f"bias{k}"))
            a = (n @ self.part(w, f"up{k}").t()).relu()
            kept.append((h, n, mean, rstd, a))
            h = h + a @ self.part(w, f"down{k}").t()
        n, mean, rstd = B.co3_layernorm(h, self.part(w, "weight_out"), self.part(w, "bias_out"))
        kept.append((h, n, mean, rstd, None))
        return n @ self.part(w, "out").t(), kept

    def backward(self, w, dy, kept, g):
        """Every user's gradient into its row of g."""
        h, n, mean, rstd, _ = kept[-1]
        self.part(g, "out").copy_(dy.mT.contiguous() @ n)
        dh = B.co3_layernorm_backward(dy @ self.part(w, "out"), h, self.part(w, "weight_out"), mean, rstd,
                                      dweight=self.part(g, "weight_out"), dbias=self.part(g, "bias_out"))
        for k in reversed(range(self.blocks)):
            h, n, mean, rstd, a = kept[k]
            self.part(g, f"down{k}").copy_(dh.mT.contiguous() @ a)
            da = (dh @ self.part(w, f"down{k}")) * (a > 0)
            self.part(g, f"up{k}").copy_(da.mT.contiguous() @ n)
            dh = dh + B.co3_layernorm_backward(da @ self.part(w, f"up{k}"), h, self.part(w, f"weight{k}"), mean, rstd,
                                               dweight=self.part(g, f"weight{k}"), dbias=self.part(g, f"bias{k}"))


class ImageNetwork(Layout):
    """The same for images of `pixels` pixels, rows / pixels of them a user, with group norms, products and what is kept in 8 bits."""

    def __init__(self, width, blocks, outputs, pixels, groups=8):
        self.width, self.blocks, self.pixels, self.groups = width, blocks, pixels, groups
        shapes = []
        for k in range(blocks):
            shapes += [(f"weight{k}", (width,)), (f"bias{k}", (width,)), (f"mix{k}", (width, width))]
        super().__init__(shapes + [("weight_out", (width,)), ("bias_out", (width,)), ("out", (outputs, width))])

    def _layer(self, w, h, name, matrix, kept, dtype):
        """matrix silu(group norm(h)) of h [users, rows, width]."""
        n, mean, rstd = B.co3_groupnorm(h.view(-1, self.pixels, self.width), self.groups, self.part(w, f"weight{name}"), self.part(w, f"bias{name}"),
                                        activation=B.ACT_SILU)
        n8, w8 = B.co3_quantize8(n.view(h.shape)), B.co3_quantize8(self.part(w, matrix))
        kept.append((B.co3_quantize8(h), n8, w8, mean, rstd))
        return B.co3_matmul8(n8, w8, dtype=dtype, transpose_b=True)

    def _layer_backward(self, w, dy, name, matrix, kept, g):
        """The gradient of h, and the layer's into every user's row of g."""
        h8, n8, w8, mean, rstd = kept
        dy8 = B.co3_quantize8(dy)
        B.co3_matmul8(dy8, n8, out=self.part(g, matrix), transpose_a=True)
        dn = B.co3_matmul8(dy8, w8)
        dh = B.co3_groupnorm_backward(dn.view(-1, self.pixels, self.width), h8, self.groups, self.part(w, f"weight{name}"), self.part(w, f"bias{name}"), mean, rstd,
                                      activation=B.ACT_SILU, users=dn.shape[0], dweight=self.part(g, f"weight{name}"), dbias=self.part(g, f"bias{name}"))
        return dh.view(dn.shape)

    def forward(self, w, x):
        kept, h = [], x.bfloat16()
        for k in range(self.blocks):
            h = h + self._layer(w, h, k, f"mix{k}", kept, torch.bfloat16)
        return self._layer(w, h, "_out", "out", kept, torch.float32), kept

    def backward(self, w, dy, kept, g):
        dh = self._layer_backward(w, dy, "_out", "out", kept[-1], g)
        for k in reversed(range(self.blocks)):
            dh = dh + self._layer_backward(w, dh, k, f"mix{k}", kept[k], g)


def train(net, users=4, rows=256, iters=100, eta=0.02, eta_vectors=0.5, gamma=0.7, refresh=10, sgd=None, E=4, M=3, seed=1, device="cuda:0"):
    """The mean squared error of every iteration, and the bits per element sent.  sgd: the step of plain updates, or None."""
    dev = torch.device(device)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    target, w = net.start(seed + 1, dev), net.start(seed + 2, dev)
    stride = (net.d + 31) // 32 * 32
    g, memory = torch.zeros((users, stride), device=dev), torch.zeros((users, stride), device=dev)
    average, momentum = torch.zeros(net.d, device=dev), torch.zeros(net.d, device=dev)
    plan = B.Plan(E, M, users, net.d, [[(1 << (E - 1)) - 1] * len(net.lengths)] * users, seg_len=net.lengths,
                  seg_book=list(range(len(net.lengths))))
    books = B.co3_build_codebook(E, M, plan.num_books, None)
    buf = B.RoundBuffers(plan, dev, max_code_len=64)
    muon = B.MatrixPlan(net.matrices, scales=[max(1.0, r / c) ** 0.5 for _, r, c in net.matrices])
    workspace = torch.empty(muon.workspace_bytes, dtype=torch.uint8, device=dev)
    vectors = net.vectors.to(dev)
    errors, bits = [], 0.0
    for t in range(iters):
        x = torch.randn((users, rows, net.width), generator=gen, device=dev) * (1 + torch.arange(users, device=dev)[:, None, None] / users)
        wanted, _ = net.forward(target, x)
        out, kept = net.forward(w, x)
        errors.append((out - wanted).square().mean())
        net.backward(w, (out - wanted) / rows, kept, g)
        if t % refresh == 0:                              # fit -> bias -> weights -> code, all on the device
            params = B.co3_gennorm_fit(plan, g, memory, gamma)
            B.co3_model_bias_device(plan, params, install=True)
            B.co3_build_codebook_device(books, B.co3_model_weights_device(plan, params), buf.status)
        B.co3_encode(plan, books, g, memory, memory, gamma, buf, mode=B.BOOK_FIXED, single_sweep=True)
        bits += float(buf.payload_bits.sum())
        if sgd is not None:
            B.co3_ps_aggregate(plan, books, buf, None, model=w, eta=sgd)
            continue
        B.co3_ps_aggregate(plan, books, buf, average)
        B.co3_muon_update(muon, average, momentum, w, eta=eta * (1 - t / iters), workspace=workspace, status=buf.status)
        w[vectors] -= eta_vectors * average[vectors] / net.matrices[-1][1]
    status = buf.status.cpu().numpy()
    assert status[B.STAT_NOCODE] == 0 and status[B.STAT_CORRUPT] == 0 and status[B.STAT_STALLED] == 0 and status[B.STAT_CAPACITY] == 0
    return torch.stack(errors).tolist(), bits / (iters * users * net.d)


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--users", type=int, default=4)
    p.add_argument("--rows", type=int, default=256)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=1024)
    p.add_argument("--outputs", type=int, default=64)
    p.add_argument("--blocks", type=int, default=3)
    p.add_argument("--iters", type=int, default=100)
    p.add_argument("--eta", type=float, default=0.02)
    p.add_argument("--sgd", type=float, default=None, help="plain updates of this step instead")
    p.add_argument("--images", type=int, default=None, help="images of so many pixels (a divisor of --rows), in 8 bits")
    a = p.parse_args()
    net = Network(a.width, a.hidden, a.blocks, a.outputs) if a.images is None else ImageNetwork(a.width, a.blocks, a.outputs, a.images)
    errors, bits = train(net, a.users, a.rows, a.iters, a.eta, sgd=a.sgd)
    print(f"U={a.users} d={net.d} {'orthogonalised updates' if a.sgd is None else 'plain updates'}: mean squared error "
          + ", ".join(f"{errors[t]:.4f} at {t}" for t in sorted({0, a.iters // 4, a.iters // 2, a.iters - 1})) + f"; {bits:.3f} bit/element")


if __name__ == "__main__":
    main()
