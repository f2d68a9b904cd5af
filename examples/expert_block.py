"""A sparse network with an expert block between its convolutions, trained for a few steps and then
asked for one row at a time.

    python examples/expert_block.py [--sites 29760] [--steps 30] [--dtype bf16]

The network takes pen strokes on 64 x 64 grids: a VSC 3 x 3 layer, the expert block on the rows of
its active sites, and a VSC 1 x 1 layer to two planes, which are to tell the local direction of the
stroke (the sums of the neighbours' offsets).  The block is

    n = layer_norm(x);  e, p = the k largest of n W_r, their softmax
    y = x + dropout(sum over the k experts of p (relu(n W1[e] + b1[e]) W2[e] + b2[e]))

Every product, norm, routing and gradient runs in the library's kernels; torch holds the tensors and
applies the updates.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1706_01307_amd as spc  # noqa: E402
from paper_1706_01307_amd import inputs  # noqa: E402


class ExpertBlock:
    """Layer norm, routing, two grouped products, combine and dropout on [n, C] rows."""

    def __init__(self, C, hidden, experts, k, p=0.1, dtype=torch.float32, seed=0, normalize=True):
        g = torch.Generator().manual_seed(seed)

        def r(*shape, std):
            return (torch.randn(*shape, generator=g) * std).cuda()
        self.k, self.p, self.seed, self.normalize = k, p, seed, normalize
        # fp32 parameters; the products take them in the rows' dtype
        self.params = {"gamma": torch.ones(C).cuda(), "beta": torch.zeros(C).cuda(),
                       "wr": r(1, C, experts, std=1 / math.sqrt(C)),
                       "w1": r(experts, C, hidden, std=math.sqrt(2 / C)),
                       "b1": torch.zeros(experts, hidden).cuda(),
                       "w2": r(experts, hidden, C, std=1 / math.sqrt(hidden)),
                       "b2": torch.zeros(experts, C).cuda()}
        self.dtype = dtype

    def _w(self, name):
        return self.params[name].to(self.dtype)

    def serve(self):
        """Keep the products' weights in the rows' dtype from now on, converted once."""
        for name in ("wr", "w1", "w2"):
            self.params[name] = self._w(name)

    def forward(self, x, step, train=True):
        """The block's output and what its gradient needs; `step` numbers the dropped elements."""
        q = self.params
        n, mean, rstd = spc.layer_norm_forward(x, q["gamma"], q["beta"], stats=train)
        # the router's product: one group of all rows
        # (offsets made on the device: nothing here waits for the host, or keeps a graph from
        # being captured)
        one = torch.arange(2, dtype=torch.int32, device=x.device) * x.shape[0]
        logits = spc.grouped_forward(n, self._w("wr"), one, out_dtype=torch.float32)
        r = spc.route_forward(logits, self.k, self.normalize)
        h = spc.grouped_forward(n, self._w("w1"), r.offsets, rows=r.rows, bias=q["b1"], relu=True)
        z = spc.grouped_forward(h, self._w("w2"), r.offsets, bias=q["b2"])
        if not train:
            return spc.combine_forward(z, r.pos, r.weights, residual=x), None
        u = spc.combine_forward(z, r.pos, r.weights)
        y = spc.dropout_forward(u, self.p, self.seed, step, residual=x)
        return y, (x, step, n, mean, rstd, one, logits, r, h, z)

    def backward(self, dy, kept):
        """(dx, gradients of the parameters)."""
        x, step, n, mean, rstd, one, logits, r, h, z = kept
        q, g = self.params, {}
        du = spc.dropout_backward(dy, self.p, self.seed, step)
        dz, dp = spc.combine_backward(du, z, r.pos, r.weights, offsets=r.offsets)
        g["w2"], g["b2"] = spc.grouped_backward_weight(h, dz, r.offsets)
        dh = spc.grouped_backward_data(dz, self._w("w2"), r.offsets, mask=h)
        g["w1"], g["b1"] = spc.grouped_backward_weight(n, dh, r.offsets, rows=r.rows)
        dl = spc.route_backward(dp, logits, r.experts, r.weights, self.normalize).to(self.dtype)
        g["wr"], _ = spc.grouped_backward_weight(n, dl, one, bias=False)
        # a row's gradient: through the router, and the sum of its k positions'
        dn = spc.grouped_backward_data(dl, self._w("wr"), one)
        dn = spc.combine_forward(spc.grouped_backward_data(dh, self._w("w1"), r.offsets), r.pos,
                                 residual=dn)
        dx, g["gamma"], g["beta"] = spc.layer_norm_backward(dn, x, mean, rstd, q["gamma"])
        return dx.add_(dy), g


def _strokes(sites):
    """Coordinates of pen strokes and, per site, the direction its neighbours lie in."""
    grids = max(1, sites // 465)
    coords = torch.from_numpy(inputs.pen_strokes(grids, 64, seed=3, target=465))
    size = [grids, 64, 64]
    lit = torch.zeros(size)
    lit[tuple(coords.long().T)] = 1.0
    kernel = torch.zeros(2, 1, 3, 3)
    for a in range(3):
        for b in range(3):
            kernel[0, 0, a, b], kernel[1, 0, a, b] = a - 1, b - 1
    field = torch.nn.functional.conv2d(lit[:, None], kernel, padding=1)
    target = field.permute(0, 2, 3, 1)[tuple(coords.long().T)]
    return coords.cuda(), size, target.cuda()


def train(sites=29760, steps=30, dtype=torch.float32, C=64, hidden=128, experts=8, k=2, lr=0.01):
    """The losses, the block and the rows it was trained on."""
    coords, size, target = _strokes(sites)
    book = spc.build_rulebook(spc.VSC, coords, size, [1, 3, 3])
    last = spc.build_rulebook(spc.VSC, coords, size, [1, 1, 1])
    n = coords.shape[0]
    g = torch.Generator().manual_seed(1)
    first = (torch.randn(9, 1, C, generator=g) / 3).cuda()
    head = (torch.randn(1, C, 2, generator=g) / math.sqrt(C)).cuda()
    block = ExpertBlock(C, hidden, experts, k, dtype=dtype)
    ones = torch.ones(n, 1, dtype=dtype, device="cuda")
    losses, x = [], None
    for step in range(steps):
        w0, w1 = first.to(dtype), head.to(dtype)
        x = spc.vsc_forward(book, ones, w0)
        y, kept = block.forward(x, step)
        out = spc.vsc_forward(last, y, w1, out_dtype=torch.float32)
        err = out - target
        losses.append(float((err * err).mean()))
        dout = (err * (2.0 / err.numel() * 1e3)).to(dtype)         # (scaled for bf16)
        dhead, _ = spc.backward_weight(last, spc.OP_VSC, y, dout, C, 2, bias=False)
        dy = spc.backward_data(last, spc.OP_VSC, dout, w1)
        dx, grads = block.backward(dy, kept)
        dfirst, _ = spc.backward_weight(book, spc.OP_VSC, ones, dx, 1, C, bias=False)
        for p, d in [(first, dfirst), (head, dhead)] + [(block.params[q], d)
                                                        for q, d in grads.items()]:
            p.add_(d, alpha=-lr * 1e-3)
    return losses, block, x


def main():
    parser = argparse.ArgumentParser()
    parser.add_argument("--sites", type=int, default=29760)
    parser.add_argument("--steps", type=int, default=30)
    parser.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    a = parser.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    losses, block, x = train(a.sites, a.steps, dtype)
    print("loss: " + " ".join("%.4f" % v for v in losses[::max(1, a.steps // 10)]))
    # one row at a time: its k experts alone are read (and no weights converted)
    block.serve()
    whole, _ = block.forward(x, 0, train=False)
    for i in range(3):
        y, _ = block.forward(x[i:i + 1], 0, train=False)
        print("row %d alone differs from its batch by %.2g" %
              (i, float((y.float() - whole[i:i + 1].float()).abs().max())))


if __name__ == "__main__":
    main()
