"""Trains one layer norm + linear layer whose parameters live in the compressed store, with products at four bits.

Every round: the weight matrix is decompressed (omc_decompress) and quantised along both of its axes
(omc_mx_quantise); forward: layer norm, quantisation of its output along features and frames, product; backward: the
incoming gradient quantised along both axes, the two products, layer norm backward.  The gradients of the matrix, the gain and
the bias are written straight into the store's gradient arena, and omc_update_recompress applies them.  A single
frame then goes through omc_mx_linear, as a streaming recogniser would send it.

    python examples/layer_training_step.py [--rounds 40]

torch holds the buffers and computes the loss; every operation of the layer is the library's.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2205_03494_b200 as omc

EPS = 1e-5


class Layer:
    """y = layer_norm(x) W^T with W (width_out x width_in), gain and bias in the store; x and y are BF16."""

    def __init__(self, width_in, width_out, frames, fmt=(5, 10), seed=0):
        self.k, self.n, self.m = width_in, width_out, frames
        dev = "cuda"
        g = torch.Generator(device=dev).manual_seed(seed)
        # variables: the matrix (quantised), gain and bias of the norm (FP32, as norm parameters always are)
        self.plan = omc.Plan([self.n * self.k, self.k, self.k], [omc.KIND_WEIGHT_MATRIX, omc.KIND_NORM, omc.KIND_NORM], fmt)
        p = self.plan
        new = lambda n, dtype: torch.zeros(max(int(n), 16), dtype=dtype, device=dev)
        self.packed, self.resid = new(p.packed_bytes, torch.uint8), new(p.resid_elems, torch.float32)
        self.sb, self.space = new(2 * p.n_quantised, torch.float32), new(p.workspace_bytes, torch.uint8)
        self.full, self.grads = new(p.full_elems, torch.float32), new(p.full_elems, torch.float32)
        p.prepare(self.space.data_ptr(), self.stream)
        lim = (6.0 / (self.n + self.k)) ** 0.5
        self.view(self.full, 0).uniform_(-lim, lim, generator=g)
        self.view(self.full, 1).fill_(1.0)
        p.compress(self.full.data_ptr(), self.packed.data_ptr(), self.resid.data_ptr(), self.sb.data_ptr(), self.space.data_ptr(), self.stream)
        # quantised matrices: W along its columns (forward) and rows (backward), the layer's input and the gradient likewise
        pair = lambda r, c: [new(n, torch.uint8) for n in omc.mx_sizes(r, c)]
        self.w, self.wt = pair(self.n, self.k), pair(self.k, self.n)
        self.a, self.at = pair(self.m, self.k), pair(self.k, self.m)
        self.g, self.gt = pair(self.m, self.n), pair(self.n, self.m)
        b16 = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)
        self.normed, self.y, self.dnormed, self.dx = b16(self.m, self.k), b16(self.m, self.n), b16(self.m, self.k), b16(self.m, self.k)
        self.mean, self.rstd = new(self.m, torch.float32), new(self.m, torch.float32)
        self.norm_space = new(omc.layer_norm_workspace_bytes(self.m, self.k), torch.uint8)
        self.frame_space = new(sum(omc.mx_sizes(1, self.k)), torch.uint8)
        self.status = new(1, torch.int32)

    @property
    def stream(self):
        return torch.cuda.current_stream().cuda_stream

    def view(self, arena, i):
        return arena[self.plan.full_off[i]:self.plan.full_off[i] + self.plan.numel[i]]

    def load(self):
        """The current weights: decompressed from the store, the matrix quantised along both axes."""
        p, st = self.plan, self.stream
        p.decompress(self.packed.data_ptr(), self.resid.data_ptr(), self.sb.data_ptr(), self.full.data_ptr(), stream=st)
        omc.mx_quantise(self.view(self.full, 0).data_ptr(), omc.F32, self.n, self.k, self.k, *[t.data_ptr() for t in self.w + self.wt], stream=st)

    def norm(self, x, out, rows, mean=0, rstd=0):
        omc.layer_norm(x.data_ptr(), omc.BF16, rows, self.k, self.k, self.view(self.full, 1).data_ptr(), self.view(self.full, 2).data_ptr(), EPS,
                       out.data_ptr(), self.k, mean, rstd, stream=self.stream)

    def forward(self, x):
        m, n, k, st = self.m, self.n, self.k, self.stream
        self.norm(x, self.normed, m, self.mean.data_ptr(), self.rstd.data_ptr())
        omc.mx_quantise(self.normed.data_ptr(), omc.BF16, m, k, k, *[t.data_ptr() for t in self.a + self.at], stream=st)
        omc.mx_matmul(self.a[0].data_ptr(), self.a[1].data_ptr(), m, self.w[0].data_ptr(), self.w[1].data_ptr(), n, k, self.y.data_ptr(), omc.BF16, n,
                      self.status.data_ptr(), stream=st)
        return self.y

    def backward(self, x, dy):
        """dx; the gradients of matrix, gain and bias go to the arena."""
        m, n, k, st = self.m, self.n, self.k, self.stream
        omc.mx_quantise(dy.data_ptr(), omc.BF16, m, n, n, *[t.data_ptr() for t in self.g + self.gt], stream=st)
        omc.mx_matmul(self.g[0].data_ptr(), self.g[1].data_ptr(), m, self.wt[0].data_ptr(), self.wt[1].data_ptr(), k, n, self.dnormed.data_ptr(),
                      omc.BF16, k, self.status.data_ptr(), stream=st)
        omc.mx_matmul(self.gt[0].data_ptr(), self.gt[1].data_ptr(), n, self.at[0].data_ptr(), self.at[1].data_ptr(), k, m,
                      self.view(self.grads, 0).data_ptr(), omc.F32, k, self.status.data_ptr(), stream=st)
        omc.layer_norm_backward(self.dnormed.data_ptr(), k, x.data_ptr(), k, omc.BF16, m, k, self.view(self.full, 1).data_ptr(), self.mean.data_ptr(),
                                self.rstd.data_ptr(), self.dx.data_ptr(), k, self.view(self.grads, 1).data_ptr(), self.view(self.grads, 2).data_ptr(),
                                self.norm_space.data_ptr(), stream=st)
        return self.dx

    def update(self, lr):
        self.plan.update_recompress(self.packed.data_ptr(), self.resid.data_ptr(), self.sb.data_ptr(), self.grads.data_ptr(), lr, self.space.data_ptr(),
                                    stream=self.stream)

    def frame(self, x):
        """One frame (1 x width_in) without keeping anything for a backward pass."""
        normed, y = torch.empty_like(x), torch.empty(1, self.n, dtype=torch.bfloat16, device=x.device)
        self.norm(x, normed, 1)
        omc.mx_linear(normed.data_ptr(), omc.BF16, 1, self.k, self.k, self.w[0].data_ptr(), self.w[1].data_ptr(), self.n, y.data_ptr(), omc.BF16,
                      self.n, self.frame_space.data_ptr(), self.status.data_ptr(), stream=self.stream)
        return y


def train(rounds=40, frames=1500, width_in=512, width_out=512, lr=0.25, seed=0):
    """Fits the layer to a random linear map of normalised features; returns (losses, layer, inputs)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(frames, width_in, generator=g, device="cuda") * 2 + 0.5).to(torch.bfloat16)
    want = torch.nn.functional.layer_norm(x.float(), (width_in,)) @ (torch.randn(width_in, width_out, generator=g, device="cuda") / width_in ** 0.5)
    layer = Layer(width_in, width_out, frames, seed=seed)
    losses = []
    for _ in range(rounds):
        layer.load()
        diff = layer.forward(x).float() - want
        losses.append(diff.square().mean().item())
        layer.backward(x, (diff * (2.0 / frames)).to(torch.bfloat16))
        layer.update(lr)
    return losses, layer, x


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=40)
    losses, layer, x = train(ap.parse_args().rounds)
    for i in range(0, len(losses), max(1, len(losses) // 8)):
        print("round %3d  loss %.4f" % (i, losses[i]))
    print("last      loss %.4f" % losses[-1])
    layer.load()
    batch, one = layer.forward(x)[3], layer.frame(x[3:4])[0]
    print("one frame alone equals the same frame in the batch:", bool(torch.equal(batch, one)))
    print("status word:", int(layer.status[0]))
