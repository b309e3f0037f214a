"""Trains a gated feed-forward block whose matrices live in the compressed store, with its products in 8-bit integers.

    h = silu(x Wg^T) * (x Wv^T),   y = h Wo^T
The store holds W = (Wg; Wv), 2 F x K, and Wo, N x F.  Every round decompresses them (omc_decompress) and quantises both along both of their axes
(omc_byte_quantise); forward: x quantised along features and frames, both projections with the gate in one product (omc_byte_gated), h quantised both
ways, the output product; backward: the incoming gradient quantised both ways, the two products of the output projection, the gate's gradients made and
quantised in one call (omc_gated_backward), the two products of the gated layer.  The matrices' gradients are written straight into the store's
gradient arena, and omc_update_recompress applies them.  A single frame goes through omc_byte_gated_linear and omc_byte_linear.

    python examples/gated_training_step.py [--rounds 30]

torch holds the buffers and computes the loss; every operation of the block is the library's.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2205_03494_b200 as omc


class Block:
    """y = (silu(x Wg^T) * (x Wv^T)) Wo^T; activations are BF16."""

    def __init__(self, width_in, width, width_out, frames, fmt=(5, 10), activation=omc.GATE_SILU, seed=0):
        self.k, self.f, self.n, self.m, self.activation = width_in, width, width_out, frames, activation
        dev = "cuda"
        g = torch.Generator(device=dev).manual_seed(seed)
        k, f, n, m = self.k, self.f, self.n, self.m
        self.plan = omc.Plan([2 * f * k, n * f], [omc.KIND_WEIGHT_MATRIX, omc.KIND_WEIGHT_MATRIX], fmt)
        p = self.plan
        new = lambda count, dtype: torch.zeros(max(int(count), 16), dtype=dtype, device=dev)
        self.packed, self.resid = new(p.packed_bytes, torch.uint8), new(p.resid_elems, torch.float32)
        self.sb, self.space = new(2 * p.n_quantised, torch.float32), new(p.workspace_bytes, torch.uint8)
        self.full, self.grads = new(p.full_elems, torch.float32), new(p.full_elems, torch.float32)
        p.prepare(self.space.data_ptr(), self.stream)
        for i, fan_in in enumerate((k, f)):
            self.view(self.full, i).normal_(0.0, fan_in ** -0.5, generator=g)
        p.compress(self.full.data_ptr(), self.packed.data_ptr(), self.resid.data_ptr(), self.sb.data_ptr(), self.space.data_ptr(), self.stream)
        both = lambda r, c: [[new(b, torch.uint8) for b in omc.byte_sizes(*s)] for s in ((r, c), (c, r))]
        self.w, self.wo, self.x, self.h, self.dy, self.dpre = both(2 * f, k), both(n, f), both(m, k), both(m, f), both(m, n), both(m, 2 * f)
        shapes = ((2 * f, k), (n, f), (m, k), (m, f), (m, n))
        self.scratch = new(max([omc.byte_quantise_workspace_bytes(*s) for s in shapes] + [omc.gated_backward_workspace_bytes(m, f)]), torch.uint8)
        b16 = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)
        self.pre, self.hidden, self.y, self.dhidden, self.dx = b16(m, 2 * f), b16(m, f), b16(m, n), b16(m, f), b16(m, k)
        self.frame_space = new(max(sum(omc.byte_sizes(1, k)), sum(omc.byte_sizes(1, f))), torch.uint8)
        self.status = new(1, torch.int32)

    @property
    def stream(self):
        return torch.cuda.current_stream().cuda_stream

    def view(self, arena, i):
        return arena[self.plan.full_off[i]:self.plan.full_off[i] + self.plan.numel[i]]

    def quantise(self, t, dtype, rows, cols, into):
        """t along its rows and its columns."""
        omc.byte_quantise(t.data_ptr(), dtype, rows, cols, cols, *[b.data_ptr() for pair in into for b in pair], self.scratch.data_ptr(), stream=self.stream)

    def product(self, a, rows, b, cols, k, out, dtype):
        omc.byte_matmul(a[0].data_ptr(), a[1].data_ptr(), rows, b[0].data_ptr(), b[1].data_ptr(), cols, k, out.data_ptr(), dtype, cols, self.status.data_ptr(),
                        stream=self.stream)

    def load(self):
        """The current weights: decompressed from the store, both matrices quantised along both axes."""
        self.plan.decompress(self.packed.data_ptr(), self.resid.data_ptr(), self.sb.data_ptr(), self.full.data_ptr(), stream=self.stream)
        self.quantise(self.view(self.full, 0), omc.F32, 2 * self.f, self.k, self.w)
        self.quantise(self.view(self.full, 1), omc.F32, self.n, self.f, self.wo)

    def forward(self, x):
        m, f, k, n = self.m, self.f, self.k, self.n
        self.quantise(x, omc.BF16, m, k, self.x)
        omc.byte_gated(*[b.data_ptr() for b in self.x[0]], m, *[b.data_ptr() for b in self.w[0]], f, k, self.activation, self.hidden.data_ptr(), omc.BF16, f,
                       self.pre.data_ptr(), 2 * f, self.status.data_ptr(), stream=self.stream)
        self.quantise(self.hidden, omc.BF16, m, f, self.h)
        self.product(self.h[0], m, self.wo[0], n, f, self.y, omc.BF16)
        return self.y

    def backward(self, dy):
        """dx; the gradients of both matrices go to the arena."""
        m, f, k, n = self.m, self.f, self.k, self.n
        self.quantise(dy, omc.BF16, m, n, self.dy)
        self.product(self.dy[0], m, self.wo[1], f, n, self.dhidden, omc.BF16)
        self.product(self.dy[1], n, self.h[1], f, m, self.view(self.grads, 1), omc.F32)
        omc.gated_backward(self.dhidden.data_ptr(), f, self.pre.data_ptr(), 2 * f, omc.BF16, m, f, self.activation, 0, 0,
                           *[b.data_ptr() for pair in self.dpre for b in pair], self.scratch.data_ptr(), stream=self.stream)
        self.product(self.dpre[0], m, self.w[1], k, 2 * f, self.dx, omc.BF16)
        self.product(self.dpre[1], 2 * f, self.x[1], k, m, self.view(self.grads, 0), omc.F32)
        return self.dx

    def update(self, lr):
        self.plan.update_recompress(self.packed.data_ptr(), self.resid.data_ptr(), self.sb.data_ptr(), self.grads.data_ptr(), lr, self.space.data_ptr(),
                                    stream=self.stream)

    def frame(self, x):
        """One frame (1 x width_in) without keeping anything for a backward pass."""
        h, y = (torch.empty(1, c, dtype=torch.bfloat16, device=x.device) for c in (self.f, self.n))
        omc.byte_gated_linear(x.data_ptr(), omc.BF16, 1, self.k, self.k, *[b.data_ptr() for b in self.w[0]], self.f, self.activation, h.data_ptr(), omc.BF16, self.f,
                              0, 0, self.frame_space.data_ptr(), self.status.data_ptr(), stream=self.stream)
        omc.byte_linear(h.data_ptr(), omc.BF16, 1, self.f, self.f, *[b.data_ptr() for b in self.wo[0]], self.n, y.data_ptr(), omc.BF16, self.n,
                        self.frame_space.data_ptr(), self.status.data_ptr(), stream=self.stream)
        return y


def train(rounds=30, frames=1500, width_in=512, width=1024, width_out=512, lr=0.01, seed=0):
    """Fits the block to another block's outputs; returns (losses, block, inputs)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = new(frames, width_in).to(torch.bfloat16)
    gate, value, out = new(width_in, width) / width_in ** 0.5, new(width_in, width) / width_in ** 0.5, new(width, width_out) / width ** 0.5
    want = (torch.nn.functional.silu(x.float() @ gate) * (x.float() @ value)) @ out
    block = Block(width_in, width, width_out, frames, seed=seed)
    losses = []
    for _ in range(rounds):
        block.load()
        diff = block.forward(x).float() - want
        losses.append(diff.square().mean().item())
        block.backward((diff * (2.0 / frames)).to(torch.bfloat16))
        block.update(lr)
    return losses, block, x


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=30)
    losses, block, x = train(ap.parse_args().rounds)
    for i in range(0, len(losses), max(1, len(losses) // 8)):
        print("round %3d  loss %.4f" % (i, losses[i]))
    print("last      loss %.4f" % losses[-1])
    block.load()
    batch, one = block.forward(x)[3], block.frame(x[3:4])[0]
    print("one frame alone equals the same frame in the batch:", bool(torch.equal(batch, one)))
    print("status word:", int(block.status[0]))
