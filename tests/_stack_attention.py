"""The routed-expert stack with an attention block in front of every layer: per layer the block over the layer's
8-bit cache (h += attention, x normalised again), then route + forward, h += out."""
from __future__ import annotations

from _stack import Stack


class AttentionStack(Stack):
    """blocks: one AttentionBlock a layer."""

    def __init__(self, *args, block, **kw):
        super().__init__(*args, **kw)
        self.blocks = [block(l) for l in range(self.L)]

    def step(self, x0, seqs, mass_rows=0, before=None, after=None):
        """One pass of the rows x0 [n, d] of the sequences; before(l) and after(l) surround every attention block."""
        import torch
        import paper_2608_23805_amd as msi
        n = x0.shape[0]
        cs, side = torch.cuda.current_stream(), torch.cuda.Stream()
        h, x, out = self.h[:n], self.x[:n], self.out[:n]
        r = msi.Routing.alloc(n, self.s.K, self.s.E)
        msi.residual_init(x0, h, x, cs)
        for l in range(self.L):
            if before:
                before(l)
            self.blocks[l].reserve(seqs, mass_rows)
            self.blocks[l].step(x, h, seqs, mass_rows=mass_rows, stream=cs)
            if after:
                after(l)
            self.plan.route(x, self.wr[l], self.bias[l], r, self.ws, cs)
            self.plan.forward(l, x, r, self.shared[l], out, self.ws, cs, side)
            msi.residual_add(out, h, x, cs)
        return h, x
