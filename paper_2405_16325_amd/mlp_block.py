"""Stacks of pre-norm blocks of double-pruned layers, trained with AdamW and served, by the library's calls; the loss, and the
first stack's relu with its gradient, are torch's.

    block:  h <- h + W2 norm2(relu(W1 norm1(h)))          W1, W2: packed 2:4 (W^R forward, W^{R,C} backward)
    gated block:  h <- h + W2 (act(g) u),  [g | u] = W1 norm1(h)
    out  =  norm(h)

Training: every norm adds the stream's last contribution itself (slope_rmsnorm_fwd with a residual) and its gradient carries the
stream's along (slope_rmsnorm_bwd with dh); the packed gradients go to AdamW as they are, with fp32 masters and 32- or 8-bit
states; slope_update_sparse brings the transposed copies in line.  The host waits for nothing in a step.
Serving: the norms write 8 bits with a scale per token, the products read them, the second one adds the stream.
The gated stack keeps 8-bit codes of what its layers' gradients want, the input and the projections (33/32 bytes an element); the layer's
output is made again from them (slope_gated_bwd).  It serves in bf16, activation and product inside the first product.

`python -m paper_2405_16325_amd.mlp_block` trains a small one of each on a random teacher and compares the paths.
"""
from __future__ import annotations

import torch

from . import binding as sl

BF16, EPS = torch.bfloat16, 1e-5


class SparseLayer:
    """A d_out x d_in weight pruned 2:4, both packed copies, its fp32 master and its gradient, all in place for good."""

    def __init__(self, d_out, d_in, generator):
        dense = torch.randn(d_out, d_in, generator=generator, device="cuda") * d_in ** -0.5
        self.vals, self.meta, _ = sl.slope_prune_rows(dense.to(BF16))
        self.vals_t, self.meta_t, _ = sl.slope_double_prune(self.vals, self.meta)
        self.master, self.grad = self.vals.float(), torch.zeros_like(self.vals)
        self.q = None

    def forward(self, x):
        return sl.slope_spmm_fwd(x, self.vals, self.meta)

    def backward(self, dy, x):
        sl.slope_wgrad_masked(dy, x, self.meta, out=self.grad)
        return sl.slope_spmm_bwd_x(dy, self.vals_t, self.meta_t)

    def updated(self):
        sl.slope_update_sparse(self.vals, self.meta, self.vals, self.meta_t, self.vals_t)
        self.q = None

    def serve(self, q, scale, add=None):
        if self.q is None:
            self.q = sl.slope_quantize_packed(self.vals)
        return sl.slope_spmm_fwd_q8(q, scale, self.q[0], self.meta, self.q[1], add=add)


class GatedLayer(SparseLayer):
    """act(g) u of the projections g, u of one weight of 2 d_ff rows, the gate's first."""

    def __init__(self, d_ff, d_in, generator, act=sl.SLOPE_ACT_SILU):
        super().__init__(2 * d_ff, d_in, generator)
        self.act = act

    def forward(self, x):
        """(output, what backward wants)"""
        h, _, codes, scale = sl.slope_gated_fwd(x, self.vals, self.meta, self.act, want_q8=True)
        return h, (sl.slope_checkpoint_q8(x), codes, scale)

    def output(self, dh, saved):
        """(gradient of the projections, the output again)"""
        return sl.slope_gated_bwd(dh, self.act, q8=saved[1], scale=saved[2])

    def backward(self, dgu, saved):
        sl.slope_wgrad_masked_q8(dgu, *saved[0], self.meta, out=self.grad)
        return sl.slope_spmm_bwd_x(dgu, self.vals_t, self.meta_t)

    def serve(self, x):
        return sl.slope_gated_fwd(x, self.vals, self.meta, self.act)[0]


class Norm:
    def __init__(self, d):
        self.w, self.master = torch.ones(d, dtype=BF16, device="cuda"), torch.ones(d, device="cuda")
        self.grad = torch.zeros_like(self.w)

    def forward(self, x, residual=None):
        """(y, the stream, what the gradient wants)"""
        y, h, rstd, _, _ = sl.slope_rmsnorm_fwd(x, self.w, EPS, residual=residual, want_rstd=True)
        h = x if residual is None else h
        return y, h, (h, rstd)

    def backward(self, dy, saved, dh=None):
        return sl.slope_rmsnorm_bwd(dy, saved[0], self.w, saved[1], dh=dh, out=(torch.empty_like(dy), self.grad))[0]

    def serve(self, x):
        return sl.slope_rmsnorm_fwd(x, self.w, EPS, want_y=False, want_q8=True)[3:]


class PrenormMLP:
    def __init__(self, d, hidden, blocks, state_bits=8, weight_decay=0.0, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.blocks = [self.block(d, hidden, gen) for _ in range(blocks)]
        self.out = Norm(d)
        self.layers = [x for b in self.blocks for x in b if isinstance(x, SparseLayer)]
        norms = [x for b in self.blocks for x in b if isinstance(x, Norm)] + [self.out]
        parts = self.layers + norms
        params = [x.vals for x in self.layers] + [x.w for x in norms]
        scales = (None, None)
        if state_bits == 8:
            moments = [[torch.zeros(p.shape, dtype=torch.uint8, device="cuda").view(sl.E4M3) for p in params] for _ in range(2)]
            scales = [[torch.zeros((p.numel() + sl.SLOPE_ADAMW_BLOCK - 1) // sl.SLOPE_ADAMW_BLOCK, device="cuda") for p in params]
                      for _ in range(2)]
        else:
            moments = [[torch.zeros(p.shape, device="cuda") for p in params] for _ in range(2)]
        self.plan = sl.slope_adamw_plan(params, [x.grad for x in parts], *moments, masters=[x.master for x in parts],
                                        m_scales=scales[0], v_scales=scales[1],
                                        weight_decay=[weight_decay] * len(self.layers) + [0.0] * len(norms))
        self.control = torch.zeros(4, device="cuda")

    def block(self, d, hidden, gen):
        return Norm(d), SparseLayer(hidden, d, gen), Norm(hidden), SparseLayer(d, hidden, gen)

    def forward(self, x):
        """x bf16[b, d] -> (out, what backward wants)"""
        saved, part, h = [], x, None
        for norm1, up, norm2, down in self.blocks:
            y, h, s1 = norm1.forward(part, residual=h)
            a = up.forward(y)
            r = torch.relu(a)
            n, _, s2 = norm2.forward(r)
            part = down.forward(n)
            saved.append((y, s1, a, n, s2))
        out, _, s = self.out.forward(part, residual=h)
        return out, (saved, s)

    def backward(self, dout, kept):
        saved, s = kept
        dh = self.out.backward(dout, s)
        for (norm1, up, norm2, down), (y, s1, a, n, s2) in zip(reversed(self.blocks), reversed(saved)):
            da = norm2.backward(down.backward(dh, n), s2) * (a > 0)
            dh = norm1.backward(up.backward(da, y), s1, dh=dh)
        return dh

    def step(self, lr, loss_scale=1.0, max_norm=1.0, betas=(0.9, 0.95)):
        """Clips, leaves the step out if a gradient is not finite, updates every tensor and both packed copies."""
        sl.slope_grad_norm(self.plan, self.control, 1.0 / loss_scale, max_norm)
        sl.slope_adamw_step(self.plan, lr, betas[0], betas[1], 1e-8, control=self.control)
        for layer in self.layers:
            layer.updated()

    def serve(self, x):
        """The forward in 8 bits, for inference."""
        h = x
        for norm1, up, norm2, down in self.blocks:
            r = torch.relu_(up.serve(*norm1.serve(h)))
            h = down.serve(*norm2.serve(r), add=h)
        return sl.slope_rmsnorm_fwd(h, self.out.w, EPS)[0]


class PrenormGatedMLP(PrenormMLP):
    def __init__(self, d, hidden, blocks, act=sl.SLOPE_ACT_SILU, **kw):
        self.act = act
        super().__init__(d, hidden, blocks, **kw)

    def block(self, d, hidden, gen):
        return Norm(d), GatedLayer(hidden, d, gen, self.act), SparseLayer(d, hidden, gen)

    def forward(self, x):
        saved, part, h = [], x, None
        for norm, gated, down in self.blocks:
            y, h, s = norm.forward(part, residual=h)
            a, kept = gated.forward(y)
            part = down.forward(a)
            saved.append((s, kept))
        out, _, s = self.out.forward(part, residual=h)
        return out, (saved, s)

    def backward(self, dout, kept):
        saved, s = kept
        dh = self.out.backward(dout, s)
        for (norm, gated, down), (s, codes) in zip(reversed(self.blocks), reversed(saved)):
            dgu, a = gated.output(sl.slope_spmm_bwd_x(dh, down.vals_t, down.meta_t), codes)
            sl.slope_wgrad_masked(dh, a, down.meta, out=down.grad)
            dh = norm.backward(gated.backward(dgu, codes), s, dh=dh)
        return dh

    def serve(self, x):
        part, h = x, None
        for norm, gated, down in self.blocks:
            y, h, _ = norm.forward(part, residual=h)
            part = down.forward(gated.serve(y))
        return self.out.forward(part, residual=h)[0]


def train(model, d, steps=150, b=512, lr=3e-3, loss_scale=1024.0, seed=1):
    """Mean squared errors, first and last, against a random smooth teacher."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    teacher = torch.randn(d, d, generator=gen, device="cuda") * d ** -0.5
    losses = []
    for _ in range(steps):
        x = torch.randn(b, d, generator=gen, device="cuda")
        want = torch.tanh(x @ teacher) * 1.5
        out, kept = model.forward(x.to(BF16))
        diff = out.float() - want
        losses.append(diff.square().mean())
        model.backward((diff * (2 * loss_scale / diff.numel())).to(BF16), kept)
        model.step(lr, loss_scale)
    return float(losses[0]), float(torch.stack(losses[-10:]).mean())


def main():
    for bits in (32, 8):
        model = PrenormMLP(256, 512, 2, state_bits=bits)
        first, last = train(model, 256)
        x = torch.randn(64, 256, device="cuda").to(BF16)
        out, served = model.forward(x)[0].float(), model.serve(x).float()
        print("%2d-bit states: loss %.3f -> %.3f; 8-bit serving differs by %.3f of the output's norm; %d steps taken"
              % (bits, first, last, float((out - served).norm() / out.norm()), int(model.control[2])))
    model = PrenormGatedMLP(256, 512, 2)
    first, last = train(model, 256)
    x = torch.randn(1, 256, device="cuda").to(BF16)
    same = torch.equal(model.forward(x)[0], model.serve(x))
    print("gated, activations kept in 8 bits: loss %.3f -> %.3f; one token served as in training: %s" % (first, last, same))


if __name__ == "__main__":
    main()
