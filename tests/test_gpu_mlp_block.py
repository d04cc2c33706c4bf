"""The stack of pre-norm blocks: its gradients against the same function in fp64 by torch's autograd on the CPU, training with both
kinds of optimizer state, and serving in 8 bits."""
import pytest
import torch

from paper_2405_16325_amd import binding as sl
from paper_2405_16325_amd import mlp_block as mb

pytestmark = pytest.mark.gpu


def dense(vals, meta):
    """Packed values as a dense fp64 weight, on the CPU."""
    vals, meta = vals.double().cpu(), meta.cpu().long()
    w = torch.zeros(vals.shape[0], 2 * vals.shape[1], dtype=torch.float64)
    for slot in range(4):
        col = 8 * torch.arange(meta.shape[1]) + 4 * (slot // 2) + ((meta >> (2 * slot)) & 3)
        w.scatter_(1, col, vals[:, slot::4])
    return w


def packed(grad, meta):
    meta = meta.cpu().long()
    out = torch.zeros(grad.shape[0], grad.shape[1] // 2, dtype=grad.dtype)
    for slot in range(4):
        col = 8 * torch.arange(meta.shape[1]) + 4 * (slot // 2) + ((meta >> (2 * slot)) & 3)
        out[:, slot::4] = torch.gather(grad, 1, col)
    return out


def rms(x, w):
    return x * (x.square().mean(1, keepdim=True) + mb.EPS).rsqrt() * w


def test_gradients_of_a_block():
    """One block, so that the backward weight W^{R,C} enters the gradient of the first layer and the input only: those of the second
    layer, the norm behind it and the output norm are autograd's.  bf16 rounding (2^-8) of every intermediate on the way, six of
    them, independent: sqrt(6) 2^-8 / sqrt(3) of a gradient's norm, taken four times."""
    model = mb.PrenormMLP(128, 256, 1, state_bits=32, seed=3)
    norm1, up, norm2, down = model.blocks[0]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    x = torch.randn(96, 128, generator=gen, device="cuda").to(sl.BF16)
    dout = (torch.randn(96, 128, generator=gen, device="cuda") * 1e-2).to(sl.BF16)
    out, kept = model.forward(x)
    model.backward(dout, kept)
    torch.cuda.synchronize()
    w1, w2 = dense(up.vals, up.meta), dense(down.vals, down.meta).requires_grad_()
    g2, g = torch.ones(256, dtype=torch.float64, requires_grad=True), torch.ones(128, dtype=torch.float64, requires_grad=True)
    xd = x.double().cpu()
    n = rms(torch.relu(rms(xd, 1.0) @ w1.T), g2)
    want = rms(xd + n @ w2.T, g)
    want.backward(dout.double().cpu())
    bar = 4 * 6 ** 0.5 * 2.0 ** -8 / 3 ** 0.5
    for got, true in ((out, want.detach()), (down.grad, packed(w2.grad, down.meta)), (model.out.grad, g.grad)):
        assert float((got.double().cpu() - true).norm() / true.norm()) < bar
    # through W^{R,C} instead of W^R: the definition of the backward pass
    ndown = torch.zeros_like(w2)
    ndown += dense(down.vals_t, down.meta_t).T
    dh = torch.autograd.grad(rms(hx := (xd + n.detach() @ w2.detach().T).requires_grad_(), g.detach()), hx, dout.double().cpu())[0]
    r = torch.relu(rms(xd, 1.0) @ w1.T)
    leaf = torch.ones(256, dtype=torch.float64, requires_grad=True)
    (rms(r, leaf) * (dh @ ndown)).sum().backward()
    assert float((norm2.grad.double().cpu() - leaf.grad).norm() / leaf.grad.norm()) < bar


@pytest.mark.parametrize("bits", [32, 8])
def test_training_and_serving(bits):
    model = mb.PrenormMLP(256, 512, 2, state_bits=bits, weight_decay=0.01)
    first, last = mb.train(model, 256, steps=150)
    print("loss", first, last, flush=True)
    assert last < 0.5 * first
    assert int(model.control[2]) == 150
    x = torch.randn(64, 256, device="cuda").to(sl.BF16)
    out, served = model.forward(x)[0].float(), model.serve(x).float()
    # four products on operands that are each off by up to 2^-4 of their values, 2^-4 / sqrt(3) in the mean
    assert float((out - served).norm() / out.norm()) < 4 ** 0.5 * 2 ** 0.5 * 2.0 ** -4 / 3 ** 0.5
    # the packed copies agree after every step: the transposed one holds the same values where it keeps any
    for layer in model.layers:
        w, wt = dense(layer.vals, layer.meta), dense(layer.vals_t, layer.meta_t).T
        assert bool(((wt == w) | (wt == 0)).all())
        assert float((layer.vals.float() - layer.master).abs().max()) <= 2.0 ** -8 * float(layer.master.abs().max())
