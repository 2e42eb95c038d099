"""The layer operators together, as the example uses them: its network's output and gradients against autograd in 64 bits, a row
served alone against the same row of a batch, and a fit with the optimizer step behind them."""
import math

import pytest
import torch

import paper_2508_16905_amd as ta
from paper_2508_16905_amd.examples import train_block as E

pytestmark = pytest.mark.gpu


def parameters(dtype, seed=3):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    init = [torch.randn(s, generator=gen, device="cuda") * (s[1] ** -0.5 if len(s) == 2 else 0.2) + (0.0 if len(s) == 2 else 1.0) for s in E.SHAPES]
    return [t.to(dtype) for t in init], torch.randn(37, E.D_IN, generator=gen, device="cuda"), torch.randn(37, E.D_OUT, generator=gen, device="cuda")


def plain(params, x):
    """The network of the example's docstring, without dropout."""
    def rms(v, w):
        return v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + E.EPS) * w

    z = x @ params[0].T + params[1]
    r = 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    y = rms(r, 1.0)
    for i in range(E.BLOCKS):
        w_gate, w_up, w_down, gate, post_w, norm_w = E.block_of(params, i)
        g = y @ w_gate.T
        b = (g * torch.sigmoid(g) * (y @ w_up.T)) @ w_down.T
        r = r + E.SCALE * gate * rms(b, post_w)
        y = rms(r, norm_w)
    return y @ params[-2].T + params[-1]


def apart(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


# About sixteen operators lie on the longest way from an input to a gradient.  In fp32 each is off by at most (172 + 8) 2^-24 of
# what it sums, in 16 bits by half a step for its result and half for what it rounds on the way; a factor of 4 for cancellation
# in the sums and for what the norms make of an error.
@pytest.mark.parametrize("dtype,bound", [(torch.float32, 16 * 180 * 2.0 ** -24 * 4), (torch.float16, 16 * 2.0 ** -10 * 4), (torch.bfloat16, 16 * 2.0 ** -7 * 4)])
def test_output_and_gradients(dtype, bound):
    params, x, d_out = parameters(dtype)
    x, d_out = x.to(dtype), d_out.to(dtype)
    leaves = [p.double().requires_grad_(True) for p in params]
    want = plain(leaves, x.double())
    want_grads = torch.autograd.grad(want, leaves, d_out.double())
    keep = []
    got = E.forward(params, x, keep=keep)
    assert got.dtype is dtype and apart(got, want.detach()) < bound
    for i, (g, w) in enumerate(zip(E.backward(params, d_out, keep), want_grads)):
        assert g.dtype is torch.float32 and g.shape == w.shape and apart(g, w) < bound, i
    assert not keep


def test_blocks_of_different_precisions():
    params, x, _ = parameters(torch.float32)
    want = plain([p.double() for p in params], x.double())
    mixed = list(params)
    mixed[2:5] = [p.bfloat16() for p in params[2:5]]
    mixed[8] = params[8].half()   # one matrix of the second block: it runs in fp32
    assert apart(E.forward(mixed, x), want) < 16 * 2.0 ** -7 * 4


def test_a_row_served_alone():
    params, x, _ = parameters(torch.float32)
    batch = E.forward(params, x)
    for i in (0, 36):
        assert apart(E.forward(params, x[i: i + 1]), batch[i: i + 1].double()) < 2 * 16 * 180 * 2.0 ** -24 * 4


def test_the_fit_improves():
    losses, params = E.train(steps=150, verbose=False)
    first, last = sum(losses[:5]) / 5, sum(losses[-10:]) / 10
    assert last < 0.5 * first and all(math.isfinite(v) for v in losses), (first, last)
    assert E.forward(params, torch.zeros(1, E.D_IN, device="cuda")).shape == (1, E.D_OUT)


def test_the_same_seed_gives_the_same_fit():
    assert E.train(steps=12, verbose=False)[0] == E.train(steps=12, verbose=False)[0]
