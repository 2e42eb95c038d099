"""Feed-forward blocks trained with the layer operators and the optimizer step, and served one row at a time.

Each block is

    r <- r + s g * P(drop(W_down (silu(W_gate y) * (W_up y)))),   y <- N(r)

with the norms P and N, a gate g per channel and a residual scale s.  The operators compute the forward and the backward
pass; the step updates the parameters from the gradients as they come out of it and chooses the precision of each.  A block
runs in the widest type that the step stores one of its matrices in.  The curvature is the empirical Fisher information,
which needs nothing beside the gradients.

    python -m paper_2508_16905_amd.examples.train_block
"""
from __future__ import annotations

import torch

import paper_2508_16905_amd as ta

HYPER = dict(
    beta_var=0.9, beta_curv=0.9, tau_low=1e-7, tau_high=1e-5, tau_curv=50.0, alpha=0.05, sparsity_ppm=900000, momentum=0.9,
    weight_decay=1e-4, ctrl_interval=5, scale_backoff=0.5, scale_growth=2.0, growth_interval=50, rho_low=0.70, rho_high=0.90,
    delta_up=16, delta_down=16, b_min=32, b_max=512, curvature_source=1,
)
_DTYPE = {ta.FP16: torch.float16, ta.BF16: torch.bfloat16, ta.FP32: torch.float32}
D_IN, D, D_HID, D_OUT, BLOCKS = 32, 64, 172, 4, 2
SCALE, EPS = 0.7, 1e-5
# parameters in order: the way in, then of each block w_gate, w_up, w_down, gate, post weight, norm weight, then the way out
SHAPES = [(D, D_IN), (D,)] + [(D_HID, D), (D_HID, D), (D, D_HID), (D,), (D,), (D,)] * BLOCKS + [(D_OUT, D), (D_OUT,)]


def widest(*tensors: torch.Tensor) -> torch.dtype:
    kinds = {t.dtype for t in tensors}
    return kinds.pop() if len(kinds) == 1 else torch.float32


def block_of(params, i: int):
    return params[2 + 6 * i: 8 + 6 * i]


def forward(params, x, drops=None, keep=None):
    """The network's output for the rows of ``x``.  ``drops``: a ``Dropout`` per block; ``keep``: a list that gets what the
    backward pass needs."""
    w_in, b_in, w_out, b_out = params[0], params[1], params[-2], params[-1]
    x = x.to(w_in.dtype)
    r = ta.linear(x, w_in, b_in, act="gelu", save=keep is not None)
    if keep is not None:
        r, pre = r
        keep.append((x, pre))
    ones = torch.ones(D, device=x.device)
    norm = ta.Norm("rms", ones, None, EPS)   # before the first block
    for i in range(BLOCKS):
        w_gate, w_up, w_down, gate, post_w, norm_w = block_of(params, i)
        dt = widest(w_gate, w_up, w_down)
        r = r.to(dt)
        w_gate, w_up, w_down = w_gate.to(dt), w_up.to(dt), w_down.to(dt)
        if i == 0:
            y = ta.residual_norm(r, norm=norm)[1]
        y = y.to(dt)
        h = ta.gated(y, w_gate, w_up, save=keep is not None)
        if keep is not None:
            h, g, u = h
        drop = drops[i] if drops is not None else None
        b = ta.linear(h, w_down, dropout=drop)
        post, after = ta.Norm("rms", post_w, None, EPS), ta.Norm("rms", norm_w, None, EPS)
        before, y_in = r, y
        r, y = ta.residual_norm(r, b, gate=gate, post=post, norm=after, scale=SCALE)
        if keep is not None:
            keep.append((before, y_in, h, g, u, b, r, drop))
    dt = w_out.dtype
    y = y.to(dt)
    if keep is not None:
        keep.append((y,))
    return ta.linear(y, w_out, b_out)


def backward(params, d_out, keep):
    """Gradients of all parameters, in their order, from that of the output."""
    w_in, w_out = params[0], params[-2]
    fp32 = torch.float32
    (y,) = keep.pop()
    dy, dw_out, db_out = ta.linear_backward(d_out, y, w_out, bias_grad=True, weight_grad_dtype=fp32)
    grads = [dw_out, db_out]
    dr = None
    for i in reversed(range(BLOCKS)):
        w_gate, w_up, w_down, gate, post_w, norm_w = block_of(params, i)
        before, y_in, h, g, u, b, r, drop = keep.pop()
        dt = r.dtype
        w_gate, w_up, w_down = w_gate.to(dt), w_up.to(dt), w_down.to(dt)
        post, after = ta.Norm("rms", post_w, None, EPS), ta.Norm("rms", norm_w, None, EPS)
        got = ta.residual_norm_backward(dr.to(dt) if dr is not None else None, dy.to(dt), r, b, gate=gate, post=post, norm=after,
                                        scale=SCALE)
        dh, dw_down, _ = ta.linear_backward(got.block, h, w_down, dropout=drop, weight_grad_dtype=fp32)
        dy, dw_gate, dw_up, _, _ = ta.gated_backward(dh, y_in, w_gate, w_up, g, u, weight_grad_dtype=fp32)
        dr = got.residual
        grads = [dw_gate, dw_up, dw_down, got.gate, got.post_weight, got.norm_weight] + grads
    norm = ta.Norm("rms", torch.ones(D, device=dr.device), None, EPS)
    dr = ta.residual_norm_backward(dr, dy, before, norm=norm).residual
    x, pre = keep.pop()
    _, dw_in, db_in = ta.linear_backward(dr.to(w_in.dtype), x, w_in, pre, act="gelu", x_grad=False, bias_grad=True, weight_grad_dtype=fp32)
    return [dw_in, db_in] + grads


def train(steps: int = 200, p: float = 0.05, seed: int = 0, device: str = "cuda:0", verbose: bool = True):
    """Fits the network to a smooth synthetic target; returns the losses and the parameters."""
    dev = torch.device(device)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    teacher = torch.randn(D_IN, D_OUT, generator=gen, device=dev) / D_IN ** 0.5
    init = [torch.randn(s, generator=gen, device=dev) * s[1] ** -0.5 if len(s) == 2 else torch.ones(s, device=dev) for s in SHAPES]
    init[1].zero_()
    init[-1].zero_()
    opt = ta.TriAccel(HYPER, [t.reshape(-1) for t in init])
    codes = [ta.FP32] * len(SHAPES)
    loss_scale, batch, losses = 1024.0, 96, []

    def parameters():
        return [opt.param(i, codes[i]).reshape(SHAPES[i]) for i in range(len(SHAPES))]

    for t in range(1, steps + 1):
        params = parameters()
        x = torch.randn(batch, D_IN, generator=gen, device=dev)
        target = torch.sin(x @ teacher)
        drops = [ta.Dropout(p, seed=seed * BLOCKS + i, offset=t) for i in range(BLOCKS)]
        keep = []
        off = forward(params, x, drops, keep).float() - target
        d_out = (off * (2.0 * loss_scale / off.numel())).to(params[-2].dtype)
        grads = backward(params, d_out, keep)
        free, total = torch.cuda.mem_get_info(dev)
        opt.step([g.reshape(-1) for g in grads], lr=0.02, loss_scale=loss_scale, batch_size=batch, mem_used_bytes=total - free,
                 mem_total_bytes=total)
        res = opt.result()
        loss_scale, batch = res.next_loss_scale, min(res.next_batch_size, HYPER["b_max"])
        codes = [s.code for s in opt.layer_state()]
        losses.append(float((off * off).mean()))
        if verbose and (t % 20 == 0 or t == 1):
            print(f"step {t:4d}  loss {losses[-1]:.5f}  skipped {res.skipped}  loss scale {loss_scale:g}  batch {batch}  codes {codes}")
    params = [v.clone() for v in parameters()]
    opt.close()
    return losses, params


if __name__ == "__main__":
    out, trained = train()
    print(f"loss {out[0]:.4f} -> {sum(out[-10:]) / 10:.4f}")
    row = forward(trained, torch.randn(1, D_IN, device="cuda"))
    print("one row served:", [round(v, 3) for v in row[0].tolist()])
