"""Products in large tiles: k that ends inside a tile, is shorter than the tiles that are on their way, or comes in two segments;
last tiles that begin earlier, by any number of rows and columns; shared k; operands at any alignment.  Against 64 bits, with the
bounds of ``test_gpu_layers``."""
import pytest
import torch

import paper_2508_16905_amd as ta
from test_gpu_layers import act, act_error, close, generator, half, make, product_error, tiny

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]
# rows, columns, k
SHAPES = [(4099, 4104, 200), (4096, 4100, 64), (4100, 4099, 72), (2304, 8192, 136), (4096, 4352, 128), (4160, 4097, 328), (600, 392, 1000), (257, 136, 4096),
          (1000, 904, 192), (300, 131, 648)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products(m, n, k, dtype):
    g = generator("tiles", m, n, k, dtype)
    x, w, r = make(g, m, k, dtype), make(g, n, k, dtype), make(g, m, n, dtype)
    close(ta.linear(x, w, residual=r), x.double() @ w.double().T + r.double(), product_error(x, w, k) + 2.0 ** -23 * r.double().abs(), "forward")
    dy = make(g, m, n, dtype)
    dx, dw, _ = ta.linear_backward(dy, x, w)
    close(dx, dy.double() @ w.double(), product_error(dy, w.T, n), "dx")
    close(dw, dy.double().T @ x.double(), product_error(dy.T, x.T, m), "dw")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 1), (4, 4), (8, 8), (0, 64)])
def test_alignment(shift, pad, dtype):
    """Loads of 16 bytes are taken only where every row allows them; the rows' places do not change what comes out but for the
    order of the sums."""
    m, n, k = 520, 392, 264
    g = generator("alignment", shift, pad, dtype)
    x, w, dy = (make(g, rows, cols, dtype, pad=pad, shift=shift) for rows, cols in ((m, k), (n, k), (m, n)))
    close(ta.linear(x, w), x.double() @ w.double().T, product_error(x, w, k), "forward")
    dx, dw, _ = ta.linear_backward(dy, x, w)
    close(dx, dy.double() @ w.double(), product_error(dy, w.T, n), "dx")
    close(dw, dy.double().T @ x.double(), product_error(dy.T, x.T, m), "dw")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(4099, 2056, 200), (520, 392, 264), (2050, 5464, 72), (1025, 1001, 136), (4099, 5464, 1032), (1500, 2731, 521), (520, 4104, 2056)])
def test_gated(m, n, k, dtype):
    g = generator("gated tiles", m, n, k, dtype)
    x, wg, wu = make(g, m, k, dtype), make(g, n, k, dtype, scale=k ** -0.5), make(g, n, k, dtype, scale=k ** -0.5)
    h, gate, up = ta.gated(x, wg, wu, act="silu", save=True)
    zg, zu = x.double() @ wg.double().T, x.double() @ wu.double().T
    eg, eu = product_error(x, wg, k), product_error(x, wu, k)
    close(gate, zg, eg, "gate")
    close(up, zu, eu, "up")
    value, _ = act("silu", zg)
    # |silu'| is below 1.1
    close(h, value * zu, (1.1 * eg + act_error(zg)) * (zu.abs() + eu) + value.abs() * eu, "h")
    dh = make(g, m, n, dtype)
    dx, dwg, dwu, _, _ = ta.gated_backward(dh, x, wg, wu, gate, up, act="silu")
    value, slope = act("silu", gate)
    dg, du = dh.double() * up.double() * slope, dh.double() * value
    # the gradients before the activation are rounded to the call's type
    ag, au = dg.abs() + act_error(gate) * (dh.double() * up.double()).abs(), du.abs() + act_error(gate) * dh.double().abs()
    extra = half(dtype)
    floor = tiny(dtype)   # what is below the type's normal numbers
    close(dx, dg @ wg.double() + du @ wu.double(),
          product_error(ag, wg.T, 2 * n, extra) + product_error(au, wu.T, 2 * n, extra) + (ag - dg.abs() + floor) @ wg.double().abs() + (au - du.abs() + floor) @ wu.double().abs(), "dx")
    close(dwg, dg.T @ x.double(), product_error(ag.T, x.T, m, extra) + (ag - dg.abs() + floor).T @ x.double().abs(), "dwg")
    close(dwu, du.T @ x.double(), product_error(au.T, x.T, m, extra) + (au - du.abs() + floor).T @ x.double().abs(), "dwu")


def test_the_same_call_gives_the_same_bits():
    g = generator("same bits")
    x, w = make(g, 4099, 328, torch.bfloat16), make(g, 4104, 328, torch.bfloat16)
    first = ta.linear(x, w)
    assert all(torch.equal(first, ta.linear(x, w)) for _ in range(3))


def test_nothing_is_written_beside_the_result():
    g = generator("beside")
    x, w = make(g, 4099, 136, torch.bfloat16), make(g, 4100, 136, torch.bfloat16)
    wide = torch.full((4101, 4120), 7.0, dtype=torch.bfloat16, device="cuda")
    ta.linear(x, w, out=wide[1:4100, 8:4108])
    assert (wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :8] == 7).all() and (wide[:, 4108:] == 7).all()
    close(wide[1:4100, 8:4108], x.double() @ w.double().T, product_error(x, w, 136), "result")
