"""Rows to 8 bits, activation functions that keep their input in 8 bits, and their gradients, against the formulas."""
import math

import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, apart, assert_within, filled, generator, normal

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -100


def to_8_bits(x, group):
    """The contract in float32 on the CPU, one rounding per operation: integers, scales."""
    rows, cols = x.shape
    group = group or cols
    t = torch.nn.functional.pad(x.float(), (0, -cols % group)).view(rows, -1, group)
    top = t.abs().amax(-1)
    top = torch.where(t.isnan().any(-1), float("nan"), top)
    finite, some = top < float("inf"), top >= TINY
    factor = torch.where(finite & some, torch.full_like(top, 127.0) / top, 0.0)
    q = torch.where(finite[..., None], torch.round(t * factor[..., None]), 0.0)
    scale = torch.where(finite, torch.where(some, top / 127, 0.0), float("nan"))
    return q.view(rows, -1)[:, :cols].to(torch.int8), scale


def rows8(x, group):
    rows, cols = x.shape
    q, scale = filled((rows, cols), torch.int8), filled((rows, -(-cols // group) if group else 1), torch.float32)
    xnor.xnor_q8_rows(x, q, scale, rows, cols, group)
    return q, scale


def difficult(gen, rows, cols, t):
    """Normal values with outliers; a row of zeros, one of tiny values, infinities, NaN, the largest numbers."""
    x = normal(gen, rows, cols) * torch.where(torch.rand(cols, generator=gen) < 0.02, 30.0, 1.0)
    for i, row in enumerate(range(1, rows, 2)):
        kind = i % 6
        if kind == 0:
            x[row] = 0.0
        elif kind == 1:
            x[row] *= 2.0 ** -104
        elif kind == 2:
            x[row, int(torch.randint(0, cols, (1,), generator=gen))] = -float("inf")
        elif kind == 3:
            x[row, int(torch.randint(0, cols, (1,), generator=gen))] = float("nan")
        elif kind == 4:
            x[row] = x[row].sign() * float(torch.finfo(t).max)
    return x.to(t)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("rows,cols,extra", [(1, 1, 0), (13, 7, 3), (5, 64, 0), (14, 100, 1), (3, 512, 0), (13, 513, 5), (2, 1003, 0), (14, 4096, 8), (3, 8192, 0),
                                             (13, 8193, 0), (2, 16384, 0), (13, 16390, 2), (1, 40001, 0), (1030, 33, 0)])
@pytest.mark.parametrize("name", TYPES)
def test_rows(name, rows, cols, extra, group):
    x = difficult(generator(rows + cols), rows, cols, TYPES[name])
    want, want_scale = to_8_bits(x, group)
    q, scale = rows8(apart(x, extra), group)
    assert torch.equal(q.cpu(), want)
    assert torch.equal(scale.cpu().nan_to_num(-1.0), want_scale.nan_to_num(-1.0))


def gelu(x):
    """(1 + erf would lose the tail: of -7 it leaves 12 bits of 64-bit numbers)"""
    return 0.5 * x * torch.special.erfc(x * -math.sqrt(0.5))


def function(x, name):
    return {"relu": torch.relu, "gelu": gelu, "silu": torch.nn.functional.silu}[name](x)


def value_error(x, name):
    """Relative error of f in float32: the functions' own (erfc 16, exp 3 units of 2 EPS32), a division and two products, and the argument's rounding, which the normal
    distribution's tail multiplies by x^2 (twice: the constant's and the product's)."""
    return {"relu": torch.zeros_like(x), "gelu": (40 + 4 * x * x) * EPS32, "silu": torch.full_like(x, 16 * EPS32)}[name]


def slope_error(x, name):
    """Absolute error of f': its terms are at most 1 + x^2 / 2, their relative errors as above."""
    return torch.zeros_like(x) if name == "relu" else 64 * EPS32 * (1 + x * x)


CASES = [(1, 8, 0), (3, 7, 5), (5, 64, 0), (6, 100, 2), (2, 512, 0), (3, 520, 0), (4, 1003, 0), (5, 4096, 8), (2, 8192, 0), (3, 16392, 0), (2, 16001, 1), (515, 96, 0)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,extra", CASES)
def test_activation(rows, cols, extra, name, gated):
    for i, (tname, t) in enumerate(TYPES.items()):
        gen = generator(rows + cols + i)
        group, kept_group = ((0, 64), (32, 0), (128, 32))[(i + rows + cols) % 3]
        wide = cols * (2 if gated else 1)
        x = (3 * normal(gen, rows, wide)).to(t)
        given = apart(x, extra)
        y, q, scale = filled((rows, cols), t), filled((rows, cols), torch.int8), filled((rows, -(-cols // group) if group else 1), torch.float32)
        kept, kept_scale = filled((rows, wide), torch.int8), filled((rows, -(-wide // kept_group) if kept_group else 1), torch.float32)
        xnor.xnor_activation_q8(given, y, q, scale, kept, kept_scale, rows, cols, group, kept_group, name, gated)
        # the input, kept as xnor_q8_rows keeps it
        want, want_scale = to_8_bits(x, kept_group)
        assert torch.equal(kept.cpu(), want) and torch.equal(kept_scale.cpu(), want_scale)
        # values
        d = x.double()
        a = function(d[:, :cols], name) * (d[:, cols:] if gated else 1.0)
        err = (value_error(d[:, :cols], name) + (EPS32 if gated else 0)) * a.abs()
        assert_within(y, a, HALF_ULP[tname] * (a.abs() + err) + err + SMALLEST[tname], "y")
        # their 8 bits: half a step, what the value is off, and the roundings of the factor and the products
        g = group or cols
        top = torch.nn.functional.pad(a, (0, -cols % g)).view(rows, -1, g).abs().amax(-1)
        off = torch.nn.functional.pad(err, (0, -cols % g)).view(rows, -1, g).amax(-1)
        some = top > 1e-6
        assert_within(scale.cpu()[some], top[some] / 127, (off[some] + 2 * EPS32 * top[some]) / 127, "scale")
        s = scale.double().cpu().repeat_interleave(g, 1)[:, :cols]
        assert_within(q.double().cpu() * s, a, 0.5 * s + err + off.repeat_interleave(g, 1)[:, :cols] + 127 * 4 * EPS32 * s + 1e-30, "q")
        # one output at a time gives the same
        y2, q2, scale2, kept2 = filled((rows, cols), t), filled((rows, cols), torch.int8), torch.full_like(scale, -1), filled((rows, wide), torch.int8)
        xnor.xnor_activation_q8(given, y2, None, None, None, None, rows, cols, group, kept_group, name, gated)
        xnor.xnor_activation_q8(given, None, q2, scale2, None, None, rows, cols, group, kept_group, name, gated)
        xnor.xnor_activation_q8(given, None, None, None, kept2, torch.full_like(kept_scale, -1), rows, cols, group, kept_group, name, gated)
        assert torch.equal(y2, y) and torch.equal(q2, q) and torch.equal(scale2, scale) and torch.equal(kept2, kept)


def gradient_of(x, g, name, gated):
    """By differentiation in 64 bits, and the bound of what float32 may be off."""
    x = x.clone().requires_grad_()
    cols = g.shape[1]
    a = function(x[:, :cols], name) * (x[:, cols:] if gated else 1.0)
    a.backward(g)
    d = x.detach()
    err = g.abs() * slope_error(d[:, :cols], name)
    if gated:
        up, f = d[:, cols:].abs(), function(d[:, :cols], name)
        err = torch.cat((err * up, g.abs() * (value_error(d[:, :cols], name) + EPS32 * (1 + d[:, :cols].abs())) * f.abs() + EPS32 * g.abs() * f.abs()), 1)
    return x.grad, err + 4 * EPS32 * x.grad.abs()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,extra", CASES)
def test_backward(rows, cols, extra, name, gated):
    for i, (tname, t) in enumerate(TYPES.items()):
        gen = generator(rows + cols + i)
        group = (0, 32, 64, 128)[(i + rows + cols) % 4]
        wide = cols * (2 if gated else 1)
        kept, scale = rows8((3 * normal(gen, rows, wide)).to(t).cuda(), group)
        g = normal(gen, rows, cols).to(t)
        g_x = filled((rows, wide), t)
        xnor.xnor_activation_backward(kept, scale, apart(g, extra), g_x, rows, cols, group, name, gated)
        values = (kept.float() * (scale.repeat_interleave(group, 1)[:, :wide] if group else scale)).double().cpu()
        want, err = gradient_of(values, g.double(), name, gated)
        assert_within(g_x, want, HALF_ULP[tname] * (want.abs() + err) + err + SMALLEST[tname], "g_x")
        if not gated:                                       # in place
            same = g.cuda()
            xnor.xnor_activation_backward(kept, scale, same, same, rows, cols, group, name)
            assert torch.equal(same, g_x)


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_gradient_against_differences(name):
    gen = generator(3)
    rows, cols, h = 4, 200, 2.0 ** -13
    kept, scale = rows8((2 * normal(gen, rows, 2 * cols)).cuda(), 32)
    g = normal(gen, rows, cols)
    g_x = filled((rows, 2 * cols), torch.float32)
    xnor.xnor_activation_backward(kept, scale, g.cuda(), g_x, rows, cols, 32, name, True)
    v = (kept.float() * scale.repeat_interleave(32, 1)[:, :2 * cols]).double().cpu()

    def total(x):
        return function(x[:, :cols], name) * x[:, cols:] * g.double()

    def moved(half):
        step = torch.zeros_like(v)
        step[:, cols * half:cols * (half + 1)] = h
        return (total(v + step) - total(v - step)) / (2 * h)

    # the third derivatives are below 2: h^2 / 3 of them, and the float32 bound
    _, err = gradient_of(v, g.double(), name, True)
    bound = err + h * h * (1 + v.abs().max()) * g.double().abs().repeat(1, 2) + EPS32 * g_x.double().cpu().abs()
    assert_within(g_x, torch.cat((moved(0), moved(1)), 1), bound, "g_x")


def test_infinities_and_nan():
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[1.0, -inf, 2.0, nan], [inf, -1.0, 0.0, -0.0]]).cuda()
    y, kept, scale = filled((2, 4), torch.float32), filled((2, 4), torch.int8), filled((2, 1), torch.float32)
    xnor.xnor_activation_q8(x, y, None, None, kept, scale, 2, 4, 0, 0, "relu")
    assert torch.equal(y.cpu().nan_to_num(-9.0, posinf=99.0), torch.tensor([[1.0, 0.0, 2.0, -9.0], [99.0, 0.0, 0.0, 0.0]]))
    assert scale.isnan().all() and (kept == 0).all()
    g_x = filled((2, 4), torch.float32)
    xnor.xnor_activation_backward(kept, scale, torch.ones((2, 4), device="cuda"), g_x, 2, 4, 0, "gelu")
    assert g_x.isnan().all()


def test_far_values():
    """Far out the functions are 0 or the value itself."""
    x = torch.tensor([[-1e4, -100.0, -40.0, 40.0, 100.0, 1e30]]).cuda()
    for name in ("gelu", "silu"):
        y = filled((1, 6), torch.float32)
        xnor.xnor_activation_q8(x, y, None, None, None, None, 1, 6, 0, 0, name)
        want = function(x.double().cpu(), name)
        assert_within(y, want, 40 * EPS32 * want.abs() + 1e-15, name)


def test_no_rows():
    e = torch.empty((0, 64), device="cuda")
    xnor.xnor_q8_rows(e, None, None, 0, 64, 0)
    xnor.xnor_activation_q8(e, None, None, None, None, None, 0, 64, 0, 0, "relu")
    xnor.xnor_activation_backward(None, None, e, None, 0, 64, 0, "relu")


def test_rows_past_32_bits_of_offset():
    """q and scale of rows whose first element is further than 2^32 bytes from the start."""
    rows, cols = 3, 64
    stride = 2 ** 30 + 8
    flat = torch.zeros(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((rows, cols), (stride, 1))
    x.copy_(normal(generator(1), rows, cols))
    q, scale = rows8(x, 32)
    want, want_scale = to_8_bits(x.cpu(), 32)
    assert torch.equal(q.cpu(), want) and torch.equal(scale.cpu(), want_scale)
    assert math.isfinite(float(scale.sum()))


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_values_everywhere(name):
    """A sweep down to where the values leave the normal numbers and past it, where both functions round to 0."""
    x = torch.cat((torch.linspace(-15, 15, 400001), torch.linspace(-110, 110, 200001), torch.logspace(-40, 0, 4001), -torch.logspace(-40, 0, 4001)))
    n = x.numel() // 8
    x = x[:8 * n].view(8, n)
    y = filled((8, n), torch.float32)
    xnor.xnor_activation_q8(x.cuda(), y, None, None, None, None, 8, n, 0, 0, name)
    a = function(x.double(), name)
    assert_within(y, a, value_error(x.double(), name) * a.abs() + SMALLEST["f32"], "y")


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_slopes_everywhere(name):
    scale = torch.logspace(-12, 0, 1500)[:, None]
    kept = torch.arange(-127, 128).to(torch.int8).expand(1500, 255).contiguous()
    g_x = filled((1500, 255), torch.float32)
    xnor.xnor_activation_backward(kept.cuda(), scale.cuda(), torch.ones((1500, 255), device="cuda"), g_x, 1500, 255, 0, name)
    values = (kept.float() * scale).double()
    want, err = gradient_of(values, torch.ones_like(values), name, False)
    assert_within(g_x, want, err + EPS32 * want.abs() + SMALLEST["f32"], "g_x")


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_infinities_of_smooth_functions(name):
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[inf, -inf, nan, 3.0e38, -3.0e38, 0.0, -0.0, 1.0e-45]]).cuda()
    y = filled((1, 8), torch.float32)
    xnor.xnor_activation_q8(x, y, None, None, None, None, 1, 8, 0, 0, name)
    y = y.cpu()[0]
    assert y[0] == inf and y[1] == 0 and y[2].isnan() and y[3] == x[0, 3].cpu() and bool((y[4:7] == 0).all()) and 0 <= float(y[7]) <= 1.5e-45
