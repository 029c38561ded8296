"""Gradients of weights and biases from 8-bit rows, against the formula in 64 bits and against differences."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, apart, assert_within, filled, generator, normal

pytestmark = pytest.mark.gpu


def gradient(q, scale, g, group, wt, accumulate=None, extra=0, bias=True):
    rows, cin = q.shape
    out = g.shape[1]
    g_w = filled((out, cin), wt) if accumulate is None else accumulate[0].clone()
    g_b = None if not bias else filled((out,), torch.float32) if accumulate is None else accumulate[1].clone()
    work = filled((xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, group, g.dtype, wt),), torch.uint8)
    xnor.xnor_q8_weight_gradient(q.cuda(), scale.cuda(), apart(g, extra), g_w, g_b, work, rows, cin, out, group, accumulate is not None)
    return g_w, g_b


def values(q, scale, group):
    return q.double() * (scale.double().repeat_interleave(group, 1)[:, :q.shape[1]] if group else scale.double())


def bounds(x, g, name, wname):
    """Per term: the value's and the gradient's representation (one 11-bit float: 2^-11, two: 2^-22 and the part of both remainders that is left out), the scale's product
    with the code; what is far below a column's largest: 2^-40 of it.  The sum: an addition every 16 rows and 16 within, with twice the rounding of float32 for the
    instruction's own order."""
    rows = x.shape[0]
    total = g.abs().t() @ x.abs()
    one = 2.0 ** -11
    term = (one + (one if name == "f32" else 0)) * 1.001 if wname == "bf16" else 2.0 ** -22 * (3 if name == "f32" else 1) * 1.001
    far = 2.0 ** -39 * rows * g.abs().amax(0)[:, None] * x.abs().amax(0)[None] + 2.0 ** -140
    return total * (term + EPS32 + 2 * EPS32 * (rows / 16 + 18)) + far, total


def make(gen, rows, cin, out, group, name):
    q = torch.randint(-127, 128, (rows, cin), generator=gen, dtype=torch.int64).to(torch.int8)
    scale = torch.exp(2 * normal(gen, rows, -(-cin // group) if group else 1)) / 50
    g = normal(gen, rows, out) * torch.exp(2 * normal(gen, rows, 1)) / 100
    return q, scale, g.to(TYPES[name])


def check(q, scale, g, group, name, wname, extra=0):
    g_w, g_b = gradient(q, scale, g, group, TYPES[wname], extra=extra)
    x, d = values(q, scale, group), g.double()
    want = d.t() @ x
    err, _ = bounds(x, d, name, wname)
    assert_within(g_w, want, err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0), "g_w")
    # parts of the rows, four waves of each, then the parts
    assert_within(g_b, d.sum(0), (q.shape[0] + 4) * EPS32 * d.abs().sum(0), "g_bias")
    return g_w, g_b


SIZES = [(1, 1, 1), (1, 128, 100), (2, 33, 31), (7, 32, 32), (16, 64, 64), (17, 100, 130), (63, 1003, 33), (64, 256, 256), (65, 257, 255), (100, 128, 1000), (129, 384, 129),
         (256, 300, 520), (300, 1003, 1000), (777, 130, 140), (1000, 512, 260), (2050, 96, 64)]


@pytest.mark.parametrize("rows,cin,out", SIZES)
@pytest.mark.parametrize("name", TYPES)
def test_gradient(name, rows, cin, out):
    for i, wname in enumerate(dict.fromkeys(("f32", name, "bf16"))):
        group = (0, 32, 64, 128)[(i + rows + cin + out) % 4]
        gen = generator(rows + cin + out + i)
        check(*make(gen, rows, cin, out, group, name), group, name, wname, extra=(0, 3, 8)[i])


@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_places(group):
    """One row and one output at a time: which value meets which gradient."""
    rows, cin, out = 150, 200, 90
    q = ((torch.arange(rows)[:, None] * 31 + torch.arange(cin)[None] * 7) % 251 - 125).to(torch.int8)
    scale = 2.0 ** ((torch.arange(rows)[:, None] + torch.arange(-(-cin // group) if group else 1)[None]) % 5).float()
    g = torch.zeros((rows, out))
    at = (torch.arange(out) * 37) % rows
    g[at, torch.arange(out)] = 1.0
    g_w, g_b = gradient(q, scale, g.bfloat16(), group, torch.float32)
    assert torch.equal(g_w.double().cpu(), values(q, scale, group)[at])
    assert torch.equal(g_b.cpu(), torch.ones(out))


@pytest.mark.parametrize("wname", TYPES)
@pytest.mark.parametrize("name", TYPES)
def test_accumulated(name, wname):
    gen = generator(11)
    rows, cin, out, group = 200, 150, 77, 64
    q, scale, g = make(gen, rows, cin, out, group, name)
    before = normal(gen, out, cin).to(TYPES[wname]).cuda(), normal(gen, out).cuda()
    g_w, g_b = gradient(q, scale, g, group, TYPES[wname], accumulate=before)
    x, d = values(q, scale, group), g.double()
    want = d.t() @ x + before[0].double().cpu()
    err, _ = bounds(x, d, name, wname)
    err = err + EPS32 * want.abs()
    assert_within(g_w, want, err + HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname], "g_w")
    want = d.sum(0) + before[1].double().cpu()
    assert_within(g_b, want, (rows + 4) * EPS32 * d.abs().sum(0) + EPS32 * want.abs(), "g_bias")


@pytest.mark.parametrize("name", TYPES)
def test_gradients_of_very_different_size(name):
    """Columns and rows that differ by many powers of two: each column counts by its own largest."""
    gen = generator(12)
    rows, cin, out = 300, 130, 70
    q, scale, g = make(gen, rows, cin, out, 32, "f32")
    small = 10 if name == "f16" else 60
    g = (g * 2.0 ** torch.linspace(-small, 3, out)).to(TYPES[name])
    scale = scale * 2.0 ** torch.linspace(-40, 40, scale.shape[1])
    check(q, scale, g, 32, name, "f32")


def test_largest_and_smallest_numbers():
    rows, cin, out = 40, 64, 48
    gen = generator(13)
    q, _, _ = make(gen, rows, cin, out, 0, "f32")
    g = torch.full((rows, out), 1.0) * 2.0 ** torch.linspace(-126, 126, out)
    scale = torch.full((rows, 1), 2.0 ** -20)
    g_w, _ = gradient(q, scale, g, 0, torch.float32)
    x, d = values(q, scale, 0), g.double()
    # (of the terms, not of the sum: 40 codes of both signs may cancel, and what the roundings leave is relative to each of them)
    assert_within(g_w, d.t() @ x, 2.0 ** -20 * (d.abs().t() @ x.abs()) + 64 * 2.0 ** -149, "g_w")


@pytest.mark.parametrize("wname", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_row_or_columns(wname):
    gen = generator(14)
    rows, cin, out, group = 100, 128, 60, 32
    q, scale, g = make(gen, rows, cin, out, group, "bf16")
    q[q == 0] = 1
    clean, _ = gradient(q, scale, g, group, TYPES[wname])
    g[30, 5], g[31, 6], scale[40, 2] = float("inf"), float("nan"), float("nan")
    g_w, g_b = gradient(q, scale, g, group, TYPES[wname])
    bad = torch.zeros((out, cin), dtype=torch.bool)
    bad[5], bad[6], bad[:, 64:96] = True, True, True
    assert torch.equal(~g_w.isfinite().cpu(), bad)
    # the exponents of the others are those of before
    assert torch.equal(g_w.cpu()[~bad], clean.cpu()[~bad])
    assert torch.equal(~g_b.isfinite().cpu(), torch.arange(out).clamp(5, 6) == torch.arange(out))
    # (no more is said of them: an infinity times a value's two floats, whose signs may differ, adds up to NaN)


def test_against_differences():
    """The loss sum(g * (x^ w^T)) is linear in w: its differences are its gradient to the roundings of 64 bits."""
    gen = generator(15)
    rows, cin, out, group = 60, 40, 20, 32
    q, scale, g = make(gen, rows, cin, out, group, "f32")
    g_w, g_b = gradient(q, scale, g, group, torch.float32)
    x, d = values(q, scale, group), g.double()
    w = normal(gen, out, cin).double()

    def loss(w, b):
        return (d * (x @ w.t() + b)).sum()

    err, _ = bounds(x, d, "f32", "f32")
    zero, h = torch.zeros(out, dtype=torch.float64), 2.0 ** -4
    for o, k in ((0, 0), (19, 39), (7, 31), (7, 32), (12, 5)):
        step = torch.zeros_like(w)
        step[o, k] = h
        slope = (loss(w + step, zero) - loss(w - step, zero)) / (2 * h)
        assert abs(float(g_w[o, k]) - float(slope)) <= float(err[o, k]) + 1e-10 * float(loss(w.abs(), zero).abs())
        step = torch.zeros_like(zero)
        step[o] = h
        slope = (loss(w, step) - loss(w, -step)) / (2 * h)
        assert abs(float(g_b[o]) - float(slope)) <= (rows + 4) * EPS32 * float(d[:, o].abs().sum()) + 1e-10 * float(loss(w.abs(), zero).abs())


def test_no_rows():
    for wname, t in TYPES.items():
        g_w, g_b = filled((7, 33), t), filled((7,), torch.float32)
        e = torch.empty((0, 7), device="cuda")
        xnor.xnor_q8_weight_gradient(None, None, e, g_w, g_b, None, 0, 33, 7, 0)
        assert (g_w == 0).all() and (g_b == 0).all()
        g_w.fill_(3.0)
        xnor.xnor_q8_weight_gradient(None, None, e, g_w, None, None, 0, 33, 7, 0, accumulate=True)
        assert (g_w == 3).all()


@pytest.mark.parametrize("wname", ["f32", "bf16"])
def test_the_same_bits_every_time_and_without_the_bias(wname):
    gen = generator(16)
    q, scale, g = make(gen, 500, 700, 300, 64, "bf16")
    first, _ = gradient(q, scale, g, 64, TYPES[wname])
    for bias in (True, False, True):
        assert torch.equal(gradient(q, scale, g, 64, TYPES[wname], bias=bias)[0], first)
