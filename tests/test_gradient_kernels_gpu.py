"""Weight gradients of special values in every kernel that takes them: the one of few products, and tiles of 64, 128 and 256 with their factors in one part and two.
Which kernel a size reaches is checked without a GPU (test_lowbit8_choices.py)."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, filled, generator, normal
from tests.test_weight_gradient_gpu import make, values

pytestmark = pytest.mark.gpu

SIZES = [(100, 128, 60), (1200, 130, 60), (150, 3300, 2300), (600, 4100, 3600)]
KINDS = [("bf16", "bf16", 32), ("bf16", "bf16", 0), ("f16", "bf16", 0), ("bf16", "f32", 64), ("bf16", "f32", 0), ("f16", "f16", 128), ("f32", "f32", 32), ("f32", "f32", 0), ("f32", "bf16", 64)]

cases = pytest.mark.parametrize("rows,cin,out,name,wname,group", [s + k for s in SIZES for k in KINDS])


def run(q, scale, g, group, wname, accumulate=None):
    (rows, cin), out = q.shape, g.shape[1]
    work = filled((xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, group, g.dtype, TYPES[wname]),), torch.uint8)
    g_w, g_b = (filled((out, cin), TYPES[wname]), filled((out,), torch.float32)) if accumulate is None else (t.clone() for t in accumulate)
    xnor.xnor_q8_weight_gradient(q.cuda(), scale.cuda(), g.cuda(), g_w, g_b, work, rows, cin, out, group, accumulate is not None)
    return g_w, g_b


def term(name, wname, group):
    """Of a product of one value and one gradient: a factor's one float16, of 11 bits, is off by half a step of 2^-10, 2^-11 of it; two are by 2^-11 of what the first leaves, 2^-22,
    and of two such factors the product of both remainders, 2^-22 more, is left out.  (A hundredth for products of these and the rounding to float32 before.)"""
    if wname != "bf16":
        return 3.01 * 2.0 ** -22
    return 2.0 ** -11 * 1.01 + (3.01 * 2.0 ** -22 if name == "f32" else 0)


@cases
def test_what_is_not_finite_stays_in_its_row_or_columns(rows, cin, out, name, wname, group):
    gen = generator(rows + group)
    q, scale, g = make(gen, rows, cin, out, group, name)
    q[q == 0] = 1
    clean, _ = run(q, scale, g, group, wname)
    assert bool(clean.isfinite().all())
    g[30, 5], g[31, 6], g[97, 59] = float("inf"), float("nan"), -float("inf")
    bad = torch.zeros((out, cin), dtype=torch.bool)
    bad[5], bad[6], bad[59] = True, True, True
    if group:
        scale[40, min(1, scale.shape[1] - 1)], scale[99, 0] = float("nan"), float("inf")
        bad[:, :2 * group] = True
    g_w, g_b = run(q, scale, g, group, wname)
    assert torch.equal(~g_w.isfinite().cpu(), bad)
    # the exponents of the others are those of before
    assert torch.equal(g_w.cpu()[~bad], clean.cpu()[~bad])
    some = torch.zeros(out, dtype=torch.bool)
    some[5], some[6], some[59] = True, True, True
    assert torch.equal(~g_b.isfinite().cpu(), some)
    if not group:
        for value in (float("nan"), float("inf")):
            scale[40] = value
            assert not bool(run(q, scale, g, group, wname)[0].isfinite().any())


@cases
def test_places(rows, cin, out, name, wname, group):
    """One row and one output at a time: which value meets which gradient.  Codes of 7 bits times powers of two are exact in one part."""
    q = ((torch.arange(rows)[:, None] * 31 + torch.arange(cin)[None] * 7) % 251 - 125).to(torch.int8)
    scale = 2.0 ** ((torch.arange(rows)[:, None] + torch.arange(-(-cin // group) if group else 1)[None]) % 5).float()
    g = torch.zeros((rows, out))
    at = (torch.arange(out) * 37) % rows
    g[at, torch.arange(out)] = 1.0
    g_w, g_b = run(q, scale, g.to(TYPES[name]), group, wname)
    assert torch.equal(g_w.double().cpu(), values(q, scale, group)[at])          # (below 2^11, of 7 bits: in every type)
    assert torch.equal(g_b.cpu(), torch.ones(out))


@cases
def test_far_below_a_columns_largest(rows, cin, out, name, wname, group):
    """One product per result, each factor up to 2^-38 of its column's largest (of a group: of 128 times its largest scale): to a factor's bits, or to 2^-39 of that largest."""
    gen = generator(rows + cin)
    q, _, _ = make(gen, rows, cin, out, group, "f32")
    groups = -(-cin // group) if group else 1
    small = 12 if name == "f16" else 38
    at = 2 + torch.arange(out) % (rows - 2)                                      # the row that counts
    g = torch.zeros((rows, out))
    g[at, torch.arange(out)] = (1 + torch.rand(out, generator=gen)) * 2.0 ** -(torch.arange(out) * 7 % (small + 1)).float()
    g[0] = 1 + torch.rand(out, generator=gen)                                    # the largest, on a row of zeros
    q[0], q[1] = 0, 127                                                          # the largest scale, on a row without a gradient
    scale = (1 + torch.rand((rows, groups), generator=gen)) * 2.0 ** -(torch.randint(0, 39 if group else 2, (rows, groups), generator=gen)).float()
    scale[:2] = 1 + torch.rand((2, groups), generator=gen)
    g = g.to(TYPES[name])
    g_w, _ = run(q, scale, g, group, wname)
    x, d = values(q, scale, group)[at], g.double()
    mine = d[at, torch.arange(out)][:, None]
    want = mine * x
    if group:
        top_x = 128 * scale.double().amax(0).repeat_interleave(group)[None, :cin]
        far = 2.0 ** -39 * (d.amax(0)[:, None] * x.abs() + top_x * mine.abs()) + 2.0 ** -78 * top_x * d.amax(0)[:, None]
    else:
        far = 2.0 ** -39 * (d * scale.double()).amax(0)[:, None] * q[at].double().abs()
    err = want.abs() * (term(name, wname, group) + EPS32) + 1.0001 * far
    err = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0)
    over = (g_w.double().cpu() - want).abs() - err
    assert int((~(over <= 0)).sum()) == 0, float(over.max())


@cases
def test_columns_of_very_different_size(rows, cin, out, name, wname, group):
    """Columns that differ by many powers of two: each counts by its own largest."""
    gen = generator(12)
    q, scale, g = make(gen, rows, cin, out, group, "f32")
    small = 10 if name == "f16" else 60
    g = (g * 2.0 ** torch.linspace(-small, 3, out)).to(TYPES[name])
    if wname != "f16":
        scale = scale * 2.0 ** torch.linspace(-40, 40, scale.shape[1])
    g_w, _ = run(q, scale, g, group, wname)
    x, d = values(q, scale, group).cuda(), g.double().cuda()
    total, want = d.abs().t().contiguous() @ x.abs(), d.t().contiguous() @ x
    top = (d.abs() * scale.double().cuda()).amax(0)[:, None] * 128 if not group else d.abs().amax(0)[:, None] * 128 * scale.double().amax(0).repeat_interleave(group)[None, :cin].cuda()
    err = total * (term(name, wname, group) + EPS32 + 2 * EPS32 * (rows / 16 + 18)) + 2.0 ** -38 * rows * top + 2.0 ** -140
    err = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0)
    assert int((~((g_w.double() - want).abs() <= err)).sum()) == 0


@cases
def test_added_to_what_is_there(rows, cin, out, name, wname, group):
    gen = generator(11)
    q, scale, g = make(gen, rows, cin, out, group, name)
    before = normal(gen, out, cin).to(TYPES[wname]).cuda(), normal(gen, out).cuda()
    g_w, g_b = run(q, scale, g, group, wname, accumulate=before)
    x, d = values(q, scale, group).cuda(), g.double().cuda()
    total, want = d.abs().t().contiguous() @ x.abs(), d.t().contiguous() @ x + before[0].double()
    err = total * (term(name, wname, group) + EPS32 + 2 * EPS32 * (rows / 16 + 18)) + 2.0 ** -38 * rows * d.abs().amax(0)[:, None] * 128 * scale.max().double().cuda() + EPS32 * want.abs()
    err = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else EPS32 * want.abs())
    assert int((~((g_w.double() - want).abs() <= err)).sum()) == 0
    want = d.sum(0) + before[1].double()
    assert bool(((g_b.double() - want).abs() <= (rows + 4) * EPS32 * d.abs().sum(0) + EPS32 * want.abs()).all())
