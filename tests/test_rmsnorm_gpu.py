"""xnor_rmsnorm_q8 and its backward pass against the formulas in 64 bits (the 8-bit integers against the same float32 operations).

Bounds: a sum of n squares or products added in a tree of at most 64 levels is off by 64 roundings of 2^-24, relative for squares (4e-6); a
result rounds once more to its type."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, apart, assert_within, filled, generator, normal

pytestmark = pytest.mark.gpu
EPS, TINY = 1e-6, 2.0 ** -100


def groups_of(cols, group):
    return -(-cols // group) if group else 1


def reference(x, residual, weight, group):
    """h, 1/rms in 64 bits; q as the float32 operations give it; top per group."""
    h = x.float() + residual.float() if residual is not None else x.float()
    rstd = 1 / (h.double().square().mean(1) + EPS).sqrt()
    t = h * weight if weight is not None else h
    rows, cols = t.shape
    g = group or cols
    t = torch.nn.functional.pad(t, (0, -cols % g)).view(rows, -1, g)
    top = t.abs().amax(-1)
    some = top >= TINY
    q = torch.round(t * torch.where(some, torch.full_like(top, 127.0) / top, torch.zeros_like(top))[..., None])
    top = torch.where(some, top, torch.zeros_like(top))
    return h, rstd, q.reshape(rows, -1)[:, :cols], top


def run(x, residual, weight, group, t, with_values=True, extra=0):
    rows, cols = x.shape
    out = {"sum": filled((rows, cols), TYPES[t]), "q": filled((rows, cols), torch.int8),
           "scale": filled((rows, groups_of(cols, group)), torch.float32), "rstd": filled((rows,), torch.float32),
           "values": filled((rows, cols), TYPES[t]) if with_values else None}
    xnor.xnor_rmsnorm_q8(apart(x, extra), apart(residual, 2 * extra) if residual is not None else None,
                         weight.cuda() if weight is not None else None, out["sum"], out["q"], out["scale"], out["values"], out["rstd"], rows, cols,
                         group, EPS)
    torch.cuda.synchronize()
    return {k: v.cpu() if v is not None else None for k, v in out.items()}


def check(x, residual, weight, group, t, extra=0):
    h, rstd, q, top = reference(x, residual, weight, group)
    got = run(x, residual, weight, group, t, extra=extra)
    assert torch.equal(got["sum"], h.to(TYPES[t]))
    assert torch.equal(got["q"].float(), q)
    assert_within(got["rstd"], rstd, 4e-6 * rstd, "rstd")
    scale = top.double() * rstd[:, None] / 127
    assert_within(got["scale"], scale, 5e-6 * scale, "scale")
    values = q.double() * scale.repeat_interleave(group or x.shape[1], 1)[:, :x.shape[1]]
    assert_within(got["values"], values, (HALF_ULP[t] + 6e-6) * values.abs() + SMALLEST[t], "values")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 0), (1, 7, 32), (3, 8, 64), (5, 31, 0), (2, 33, 32), (7, 500, 128), (4, 512, 64), (3, 513, 0),
                                             (2, 1003, 32), (9, 4096, 128), (3, 4097, 0), (2, 9216, 64), (1, 16384, 0), (2, 16391, 128),
                                             (1, 32768, 32)])
def test_sizes(t, rows, cols, group):
    gen = generator(rows * 100003 + cols)
    x, r = normal(gen, rows, cols, scale=3).to(TYPES[t]), normal(gen, rows, cols).to(TYPES[t])
    w = torch.rand(cols, generator=gen) + 0.5
    check(x, r, w, group, t)


@pytest.mark.parametrize("residual,weight", [(False, True), (True, False), (False, False)])
def test_absent_inputs(residual, weight):
    gen = generator(5)
    x = normal(gen, 6, 300).to(torch.bfloat16)
    check(x, normal(gen, 6, 300).to(torch.bfloat16) if residual else None, torch.rand(300, generator=gen) - 0.5 if weight else None, 64, "bf16")


@pytest.mark.parametrize("extra", [1, 5, 8])
@pytest.mark.parametrize("t", ["f32", "f16"])
def test_rows_that_lie_apart(t, extra):
    gen = generator(extra)
    check(normal(gen, 11, 264).to(TYPES[t]), normal(gen, 11, 264).to(TYPES[t]), None, 32, t, extra=extra)


def test_halves_round_to_even_and_the_largest_is_127():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -127.0, 126.5]])
    got = run(x, None, None, 0, "f32")
    assert got["q"].tolist() == [[127, 0, 2, 2, 0, -2, -127, 126]]


def test_rows_and_groups_of_zeros_infinities_and_nan():
    x = torch.zeros(5, 128)
    x[1, 40:] = normal(generator(1), 88)            # zeros in the first group
    x[2] = normal(generator(2), 128)
    x[2, 70] = float("inf")                         # an infinity in the third of four groups: 1/rms is 0
    x[3] = normal(generator(3), 128)
    x[3, 5] = float("nan")
    x[4] = 1e-35 * normal(generator(4), 128)        # below the least top of a group
    got = run(x, None, None, 32, "f32")
    nan = float("nan")
    assert got["scale"][0].tolist() == [0, 0, 0, 0] and not got["q"][0].any()
    assert got["scale"][1, 0] == 0 and (got["scale"][1, 1:] > 0).all()
    assert torch.equal(got["scale"][2].nan_to_num(nan=-1.0), torch.tensor([0.0, 0.0, -1.0, 0.0])) and got["rstd"][2] == 0
    assert not got["q"][2, 64:96].any() and got["q"][2, :64].any()
    assert got["scale"][3].isnan().all() and got["rstd"][3] != got["rstd"][3] and not got["q"][3, :32].any()
    assert got["scale"][4].tolist() == [0, 0, 0, 0] and not got["q"][4].any()
    assert got["values"][3].isnan().all() and not got["values"][0].any() and nan != nan


def test_sum_in_place_and_outputs_that_are_not_wanted():
    gen = generator(8)
    x, r = normal(gen, 33, 777).to(torch.bfloat16), normal(gen, 33, 777).to(torch.bfloat16)
    want = run(x, r, None, 32, "bf16")
    xd, rd = x.cuda(), r.cuda()
    values = filled((33, 777), torch.bfloat16)
    xnor.xnor_rmsnorm_q8(xd, rd, None, rd, None, None, values, None, 33, 777, 32, EPS)      # the residual stream in place
    assert torch.equal(rd.cpu(), want["sum"]) and torch.equal(values.cpu(), want["values"])
    q, scale = filled((33, 777), torch.int8), filled((33, 25), torch.float32)
    xnor.xnor_rmsnorm_q8(xd, r.cuda(), None, None, q, scale, None, None, 33, 777, 32, EPS)
    assert torch.equal(q.cpu(), want["q"]) and torch.equal(scale.cpu(), want["scale"])


def reference_backward(h, rstd, weight, g, g_sum):
    h, rstd, g = h.double(), rstd.double()[:, None], g.double()
    w = weight.double() if weight is not None else torch.ones(h.shape[1], dtype=torch.float64)
    n, wg = h * rstd, g * w
    dot = (wg * n).mean(1, keepdim=True)
    g_h = rstd * (wg - n * dot) + (g_sum.double() if g_sum is not None else 0)
    # roundings of the terms, of their difference, and of the dot product (64 levels)
    bound = EPS32 * (rstd * (8 * wg.abs() + n.abs() * (8 * dot.abs() + 64 * (wg * n).abs().mean(1, keepdim=True))) + 2 * g_h.abs())
    return g_h, bound, (g * n).sum(0), (g * n).abs().sum(0)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,weight,g_sum,extra", [(1, 1, True, True, 0), (1, 9, True, False, 0), (3, 511, False, True, 3), (5, 512, True, True, 0),
                                                          (600, 77, True, True, 8), (4, 4096, True, True, 0), (2, 4099, False, False, 1),
                                                          (7, 9216, True, True, 0), (2, 16390, True, True, 0), (1, 32768, True, False, 0)])
def test_backward(t, rows, cols, weight, g_sum, extra):
    gen = generator(rows + cols)
    h, g, gs = (normal(gen, rows, cols).to(TYPES[t]) for _ in range(3))
    w = torch.rand(cols, generator=gen) + 0.5 if weight else None
    rstd = (1 / (h.double().square().mean(1) + EPS).sqrt()).float()
    want, bound, want_w, sum_w = reference_backward(h, rstd, w, g, gs if g_sum else None)
    g_h, g_w = filled((rows, cols), TYPES[t]), filled((cols,), torch.float32)
    size = xnor.rmsnorm_backward_workspace_bytes(rows, cols)
    xnor.xnor_rmsnorm_backward(apart(h, extra), rstd.cuda(), w.cuda() if weight else None, apart(g, 2 * extra),
                               apart(gs, extra) if g_sum else None, g_h, g_w, filled((size,), torch.uint8), rows, cols)
    assert_within(g_h, want, bound + HALF_ULP[t] * want.abs() + SMALLEST[t], "g_h")
    assert_within(g_w, want_w, (rows + 64) * EPS32 * sum_w, "g_weight")


def test_backward_against_differences():
    """The norm without its rounding, differentiated numerically in 64 bits."""
    gen = generator(77)
    rows, cols = 2, 40
    h, g, w = normal(gen, rows, cols).double(), normal(gen, rows, cols).double(), torch.rand(cols, generator=gen).double() + 0.5

    def loss(h):
        return (g * w * h / (h.square().mean(1, keepdim=True) + EPS).sqrt()).sum()

    want = torch.empty_like(h)
    for i in range(rows):
        for j in range(cols):
            d = torch.zeros_like(h)
            d[i, j] = 1e-5
            want[i, j] = (loss(h + d) - loss(h - d)) / 2e-5
    rstd = (1 / (h.square().mean(1) + EPS).sqrt()).float()
    g_h = filled((rows, cols), torch.float32)
    xnor.xnor_rmsnorm_backward(h.float().cuda(), rstd.cuda(), w.float().cuda(), g.float().cuda(), None, g_h, None, None, rows, cols)
    assert_within(g_h, want, 1e-5 * (1 + want.abs()), "g_h")


def test_backward_in_place_and_twice_the_same_bits():
    gen = generator(9)
    h, g, gs = (normal(gen, 700, 333).to(torch.bfloat16).cuda() for _ in range(3))
    rstd, w = torch.rand(700, generator=gen).cuda(), torch.rand(333, generator=gen).cuda()
    ws = filled((xnor.rmsnorm_backward_workspace_bytes(700, 333),), torch.uint8)
    first, gw1, gw2 = filled((700, 333), torch.bfloat16), filled((333,), torch.float32), filled((333,), torch.float32)
    xnor.xnor_rmsnorm_backward(h, rstd, w, g, gs, first, gw1, ws, 700, 333)
    xnor.xnor_rmsnorm_backward(h, rstd, w, g, gs, gs, gw2, ws, 700, 333)
    assert torch.equal(first, gs) and torch.equal(gw1, gw2)


def test_no_rows():
    empty = torch.empty((0, 64), device="cuda")
    g_w = filled((64,), torch.float32)
    xnor.xnor_rmsnorm_q8(empty, empty, None, empty, None, None, empty, None, 0, 64, 0, EPS)
    xnor.xnor_rmsnorm_backward(empty, empty, None, empty, None, empty, g_w, None, 0, 64)
    assert not g_w.any()
