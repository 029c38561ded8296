"""4-bit products of float32 rows that are staged first, at the accuracy of 32-bit sums: rows of one sign (what a layer behind a ReLU gets), single terms.

Bounds.  A code enters the products as 16 + u, and what that and the zero point add is taken out again with the groups' sums.  `group_by_group` does so for
one group after the other, each 32 inputs' terms added exactly and rounded once.  The kernels may take four groups out at a time: their totals, and so their
roundings, are up to four times as large.  Errors are compared as root mean squares over some 10^4 results."""
import math

import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, TYPES, apart, assert_within, filled, generator, normal
from tests.test_w4_linear_gpu import codes_of, scratch

pytestmark = pytest.mark.gpu


def weights(gen, out, cin, group):
    """Codes 0..15 around 8, scales and zero points per group; the image."""
    groups = -(-cin // group)
    u = torch.round(4 * torch.randn((out, cin), generator=gen) + 8).clamp(0, 15).to(torch.uint8)
    scale = (torch.rand((out, groups), generator=gen) + 0.5) * 0.01
    zero = torch.randint(5, 11, (out, groups), generator=gen, dtype=torch.uint8)
    return u, scale, zero, xnor.W4Weights(codes_of(u).cuda(), scale.cuda(), zero.cuda(), cin, group)


def group_by_group(x, u, scale, zero, group):
    """The sums of the definition in float32, and in 64 bits."""
    total = torch.zeros(x.shape[0], u.shape[0])
    exact = total.double()
    for g, k in enumerate(range(0, x.shape[1], group)):
        xs, us = x[:, k:k + group].double(), u[:, k:k + group].double()
        acc = torch.zeros_like(total)
        for i in range(0, xs.shape[1], 32):
            acc = (acc.double() + xs[:, i:i + 32] @ (16 + us[:, i:i + 32]).t()).float()
        offset = 16 + zero[:, g].double()
        part = (acc.double() - xs.sum(1, keepdim=True).float().double() * offset).float()
        total = (total.double() + part.double() * scale[:, g].double()).float()
        exact += (xs @ us.t() - xs.sum(1, keepdim=True) * zero[:, g].double()) * scale[:, g].double()
    return total, exact


@pytest.mark.parametrize("sign", ["one sign", "relu", "both signs"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,out,cin", [(256, 4096, 9216), (2048, 4096, 9216), (200, 4000, 1030), (2100, 8200, 520)])
def test_error_of_staged_float32_rows(rows, out, cin, group, sign):
    """256 x 9216 -> 4096 and 200 x 1030 -> 4000: eight waves share the inputs; the others: the largest tiles (9216 inputs in groups of 64: by waves)."""
    gen = generator(rows + group)
    u, scale, zero, packed = weights(gen, out, cin, group)
    x = torch.randn((rows, cin), generator=gen)
    x = {"one sign": x.abs(), "relu": x.relu(), "both signs": x}[sign]
    y = filled((rows, out), torch.float32)
    xnor.xnor_w4_linear(x.cuda(), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group)
    some, which = torch.randperm(rows, generator=gen)[:32], torch.randperm(out, generator=gen)[:384]
    near, exact = group_by_group(x[some], u[which], scale[which], zero[which], group)
    error = (y[some.cuda()][:, which.cuda()].cpu().double() - exact).square().mean().sqrt()
    assert error <= 4 * (near.double() - exact).square().mean().sqrt()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,out,cin", [(200, 4000, 1030), (2100, 8200, 520)])
def test_single_terms_keep_their_24_bits(rows, out, cin, group):
    """One input per row, of which every part of 8 bits counts: y = x s (u - z) within the roundings of x s (16 + u) and x s (16 + z), eight of them.
    (Without its last part a term would be off by 2^-16.5 of itself, 15 s at most: five times as much.)"""
    gen = generator(rows + group)
    u, scale, zero, packed = weights(gen, out, cin, group)
    at = torch.arange(rows) * 37 % cin
    x = torch.zeros(rows, cin)
    x[torch.arange(rows), at] = (1 + 2.0 ** -8 + 2.0 ** -16 + 2.0 ** -23) * 2.0 ** (torch.arange(rows) % 9 * 8 - 32).float()
    y = filled((rows, out), torch.float32)
    xnor.xnor_w4_linear(apart(x, 3), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group)
    some = torch.cat((torch.arange(70), torch.arange(rows - 70, rows)))
    at, value = at[some], x.amax(1)[some].double()[:, None]
    s, z = scale[:, at // group].t().double(), zero[:, at // group].t().double()
    assert_within(y[some.cuda()], value * s * (u[:, at].t().double() - z), 8 * EPS32 * 31 * value * s, "single terms")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("rows,out,cin", [(5, 100, 300), (20, 1000, 1003), (200, 4000, 1030), (2100, 8200, 520)])
def test_rows_as_large_as_their_type(rows, out, cin, group, t):
    """Finite rows of any size give finite results: sums of 16 + u terms must not leave the range that those of u - z keep."""
    gen = generator(rows + group)
    u, scale, zero, _ = weights(gen, out, cin, group)
    scale = scale * 1e-3
    packed = xnor.W4Weights(codes_of(u).cuda(), scale.cuda(), zero.cuda(), cin, group)
    largest = torch.finfo(TYPES[t]).max
    x = (torch.rand((rows, cin), generator=gen) * 2 - 1) * largest
    x[0], x[1], x[2] = largest, -largest, torch.where(torch.arange(cin) % 2 == 0, largest, -largest)
    x = x.to(TYPES[t])
    y = filled((rows, out), TYPES[t])
    xnor.xnor_w4_linear(x.cuda(), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group)
    some = torch.cat((torch.arange(5), torch.randint(0, rows, (50,), generator=gen)))
    whole = u.double() - zero.double().repeat_interleave(group, 1)[:, :cin]
    want = x[some].double() @ (whole * scale.double().repeat_interleave(group, 1)[:, :cin]).t()
    # (every rounding relative to 62 scales of the row's sum, 4 of them for each 32 inputs, added at random: eight standard deviations)
    bound = 8 * math.sqrt(4 * cin / 32) * EPS32 * 62 * x[some].double().abs().amax(1)[:, None] * 512 * scale.double().amax(1)
    assert_within(y[some.cuda()], want, bound + HALF_ULP[t] * want.abs(), "y")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
def test_weights_as_large_as_their_type(t, zeros):
    """Finite weights have finite scales, and codes within half a step of them (and a zero point's half, with zero points)."""
    gen = generator(17)
    out, cin, group = 9, 300, 32
    largest = torch.finfo(TYPES[t]).max
    w = ((torch.rand((out, cin), generator=gen) * 2 - 1) * largest).to(TYPES[t])
    w[0, :2], w[1], w[2] = torch.tensor([largest, -largest]), largest, -largest
    groups = -(-cin // group)
    codes, scale = filled((out, 16 * -(-cin // 32)), torch.uint8), filled((out, groups), torch.float32)
    zero = filled((out, groups), torch.uint8) if zeros else None
    xnor.xnor_w4_quantize(w.cuda(), codes, scale, zero, out, cin, group)
    codes = codes.cpu()
    u = torch.stack((codes & 15, codes >> 4), -1).flatten(1)[:, :cin].double()
    z = (zero.cpu() if zeros else torch.full((out, groups), 8)).double().repeat_interleave(group, 1)[:, :cin]
    s = scale.cpu().double().repeat_interleave(group, 1)[:, :cin]
    assert scale.isfinite().all() and (scale > 0).all()
    assert (((u - z) * s - w.double()).abs() <= (1.001 if zeros else 0.501) * s).all()
