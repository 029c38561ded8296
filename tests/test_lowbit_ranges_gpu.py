"""Sizes, strides and masks where include/xnor_lowbit.h's calls change what they do: products whose rows are staged first, narrow and wide rows of
logits, rows further apart than 32 bits count.  Bounds as in the tests of each call."""
import math

import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, assert_within, filled, generator, normal
from tests import test_w4_linear_gpu as products
from tests.test_logprobs_gpu import check as check_logprobs
from tests.test_logprobs_gpu import run as run_logprobs
from tests.test_w4_linear_gpu import check as check_product
from tests.test_w4_linear_gpu import make, product, scratch

pytestmark = pytest.mark.gpu
STAGED = [(200, 4000, 1030), (129, 4001, 2051)]              # enough rows that they are staged, too few results for the largest tiles


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,out,cin", STAGED)
def test_staged_products(t, group, rows, out, cin):
    gen = generator(rows + group)
    packed, w, top = make(gen, out, cin, group, True)
    check_product(packed, w, top, normal(gen, rows, cin).to(TYPES[t]), t, group)
    check_product(packed, w, top, normal(gen, rows, cin).to(TYPES[t]), t, group, extra=3)


@pytest.mark.parametrize("x_group", [0, 128])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,out,cin", STAGED + [(200, 4000, 1024), (131, 4001, 2048)])
def test_staged_8_bit_products(x_group, group, rows, out, cin):
    gen = generator(rows + group + x_group)
    packed, w, _ = make(gen, out, cin, group, True)
    q = torch.randint(-127, 128, (rows, cin), generator=gen, dtype=torch.int8)
    xs = torch.rand((rows, -(-cin // x_group) if x_group else 1), generator=gen) + 0.5
    y = filled((rows, out), torch.bfloat16)
    xnor.xnor_w4_linear_q8(q.cuda(), xs.cuda(), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group, x_group)
    want = sums = 0
    for k in range(0, cin, group):
        whole = torch.round(w[:, k:k + group] / packed.test_scale[:, k // group, None])
        part = (q[:, k:k + group].double() @ whole.t()) * packed.test_scale[:, k // group] * xs.double()[:, k // x_group if x_group else 0, None]
        want, sums = want + part, sums + part.abs()
    assert_within(y, want, (-(-cin // group) + 8) * 2 * EPS32 * sums + HALF_ULP["bf16"] * want.abs() + SMALLEST["bf16"], "y")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16", "q8"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_the_largest_tiles(t, group):
    """Every type and group on results enough for them, sizes that no tile divides."""
    products.test_products_of_very_many_rows(t, 2050, 8198, 261, group)


@pytest.mark.parametrize("out,cin", [(20, 40), (600, 200)])
def test_a_million_rows(out, cin):
    """More rows than 65535 tiles of 16: the first, the last and some between are looked at."""
    gen = generator(out)
    rows = 1_100_003
    packed, w, top = make(gen, out, cin, 32, True)
    x = torch.randn((rows, cin), device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).to(torch.bfloat16)
    y = torch.empty((rows, out), dtype=torch.bfloat16, device="cuda")
    xnor.xnor_w4_linear(x, packed.wimg, y, scratch(rows, cin, out, 32), rows, cin, out, 32)
    some = torch.cat((torch.arange(40), torch.randint(0, rows, (40,), generator=gen), torch.arange(rows - 40, rows))).cuda()
    x = x[some].double().cpu()
    want = x @ w.t()
    bound = 4 * cin * 62 * EPS32 * x.square().mean(1).sqrt()[:, None] * top[None]
    assert_within(y[some], want, bound + HALF_ULP["bf16"] * want.abs() + SMALLEST["bf16"], "y")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,out,cin", [(200, 4000, 1030), (2100, 8200, 520)])
def test_infinities_and_nan_in_staged_rows(t, rows, out, cin):
    gen = generator(8)
    packed, w, top = make(gen, out, cin, 32, True)
    x = normal(gen, rows, cin).to(TYPES[t])
    x[2, cin - 1], x[rows - 1, 0] = math.inf, math.nan
    y = product(packed, x, t, rows, cin, out, 32)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[2, rows - 1]] = True
    assert y[bad].isnan().all() and y[~bad].isfinite().all()


def test_8_bit_rows_whose_scale_is_nan():
    gen = generator(9)
    for rows, out, cin in ((5, 100, 300), (200, 4000, 1030), (200, 4000, 1024), (2100, 8200, 520)):
        packed, _, _ = make(gen, out, cin, 64, False)
        q = torch.randint(-127, 128, (rows, cin), generator=gen, dtype=torch.int8).cuda()
        for x_group in (0, 64):
            xs = torch.ones((rows, -(-cin // x_group) if x_group else 1), device="cuda")
            xs[3, -1] = math.nan
            y = filled((rows, out), torch.bfloat16)
            xnor.xnor_w4_linear_q8(q, xs, packed.wimg, y, scratch(rows, cin, out, 64), rows, cin, out, 64, x_group)
            bad = torch.arange(rows, device="cuda") == 3
            assert y[bad].isnan().all() and y[~bad].isfinite().all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [63, 64, 65, 511, 512, 513, 1025, 2047, 2048, 2049, 8191, 8193, 16384, 16385])
def test_widths_of_logits(t, vocab):
    gen = generator(vocab)
    for rows in (1, 5, 300):
        l = normal(gen, rows, vocab, scale=4).to(TYPES[t])
        l[torch.rand((rows, vocab), generator=gen) < 0.5] = -math.inf
        l[rows // 2] = -math.inf                                            # (a row that its mask leaves nothing of)
        l[rows // 3, : vocab // 2] = 1.0                                    # (and one of ties)
        check_logprobs(l, torch.randint(-1, vocab + 1, (rows, 2), generator=gen), 20)
        check_logprobs(l, torch.randint(0, vocab, (rows, 1), generator=gen, dtype=torch.int32), 0, extra=5)


@pytest.mark.parametrize("t,vocab", [("bf16", 20003), ("f32", 9000)])
def test_many_long_rows_of_every_order(t, vocab):
    """Enough rows that none is shared out: alternatives are found over many chunks, of random, rising, falling, equal, masked and lopsided rows."""
    gen = generator(vocab)
    at = torch.arange(vocab)
    lowest = torch.finfo(TYPES[t]).min
    kinds = [normal(gen, vocab, scale=3), at / 64.0, -at / 64.0, torch.zeros(vocab), torch.full((vocab,), lowest), torch.full((vocab,), -math.inf),
             torch.where(at < 5, 1.0, -math.inf), torch.where(at % 2048 < 32, at / 64.0, 0.0), torch.where(at >= vocab - 7, 2.0, lowest),
             torch.where(torch.rand(vocab, generator=gen) < 0.99, lowest, 3.0), (at % 3).float(), torch.randint(0, 5, (vocab,), generator=gen).float()]
    few = torch.stack(kinds).to(TYPES[t])
    tokens = torch.randint(0, vocab, (len(kinds), 1), generator=gen)
    times = 4200 // len(kinds)
    for top in (1, 20, 32):
        want = check_logprobs(few, tokens, top)
        got = run_logprobs(few.repeat(times, 1), tokens.repeat(times, 1), top)
        for name in ("lse", "shift", "entropy", "logprob", "top_logprob"):
            a, b = got[name].view(times, *want[name].shape), want[name][None]
            assert ((a == b) | ((a - b).abs() <= 2e-5 * (1 + b.abs()))).all(), name
        assert torch.equal(got["top_index"].view(times, *want["top_index"].shape), want["top_index"].expand(times, -1, -1))


FAR = 2 ** 31 + 24                                                          # elements between two rows: three rows pass 32 bits of elements


def far(x, stride=FAR):
    wide = torch.empty((len(x) - 1) * stride + x.shape[1], dtype=x.dtype, device="cuda").as_strided(x.shape, (stride, 1))
    wide.copy_(x)
    return wide


def test_rows_far_apart_in_the_norm():
    gen = generator(10)
    x = normal(gen, 3, 1000).to(torch.bfloat16).cuda()
    w = (torch.rand(1000, generator=gen) + 0.5).cuda()
    outs = []
    for rows in (x, far(x)):
        o = [filled((3, 1000), torch.int8), filled((3, 1), torch.float32), filled((3, 1000), torch.bfloat16), filled((3,), torch.float32)]
        xnor.xnor_rmsnorm_q8(rows, None, w, None, *o, 3, 1000, 0, 1e-6)
        g = [filled((3, 1000), torch.bfloat16), filled((1000,), torch.float32)]
        xnor.xnor_rmsnorm_backward(rows, o[3], w, rows, rows, *g, filled((xnor.rmsnorm_backward_workspace_bytes(3, 1000),), torch.uint8), 3, 1000)
        outs.append(o + g)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("rows,out,cin,stride", [(3, 100, 500, FAR), (3, 32000, 4100, FAR), (200, 4000, 1030, 2 ** 24 + 24)])
def test_rows_far_apart_in_a_product(rows, out, cin, stride):
    gen = generator(11)
    packed, _, _ = make(gen, out, cin, 64, True)
    x = normal(gen, rows, cin).to(torch.float16).cuda()
    near, wide = filled((rows, out), torch.float16), filled((rows, out), torch.float16)
    xnor.xnor_w4_linear(x, packed.wimg, near, scratch(rows, cin, out, 64), rows, cin, out, 64)
    xnor.xnor_w4_linear(far(x, stride), packed.wimg, wide, scratch(rows, cin, out, 64), rows, cin, out, 64)
    assert torch.equal(near, wide)
