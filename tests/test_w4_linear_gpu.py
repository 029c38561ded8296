"""4-bit weights: rounding, packing and products against the formulas in 64 bits.

Bounds of a product (float32 sums of n terms |x| (16 + u) <= 31 |x|, and as much again for the offset's sum): n roundings of 2^-24 of partial
sums that grow like sqrt(n) for inputs of random sign, four standard deviations: 4 n 62 2^-24 rms(x) scale.  8-bit rows: integers up to the
groups' sums, whose float32 additions round."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, apart, assert_within, filled, generator, normal

pytestmark = pytest.mark.gpu
# out, in, group, zero points
SHAPES = [(1, 1, 32, True), (16, 32, 32, False), (17, 128, 128, True), (5, 129, 64, True), (33, 100, 128, False), (48, 257, 32, True),
          (1000, 1003, 64, True), (64, 4096, 128, False), (130, 2080, 32, True)]


def codes_of(u):
    """[out][in] codes to bytes, rows of whole 32 inputs; the padding holds 15."""
    u = torch.nn.functional.pad(u, (0, -u.shape[1] % 32), value=15)
    return (u[:, 0::2] | u[:, 1::2] << 4).contiguous()


def make(gen, out, cin, group, zeros):
    groups = -(-cin // group)
    u = torch.randint(0, 16, (out, cin), generator=gen, dtype=torch.uint8)
    scale = (torch.rand((out, groups), generator=gen) + 0.5) * 0.01
    zero = torch.randint(0, 16, (out, groups), generator=gen, dtype=torch.uint8) if zeros else None
    packed = xnor.W4Weights(codes_of(u).cuda(), scale.cuda(), zero.cuda() if zeros else None, cin, group)
    z = (zero if zeros else torch.full((out, groups), 8)).double().repeat_interleave(group, 1)[:, :cin]
    s = scale.double().repeat_interleave(group, 1)[:, :cin]
    packed.test_scale = scale.double()
    return packed, (u.double() - z) * s, scale.double().amax(1)


def scratch(rows, cin, out, group):
    size = xnor.w4_linear_workspace_bytes(rows, cin, out, group)
    return filled((size,), torch.uint8) if size else None


def product(packed, x, t, rows, cin, out, group, extra=0):
    y = filled((rows, out), TYPES[t])
    xnor.xnor_w4_linear(apart(x, extra), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group)
    return y


def check(packed, w, top_scale, x, t, group, extra=0):
    (rows, cin), out = x.shape, w.shape[0]
    y = product(packed, x, t, rows, cin, out, group, extra)
    want = x.double() @ w.t()
    rms = x.double().square().mean(1).sqrt()
    bound = 4 * cin * 62 * EPS32 * rms[:, None] * top_scale[None]
    assert_within(y, want, bound + HALF_ULP[t] * want.abs() + SMALLEST[t], "y")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("out,cin,group,zeros", SHAPES)
def test_products(t, out, cin, group, zeros):
    gen = generator(out + cin)
    packed, w, top = make(gen, out, cin, group, zeros)
    for rows in (1, 2, 16, 17, 37, 64, 65, 130):
        check(packed, w, top, normal(gen, rows, cin).to(TYPES[t]), t, group)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,out,cin,group", [(300, 520, 600, 128), (1030, 260, 1003, 32), (129, 1000, 4096, 64), (4, 8192, 1024, 128), (257, 129, 96, 64)])
def test_products_of_many_rows(t, rows, out, cin, group):
    gen = generator(rows)
    packed, w, top = make(gen, out, cin, group, rows % 2 == 0)
    check(packed, w, top, normal(gen, rows, cin).to(TYPES[t]), t, group)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16", "q8"])
@pytest.mark.parametrize("rows,out,cin,group", [(2100, 8200, 520, 32), (2049, 8192, 384, 64), (2050, 8190, 640, 128)])
def test_products_of_very_many_rows(t, rows, out, cin, group):
    """Enough results for the largest tiles; the first and last rows and some between are looked at."""
    gen = generator(rows)
    packed, w, top = make(gen, out, cin, group, True)
    some = torch.cat((torch.arange(130), torch.randint(0, rows, (64,), generator=gen), torch.arange(rows - 66, rows)))
    if t != "q8":
        x = normal(gen, rows, cin).to(TYPES[t])
        y = product(packed, x, t, rows, cin, out, group)[some.cuda()]
        want = x[some].double() @ w.t()
        rms = x[some].double().square().mean(1).sqrt()
        assert_within(y, want, 4 * cin * 62 * EPS32 * rms[:, None] * top[None] + HALF_ULP[t] * want.abs() + SMALLEST[t], "y")
        return
    for x_group in (0, 128):
        q = torch.randint(-127, 128, (rows, cin), generator=gen, dtype=torch.int8)
        xs = torch.rand((rows, -(-cin // x_group) if x_group else 1), generator=gen) + 0.5
        y = filled((rows, out), torch.float32)
        xnor.xnor_w4_linear_q8(q.cuda(), xs.cuda(), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group, x_group)
        want = sums = 0
        for k in range(0, cin, group):
            whole = torch.round(w[:, k:k + group] / packed.test_scale[:, k // group, None])
            part = (q[some, k:k + group].double() @ whole.t()) * packed.test_scale[:, k // group] * xs[some].double()[:, k // x_group if x_group else 0, None]
            want, sums = want + part, sums + part.abs()
        assert_within(y[some.cuda()], want, (-(-cin // group) + 8) * 2 * EPS32 * sums + HALF_ULP["f32"] * want.abs(), "y")


@pytest.mark.parametrize("t,extra", [("f32", 1), ("bf16", 3), ("f16", 8), ("bf16", 8)])
@pytest.mark.parametrize("rows", [3, 40, 200])
def test_rows_that_lie_apart(t, extra, rows):
    gen = generator(rows)
    packed, w, top = make(gen, 96, 392, 64, True)
    check(packed, w, top, normal(gen, rows, 392).to(TYPES[t]), t, 64, extra)


def test_float32_rows_of_any_magnitude_keep_their_bits():
    gen = generator(3)
    packed, w, top = make(gen, 32, 64, 32, True)
    for scale in (1e-30, 1e30):
        check(packed, w, top, normal(gen, 5, 64, scale=scale), "f32", 32)
    x = torch.zeros(2, 64)
    x[0, 10], x[1, 10] = 1 + 2.0 ** -23, 2.0 ** -100
    y = product(packed, x, "f32", 2, 64, 32, 32).cpu().double()
    assert_within(y, x.double() @ w.t(), 4 * EPS32 * 62 * x.double()[:, 10:11].abs() * top[None], "single terms")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [20, 200])
def test_a_row_with_an_infinity_or_a_nan_gives_nan_and_no_other_does(t, rows):
    gen = generator(4)
    packed, w, top = make(gen, 50, 200, 32, True)
    x = normal(gen, rows, 200).to(TYPES[t])
    x[2, 199], x[5, 0] = float("inf"), float("nan")
    y = product(packed, x, t, rows, 200, 50, 32).cpu()
    bad = torch.zeros(rows, dtype=torch.bool)
    bad[[2, 5]] = True
    assert y[bad].isnan().all() and y[~bad].isfinite().all()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("out,cin,group,zeros", SHAPES)
@pytest.mark.parametrize("x_group", [0, 128])
def test_8_bit_rows(t, out, cin, group, zeros, x_group):
    gen = generator(out + cin + x_group)
    packed, w, _ = make(gen, out, cin, group, zeros)
    for rows in (1, 16, 33, 70, 300):
        q = torch.randint(-127, 128, (rows, cin), generator=gen, dtype=torch.int8)
        xs = torch.rand((rows, -(-cin // x_group) if x_group else 1), generator=gen) + 0.5
        y = filled((rows, out), TYPES[t])
        xnor.xnor_w4_linear_q8(q.cuda(), xs.cuda(), packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group, x_group)
        want, sums = torch.zeros(rows, out, dtype=torch.float64), torch.zeros(rows, out, dtype=torch.float64)
        for k in range(0, cin, group):                      # whole numbers per group, then its two scales
            whole = torch.round(w[:, k:k + group] / packed.test_scale[:, k // group, None])
            part = (q[:, k:k + group].double() @ whole.t()) * packed.test_scale[:, k // group] * xs.double()[:, k // x_group if x_group else 0, None]
            want += part
            sums += part.abs()
        assert_within(y, want, (-(-cin // group) + 8) * 2 * EPS32 * sums + HALF_ULP[t] * want.abs() + SMALLEST[t], "y")


def test_the_norms_output_feeds_the_product():
    gen = generator(12)
    rows, cin, out = 19, 640, 200
    for group, x_group in ((32, 32), (64, 64), (32, 64), (128, 128), (64, 0)):
        packed, w, _ = make(gen, out, cin, group, True)
        x = normal(gen, rows, cin).cuda()
        q, xs, v = filled((rows, cin), torch.int8), filled((rows, -(-cin // x_group) if x_group else 1), torch.float32), filled((rows, cin), torch.float32)
        xnor.xnor_rmsnorm_q8(x, None, None, None, q, xs, v, None, rows, cin, x_group, 1e-6)
        y = filled((rows, out), torch.float32)
        xnor.xnor_w4_linear_q8(q, xs, packed.wimg, y, scratch(rows, cin, out, group), rows, cin, out, group, x_group)
        want = v.cpu().double() @ w.t()
        assert_within(y, want, 64 * EPS32 * (v.cpu().double().abs() @ w.abs().t()), "y")


def test_rounding_to_codes():
    """The float32 operations of the definition, in torch."""
    gen = generator(6)
    for t, (out, cin, group) in zip(("f32", "bf16", "f16", "f32"), ((9, 300, 64), (16, 128, 128), (3, 1003, 32), (2, 5000, 128))):
        w = normal(gen, out, cin).to(TYPES[t])
        w[0, :group] = 0
        w[1, 3:group] = w[1, 3:group].abs()
        for zeros in (False, True):
            groups = -(-cin // group)
            f = torch.nn.functional.pad(w.float(), (0, groups * group - cin)).view(out, groups, group)
            lo, hi = f.amin(-1).clamp(max=0), f.amax(-1).clamp(min=0)
            span, levels = (hi - lo, 15.0) if zeros else (torch.maximum(hi, -lo), 7.0)
            some = span >= 2.0 ** -100
            inv = torch.where(some, torch.full_like(span, levels) / span, torch.zeros_like(span))
            z = torch.round(-lo * inv) if zeros else torch.full_like(span, 8.0)
            u = (torch.round(f * inv[..., None]) + z[..., None]).clamp(0, 15).reshape(out, -1)[:, :cin].to(torch.uint8)
            codes, scale = filled((out, 16 * -(-cin // 32)), torch.uint8), filled((out, groups), torch.float32)
            zero = filled((out, groups), torch.uint8) if zeros else None
            xnor.xnor_w4_quantize(apart(w, 3), codes, scale, zero, out, cin, group)
            got = codes.cpu()
            got = torch.stack((got & 15, got >> 4), -1).flatten(1)[:, :cin]
            assert torch.equal(got, u)
            assert torch.equal(scale.cpu(), torch.where(some, span / torch.full_like(span, levels), torch.zeros_like(span)))
            assert not zeros or torch.equal(zero.cpu().float(), z)
            # half a step where nothing is clamped; what lies past a zero point's rounding is another half
            packed = xnor.W4Weights.quantized(w.cuda(), group, zeros)
            eye = torch.eye(cin)[: min(cin, 70)]
            y = product(packed, eye, "f32", eye.shape[0], cin, out, group).cpu().t()
            assert ((y - w.float()[:, : eye.shape[0]]).abs() <= (1.0 if zeros else 0.51) * scale.cpu().repeat_interleave(group, 1)[:, : eye.shape[0]] + 1e-6).all()


def test_same_call_same_bits_and_no_rows():
    gen = generator(21)
    packed, w, top = make(gen, 300, 2000, 64, True)
    for rows in (1, 50, 200):
        x = normal(gen, rows, 2000).to(torch.bfloat16)
        assert torch.equal(product(packed, x, "bf16", rows, 2000, 300, 64), product(packed, x, "bf16", rows, 2000, 300, 64))
    empty = torch.empty((0, 2000), device="cuda")
    xnor.xnor_w4_linear(empty, packed.wimg, torch.empty((0, 300), device="cuda"), None, 0, 2000, 300, 64)
