"""Products of 8-bit rows with 8-bit weights against exact integer sums."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, assert_within, filled, generator, normal

pytestmark = pytest.mark.gpu


def product(q, xs, w, ws, bias, t):
    rows, cin = q.shape
    y = filled((rows, w.shape[0]), t)
    n = xnor.w8_linear_workspace_bytes(rows, cin, w.shape[0])
    xnor.xnor_w8_linear(q.cuda(), xs.cuda(), w.cuda(), ws.cuda(), None if bias is None else bias.cuda(), y, filled((n,), torch.uint8) if n else None, rows, cin,
                        w.shape[0])
    return y


def check(q, xs, w, ws, bias, name):
    """The sum to float32, the scales' product and both together: three roundings; the bias' addition; the result's type."""
    y = product(q, xs, w, ws, bias, TYPES[name])
    p = (q.double() @ w.double().t()) * (xs.double()[:, None] * ws.double())
    want = p if bias is None else p + bias.double()
    err = 3.01 * EPS32 * p.abs() + (0 if bias is None else EPS32 * want.abs())
    bound = err + (HALF_ULP[name] * (want.abs() + err) if name != "f32" else 0) + SMALLEST[name]
    # past the type's largest number a result rounds to that or to an infinity
    most = torch.finfo(TYPES[name]).max
    past = want.abs() > most * (1 - HALF_ULP[name])
    got = y.double().cpu()
    assert (got[past] * want[past].sign() >= most * (1 - 2 * HALF_ULP[name])).all()
    assert_within(got[~past], want[~past], bound[~past], "y")
    return y


def codes(gen, *shape):
    return torch.randint(-128, 128, shape, generator=gen, dtype=torch.int64).to(torch.int8)


def scales(gen, n):
    return torch.exp(2 * normal(gen, n)) / 100


SIZES = [(1, 1, 1), (1, 64, 16), (1, 9216, 100), (2, 15, 17), (3, 127, 1003), (16, 128, 64), (15, 1003, 33), (17, 256, 48), (32, 1000, 1000), (33, 513, 130), (40, 4096, 70),
         (64, 640, 256), (65, 144, 257), (96, 2048, 320), (128, 1024, 512), (129, 1003, 511), (200, 272, 1025), (256, 512, 256), (257, 1040, 513), (300, 333, 300), (513, 384, 260),
         (700, 1008, 777), (1024, 256, 768)]


@pytest.mark.parametrize("rows,cin,out", SIZES)
def test_product(rows, cin, out):
    for i, name in enumerate(TYPES):
        gen = generator(rows + cin + out + i)
        bias = normal(gen, out) if (i + rows) % 2 else None
        check(codes(gen, rows, cin), scales(gen, rows), codes(gen, out, cin), scales(gen, out), bias, name)


@pytest.mark.parametrize("rows", [1, 5, 70, 300])
def test_every_size_around_the_steps_of_the_instructions(rows):
    gen = generator(rows)
    for cin in list(range(1, 20)) + [31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 1023, 1024, 1025]:
        check(codes(gen, rows, cin), scales(gen, rows), codes(gen, 37, cin), scales(gen, 37), None, "f32")
    for out in list(range(1, 18)) + [255, 256, 257]:
        check(codes(gen, rows, 80), scales(gen, rows), codes(gen, out, 80), scales(gen, out), None, "f32")


def test_codes_that_depend_on_their_place():
    """Each weight alone: what is multiplied with what."""
    cin, out, rows = 300, 40, 20
    q = (torch.arange(rows)[:, None] * 7 + torch.arange(cin)[None] * 3) % 251 - 125
    w = torch.zeros((out, cin), dtype=torch.int8)
    w[torch.arange(out), (torch.arange(out) * 53) % cin] = 1
    y = product(q.to(torch.int8), torch.ones(rows), w, torch.ones(out), None, torch.float32)
    assert torch.equal(y.cpu(), q[:, (torch.arange(out) * 53) % cin].float())


@pytest.mark.parametrize("rows", [1, 64, 300])
def test_largest_sums(rows):
    """131071 products of -128 and -128: 2^31 - 2^14."""
    cin = 131071
    q, w = torch.full((rows, cin), -128, dtype=torch.int8), torch.full((17, cin), -128, dtype=torch.int8)
    y = product(q, torch.ones(rows), w, torch.ones(17), None, torch.float32)
    assert (y == 2.0 ** 31 - 2.0 ** 14).all()


@pytest.mark.parametrize("rows", [1, 300])
def test_scales_of_any_size(rows):
    """Their product may be outside of float32's range where the result is not, or the other way round."""
    gen = generator(4)
    cin = 64
    q, w = codes(gen, rows, cin), codes(gen, 24, cin)
    xs = torch.full((rows,), 2.0 ** 120)
    ws = torch.tensor([2.0 ** -140, 2.0 ** -100, 1.0, 0.0, 2.0 ** 5, 2.0 ** 20]).repeat(4)
    y = product(q, xs, w, ws, None, torch.float32).double().cpu()
    want = (q.double() @ w.double().t()) * (xs.double()[:, None] * ws.double())
    big = want.abs() > 3.4028235e38
    assert torch.equal(y[big].isinf(), torch.ones_like(y[big], dtype=torch.bool)) and not y.isnan().any()
    assert ((y - want).abs()[~big] <= 3.01 * EPS32 * want.abs()[~big] + 2.0 ** -149).all()


@pytest.mark.parametrize("rows", [3, 300])
def test_nan_stays_in_its_row_and_output(rows):
    gen = generator(5)
    q, w, xs, ws, bias = codes(gen, rows, 200), codes(gen, 50, 200), scales(gen, rows), scales(gen, 50), normal(gen, 50)
    xs[1], ws[7], bias[9] = float("nan"), float("inf"), float("nan")
    y = product(q, xs, w, ws, bias, torch.float32).cpu()
    bad = torch.zeros((rows, 50), dtype=torch.bool)
    bad[1], bad[:, 7], bad[:, 9] = True, True, True
    assert torch.equal(~y.isfinite(), bad)


def test_weights_from_real_ones():
    gen = generator(6)
    w = normal(gen, 70, 130)
    made = xnor.W8Weights(w.cuda())
    top = w.abs().amax(1)                                      # (on the CPU: the GPU's torch multiplies by a rounded 1 / 127)
    assert torch.equal(made.scale.cpu(), top / torch.tensor(127.0))
    assert torch.equal(made.codes.cpu(), torch.round(w * (127.0 / top)[:, None]).to(torch.int8))
    made.quantize(2 * w.cuda())
    assert torch.equal(made.scale.cpu(), 2 * top / torch.tensor(127.0))


def test_norm_then_product():
    """The 8-bit rows that the norm writes with one scale each."""
    gen = generator(7)
    rows, cin, out = 40, 300, 90
    x, w = normal(gen, rows, cin), normal(gen, out, cin)
    q, scale = filled((rows, cin), torch.int8), filled((rows, 1), torch.float32)
    xnor.xnor_rmsnorm_q8(x.cuda(), None, None, None, q, scale, None, None, rows, cin, 0, 1e-6)
    made = xnor.W8Weights(w.cuda())
    check(q.cpu(), scale.cpu().flatten(), made.codes.cpu(), made.scale.cpu(), None, "f32")


@pytest.mark.parametrize("rows,cin,out", [(1, 9216, 4096), (16, 4096, 4096), (256, 9216, 1024), (640, 2048, 1536)])
def test_the_same_bits_every_time(rows, cin, out):
    gen = generator(rows)
    args = codes(gen, rows, cin), scales(gen, rows), codes(gen, out, cin), scales(gen, out), normal(gen, out)
    first = product(*args, torch.bfloat16)
    assert all(torch.equal(product(*args, torch.bfloat16), first) for _ in range(3))


def test_results_past_32_bits_of_offset():
    rows, cin, out = 70000, 16, 32768
    gen = generator(8)
    q, w, xs, ws = codes(gen, rows, cin).cuda(), codes(gen, out, cin).cuda(), scales(gen, rows).cuda(), scales(gen, out).cuda()
    y = torch.full((rows, out), float("nan"), dtype=torch.bfloat16, device="cuda")
    n = xnor.w8_linear_workspace_bytes(rows, cin, out)
    xnor.xnor_w8_linear(q, xs, w, ws, None, y, filled((n,), torch.uint8) if n else None, rows, cin, out)
    for at in (slice(0, 64), slice(65500, 65600), slice(69940, 70000)):
        want = (q[at].double() @ w.double().t()) * (xs[at].double()[:, None] * ws.double())
        assert ((y[at].double() - want).abs() <= 1.001 * HALF_ULP["bf16"] * want.abs() + 1e-30).all()


def test_no_rows():
    y = torch.empty((0, 8), device="cuda")
    xnor.xnor_w8_linear(None, None, None, None, None, y, None, 0, 16, 8)
