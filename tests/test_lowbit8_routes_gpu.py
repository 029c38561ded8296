"""The 8-bit products, weight gradients and draws at sizes that reach each of their kernels, workspaces of more rows and their ends, captured and replayed.
The reference is the formula in 64 bits on the GPU (the products' sums are integers below 2^53: exact)."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, apart, assert_within, filled, generator, normal
from tests.test_weight_gradient_gpu import bounds, make, values

pytestmark = pytest.mark.gpu

GUARD = 4096


def guarded(nbytes):
    """`nbytes` between two guards."""
    whole = torch.full((nbytes + 2 * GUARD,), 201, dtype=torch.uint8, device="cuda")
    return whole, whole[GUARD:GUARD + nbytes] if nbytes else None


def untouched(whole):
    return bool((whole[:GUARD] == 201).all()) and bool((whole[-GUARD:] == 201).all())


def codes(gen, *shape):
    return torch.randint(-128, 128, shape, generator=gen, dtype=torch.int64).to(torch.int8).cuda()


# tiles of 256 with rows of whole 16 bytes and others, of 128 in one and in shares, few and many workgroups; rows in 16, 32, 64 at a time
PRODUCTS = [(2048, 4096, 8192), (1973, 2192, 8129), (1968, 1457, 8183), (2048, 4100, 8192), (13, 88, 201), (408, 64, 6628), (3, 64, 2076), (300, 4096, 1000),
            (300, 4100, 1000), (37, 5824, 4220), (71, 2192, 2781), (257, 8205, 2000), (1, 5639, 7917), (1, 608, 479), (7, 306, 90), (129, 2064, 1025),
            (256, 9216, 4096), (513, 2048, 4100), (4096, 1024, 4100)]


def product_error(y, q, xs, w, ws, name):
    want = (q.double() @ w.double().t().contiguous()) * (xs.double()[:, None] * ws.double())
    err = 3.01 * EPS32 * want.abs()
    over = (y.double() - want).abs() - err - (HALF_ULP[name] * (want.abs() + err) if name != "f32" else 0) - SMALLEST[name]
    return int((~(over <= 0)).sum())


@pytest.mark.parametrize("rows,cin,out", PRODUCTS)
def test_products(rows, cin, out):
    gen = generator(rows + out)
    q, w = codes(gen, rows, cin), codes(gen, out, cin)
    xs, ws = (torch.exp(normal(gen, n)).cuda() / 300 for n in (rows, out))
    n = xnor.w8_linear_workspace_bytes(rows, cin, out)
    for name in ("bf16", "f32"):
        space, work = guarded(n)
        whole = torch.full((rows + 2, out), float("nan"), dtype=TYPES[name], device="cuda")       # (a row behind the last, one more in front: 16 bytes for these types and outs)
        y = filled((rows, out), TYPES[name])
        xnor.xnor_w8_linear(q, xs, w, ws, None, y, work, rows, cin, out)
        assert product_error(y, q, xs, w, ws, name) == 0 and untouched(space)
        if out * whole.element_size() % 16 == 0:
            xnor.xnor_w8_linear(q, xs, w, ws, None, whole[1:-1], work, rows, cin, out)
            assert torch.equal(whole[1:-1], y) and bool(whole[0].isnan().all()) and bool(whole[-1].isnan().all())


@pytest.mark.parametrize("cin,out", [(4096, 1000), (9216, 4096), (5639, 7917)])
def test_a_workspace_of_more_rows_serves_fewer(cin, out):
    gen = generator(cin)
    w, ws = codes(gen, out, cin), torch.exp(normal(gen, out)).cuda() / 300
    space, work = guarded(xnor.w8_linear_workspace_bytes(700, cin, out))
    for rows in (700, 640, 385, 300, 256, 129, 128, 100, 37, 16, 1):
        assert xnor.w8_linear_workspace_bytes(rows, cin, out) <= xnor.w8_linear_workspace_bytes(700, cin, out)
        q, xs = codes(gen, rows, cin), torch.exp(normal(gen, rows)).cuda() / 300
        y = filled((rows, out), torch.float32)
        xnor.xnor_w8_linear(q, xs, w, ws, None, y, work, rows, cin, out)
        assert product_error(y, q, xs, w, ws, "f32") == 0 and untouched(space), rows


# sides of 64, 128 and 256 with one and two parts of each operand
GRADIENTS = [(1077, 33, 31), (18, 161, 46), (215, 36, 65), (1, 4196, 405), (12, 322, 5973), (2, 1050, 2431), (257, 2100, 2300), (266, 4556, 3575), (3, 3297, 4802),
             (2048, 4096, 8192), (1030, 4099, 4100), (1200, 100, 100), (1500, 65, 130),
             # few products: one launch, pairs of columns
             (5, 2, 2), (9, 3, 2), (40, 65, 2), (100, 2, 129), (33, 127, 63), (1, 371, 2011), (64, 1003, 1000), (129, 128, 192), (777, 1003, 1000)]


@pytest.mark.parametrize("name,wname", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cin,out", GRADIENTS)
def test_gradients(rows, cin, out, name, wname):
    group = (0, 128, 32)[(rows + cin) % 3]
    q, scale, g = (t.cuda() for t in make(generator(rows + cin), rows, cin, out, group, name))
    space, work = guarded(xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, group, TYPES[name], TYPES[wname]))
    g_w, g_b = filled((out, cin), TYPES[wname]), filled((out,), torch.float32)
    xnor.xnor_q8_weight_gradient(q, scale, g, g_w, g_b, work, rows, cin, out, group)
    x, d = values(q, scale, group), g.double()
    err, _ = bounds(x, d, name, wname)
    want = d.t().contiguous() @ x
    bound = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0)
    assert int((~((g_w.double() - want).abs() <= bound)).sum()) == 0 and untouched(space)
    assert_within(g_b, d.sum(0), ((rows + 4) * EPS32 * d.abs().sum(0)).cpu(), "g_bias")


@pytest.mark.parametrize("rows,cin,out,extra", [(1200, 100, 100, 0), (1200, 99, 101, 3), (300, 1100, 4200, 0), (65, 66, 67, 5), (40, 128, 64, 0), (3, 5, 7, 1)])
@pytest.mark.parametrize("name,wname", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_gradients_added_to_what_is_there(name, wname, rows, cin, out, extra):
    """Rows of the gradient further apart than they are long, and results added: the sum without them, one more addition and rounding."""
    group = (0, 128, 32)[(rows + cin) % 3]
    gen = generator(rows + out)
    q, scale, g = make(gen, rows, cin, out, group, name)
    q, scale, g = q.cuda(), scale.cuda(), apart(g, extra)
    n = xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, group, TYPES[name], TYPES[wname])
    g_w, g_b = normal(gen, out, cin).to(TYPES[wname]).cuda(), normal(gen, out).cuda()
    before = g_w.double(), g_b.double()
    xnor.xnor_q8_weight_gradient(q, scale, g, g_w, g_b, filled((n,), torch.uint8), rows, cin, out, group, accumulate=True)
    x, d = values(q, scale, group), g.double()
    err, _ = bounds(x, d, name, wname)
    want = d.t().contiguous() @ x + before[0]
    err = err + EPS32 * want.abs()
    bound = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0)
    assert int((~((g_w.double() - want).abs() <= bound)).sum()) == 0
    want = d.sum(0) + before[1]
    assert_within(g_b, want, ((rows + 4) * EPS32 * d.abs().sum(0) + EPS32 * want.abs()).cpu(), "g_bias")


@pytest.mark.parametrize("name,wname", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_gradients_with_scales_of_rows_of_any_size(name, wname):
    """Scales of 2^-140 to 2^120 on rows whose gradients are as much the other way: each product counts by its own size, wherever its factors lie."""
    gen = generator(21)
    rows, cin, out = 200, 140, 90
    q, scale, g = make(gen, rows, cin, out, 0, "f32")
    most = 10 if name == "f16" else 100
    tilt = torch.linspace(-most, most, rows)[:, None]
    scale, g = (scale * 2.0 ** -tilt).cuda(), (g * 2.0 ** tilt).to(TYPES[name]).cuda()
    q = q.cuda()
    work = filled((xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, 0, TYPES[name], TYPES[wname]),), torch.uint8)
    g_w = filled((out, cin), TYPES[wname])
    xnor.xnor_q8_weight_gradient(q, scale, g, g_w, None, work, rows, cin, out, 0)
    both = g.double() * scale.double()
    total = both.abs().t().contiguous() @ q.double().abs()
    want = both.t().contiguous() @ q.double()
    # the product of both rounded once, kept in one or two floats of 11 bits; the sums; 2^-40 of a column's largest for each row
    err = total * ((2.0 ** -11 if wname == "bf16" else 2.0 ** -22) * 1.001 + EPS32 + 2 * EPS32 * (rows / 16 + 18)) + 2.0 ** -39 * rows * 127 * both.abs().amax(0)[:, None]
    bound = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0)
    assert int((~((g_w.double() - want).abs() <= bound)).sum()) == 0


def test_a_row_scale_that_is_not_finite_and_products_past_the_largest_number():
    gen = generator(22)
    rows, cin, out = 70, 50, 40
    q, scale, g = make(gen, rows, cin, out, 0, "f32")
    q[q == 0], g[g == 0] = 1, 1.0
    q[3] = 0
    q[3, 7] = -2
    scale[3], g[3, 5] = 2.0 ** 100, 2.0 ** 100                     # (the other columns of g: 2^100 as much as before)
    work = filled((xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, 0, torch.float32, torch.float32),), torch.uint8)
    g_w = filled((out, cin), torch.float32)
    xnor.xnor_q8_weight_gradient(q.cuda(), scale.cuda(), g.cuda(), g_w, None, work, rows, cin, out, 0)
    past = torch.zeros((out, cin), dtype=torch.bool)
    past[5, 7] = True                                              # the one sum of 2^201; zeros of q leave nothing behind
    assert torch.equal(g_w.cpu() == -float("inf"), past) and bool(g_w.cpu()[~past].isfinite().all())
    for value in (float("inf"), float("nan")):
        scale[3] = value
        xnor.xnor_q8_weight_gradient(q.cuda(), scale.cuda(), g.cuda(), g_w, None, work, rows, cin, out, 0)
        assert not bool(g_w.isfinite().any())


def replayed(call, outputs, scratch, other):
    """What `call` leaves in `outputs`, eagerly, is what a captured one leaves each time, with eager work of `other` in the same workspaces between."""
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.synchronize()
    for replay in range(4):
        other()
        for t in scratch:
            t.fill_(201)
        for t in outputs:
            t.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want)), replay
    return want


@pytest.mark.parametrize("rows,cin,out", [(300, 4100, 1000), (71, 2192, 2781), (13, 88, 201), (1973, 2192, 8129)])
def test_captured_products(rows, cin, out):
    gen = generator(rows)
    q, w, xs, ws = codes(gen, rows, cin), codes(gen, out, cin), torch.rand(rows, generator=gen).cuda(), torch.rand(out, generator=gen).cuda()
    n = xnor.w8_linear_workspace_bytes(rows, cin, out)
    work = filled((max(n, 1),), torch.uint8)
    y, y2, q2 = filled((rows, out), torch.float32), filled((rows, out), torch.float32), codes(gen, rows, cin)
    replayed(lambda: xnor.xnor_w8_linear(q, xs, w, ws, None, y, work, rows, cin, out), [y], [work],
             lambda: xnor.xnor_w8_linear(q2, xs, w, ws, None, y2, work, rows, cin, out))


@pytest.mark.parametrize("rows,cin,out,name,wname", [(100, 300, 400, "bf16", "bf16"), (257, 2100, 2300, "f32", "f32"), (3, 3297, 4802, "bf16", "f32")])
def test_captured_gradients(rows, cin, out, name, wname):
    q, scale, g = (t.cuda() for t in make(generator(rows), rows, cin, out, 0, name))
    work = filled((xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, 0, TYPES[name], TYPES[wname]),), torch.uint8)
    g_w, g_b, g_w2 = filled((out, cin), TYPES[wname]), filled((out,), torch.float32), filled((out, cin), TYPES[wname])
    g2 = (g * 3).contiguous()
    replayed(lambda: xnor.xnor_q8_weight_gradient(q, scale, g, g_w, g_b, work, rows, cin, out, 0), [g_w, g_b], [work],
             lambda: xnor.xnor_q8_weight_gradient(q, scale, g2, g_w2, None, work, rows, cin, out, 0))


@pytest.mark.parametrize("rows,vocab,top_k", [(1, 128000, False), (5, 100003, False), (2, 128000, True), (300, 9000, False), (3, 100, True)])
def test_captured_draws(rows, vocab, top_k):
    gen = generator(rows)
    logits, other = ((3 * normal(gen, rows, vocab)).to(torch.bfloat16).cuda() for _ in range(2))
    uniform, p = torch.rand(rows, generator=gen).cuda(), torch.full((rows,), 0.95, device="cuda")
    k = torch.full((rows,), 40, dtype=torch.int32, device="cuda") if top_k else None
    space, work = guarded(max(xnor.sample_workspace_bytes(rows, vocab), 16))
    token, kept, token2 = (filled((rows,), torch.int32) for _ in range(3))
    logprob = filled((rows,), torch.float32)
    replayed(lambda: xnor.xnor_sample(logits, None, k, p, None, uniform, token, logprob, kept, work, rows, vocab), [token, logprob, kept], [work],
             lambda: xnor.xnor_sample(other, None, None, None, None, uniform, token2, None, None, work, rows, vocab))
    assert untouched(space) and bool((token2 >= 0).all())


def test_draws_of_fewer_rows_in_a_workspace_of_more():
    vocab = 60001
    gen = generator(8)
    logits, uniform = (2 * normal(gen, 100, vocab)).cuda(), torch.rand(100, generator=gen).cuda()
    space, work = guarded(xnor.sample_workspace_bytes(100, vocab))
    want = None
    for rows in (100, 33, 32, 31, 17, 16, 15, 2, 1):
        assert xnor.sample_workspace_bytes(rows, vocab) <= xnor.sample_workspace_bytes(100, vocab)
        token, kept = filled((rows,), torch.int32), filled((rows,), torch.int32)
        xnor.xnor_sample(logits, None, None, torch.full((rows,), 0.9, device="cuda"), None, uniform, token, None, kept, work, rows, vocab)
        want = (token, kept) if want is None else want
        assert torch.equal(token, want[0][:rows]) and torch.equal(kept, want[1][:rows]) and untouched(space), rows
