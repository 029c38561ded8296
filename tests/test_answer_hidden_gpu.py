"""The end with a hidden layer in 8 bits as it is used: trained, captured in a graph, on a stream of its own, answering and drawing."""
import math

import pytest
import torch

from paper_1603_05279_amd import answer as ans
from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, assert_within, generator, normal

pytestmark = pytest.mark.gpu

# rows, width, inner, classes, gated, function: one row, few, ones with tiles of each kind, odd sizes
CASES = [(1, 512, 256, 1000, False, "gelu", torch.bfloat16), (37, 1003, 131, 1000, True, "silu", torch.float32), (200, 1030, 520, 4000, False, "relu", torch.bfloat16),
         (600, 512, 1024, 2048, True, "gelu", torch.float16)]
TRAINED = [(70, 130, 96, 45, False, "gelu", 0), (300, 260, 131, 2100, True, "silu", 32), (65, 512, 512, 1000, False, "relu", 128)]


def busy_stream():
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = torch.ones((4096, 4096), device="cuda")
        for _ in range(20):
            a = a @ a * 2.0 ** -12
    return side


def make(rows, width, inner, classes, gated, function, dtype):
    gen = generator(rows + inner)
    hidden, head = normal(gen, inner * (1 + gated), width, scale=width ** -0.5), normal(gen, classes, inner, scale=inner ** -0.5)
    end = ans.HiddenAnswer((torch.rand(width, generator=gen) + 0.5).cuda(), xnor.W8Weights(hidden.cuda()), xnor.W8Weights(head.cuda()), rows, function, gated, dtype)
    x, residual = (normal(gen, rows, width).to(dtype).cuda() for _ in range(2))
    return end, x, residual, torch.randint(0, classes, (rows, 1), generator=gen).cuda(), torch.rand(rows, generator=gen).cuda()


def answer_and_draw(end, x, residual, tokens, uniform, stream=None):
    end(x, tokens, residual, stream)
    end.drawn(end.logits, uniform, stream=stream)


def results(end):
    return [t.clone() for t in (end.before, end.logits, end.logprob, end.entropy, end.top_index, end.top_logprob, end.drawn.token, end.drawn.logprob, end.drawn.kept)]


def blank(end):
    for t in (end.before, end.logits, end.logprob, end.entropy, end.top_logprob, end.scale, end.inner_scale, end.drawn.logprob):
        t.fill_(float("nan"))
    for t in (end.q, end.inner_q, end.top_index, end.drawn.token, end.drawn.kept):
        t.fill_(-77)
    end.workspace.fill_(201)
    end.drawn.workspace.fill_(201)


@pytest.mark.parametrize("case", CASES)
def test_graph_replays_reproduce_eager_results(case):
    end, *given = make(*case)
    answer_and_draw(end, *given)
    torch.cuda.synchronize()
    eager = results(end)
    assert all(t.isfinite().all() for t in eager) and bool((end.drawn.token >= 0).all())
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        answer_and_draw(end, *given)
    torch.cuda.synchronize()
    for replay in range(4):
        blank(end)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(end), eager)), replay
        answer_and_draw(end, *given)                                    # eager work between replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("case", CASES)
def test_on_a_busy_stream(case):
    end, *given = make(*case)
    answer_and_draw(end, *given)
    eager = results(end)
    for _ in range(2):
        blank(end)
        side = busy_stream()
        answer_and_draw(end, *given, stream=side)
        noise = [torch.full_like(end.logits, float("nan")) for _ in range(4)]       # (the current stream's memory is used again)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(end), eager)) and noise
    torch.cuda.synchronize()


def training(rows, width, inner, classes, gated, function, group):
    gen = generator(rows + classes)
    hidden, head = normal(gen, inner * (1 + gated), width, scale=width ** -0.5).cuda(), normal(gen, classes, inner, scale=inner ** -0.5).cuda()
    x, labels = normal(gen, rows, width).cuda(), torch.randint(0, classes, (rows, 1), generator=gen).cuda()
    return ans.HiddenTraining((torch.rand(width, generator=gen) + 0.5).cuda(), hidden, head, rows, function, gated, group), x, labels


@pytest.mark.parametrize("case", TRAINED)
def test_gradients_against_64_bits(case):
    """Each gradient from the 8-bit rows and the float32 gradient before it, by the formula in 64 bits."""
    rows, width, inner, classes, gated, function, group = case
    end, x, labels = training(*case)
    end.gradients(x, labels)
    d = lambda t: t.double().cpu()
    before = (d(end.q) @ d(end.hidden8.codes).t()) * d(end.scale) * d(end.hidden8.scale)
    assert_within(end.before, before, 4 * EPS32 * before.abs(), "before")
    logits = (d(end.inner_q) @ d(end.head8.codes).t()) * d(end.inner_scale) * d(end.head8.scale)
    assert_within(end.logits, logits, 4 * EPS32 * logits.abs(), "logits")
    want = torch.softmax(logits, 1)
    want[torch.arange(rows), labels.cpu().flatten()] -= 1
    g_logits = d(end.g_logits)
    assert_within(end.g_logits, want / rows, 2e-5 / rows, "g_logits")
    # sums of `rows` float32 products of a row's value and a gradient's, both to 2^-21
    inner_rows, first_rows = d(end.inner_q) * d(end.inner_scale), d(end.q) * d(end.scale)
    assert_within(end.g_head, g_logits.t() @ inner_rows, (rows + 16) * EPS32 * (g_logits.abs().t() @ inner_rows.abs()) + 1e-12, "g_head")
    g_inner = g_logits @ d(end.head)
    wide = inner * (1 + gated)
    size = group or wide
    kept = d(end.kept) * d(end.kept_scale).repeat_interleave(size, 1)[:, :wide]
    kept.requires_grad_()
    f = {"relu": torch.relu, "gelu": lambda v: 0.5 * v * torch.special.erfc(v * -0.5 ** 0.5), "silu": torch.nn.functional.silu}[function]
    value = f(kept[:, :inner]) * (kept[:, inner:] if gated else 1.0)
    value.backward(g_inner)
    # the product that makes g_inner is off by classes float32 roundings of its terms, the slope by 64 of its own
    off = (classes * EPS32 * (g_logits.abs() @ d(end.head).abs()) + 128 * EPS32 * g_inner.abs()) * 4 * (1 + kept.detach().abs().max())
    assert_within(end.g_before, kept.grad, off.repeat(1, 1 + gated) + 1e-12, "g_before")
    g_before = d(end.g_before)
    assert_within(end.g_hidden, g_before.t() @ first_rows, (rows + 16) * EPS32 * (g_before.abs().t() @ first_rows.abs()) + 1e-12, "g_hidden")
    h, n = d(x).requires_grad_(), d(end.norm_weight).requires_grad_()
    (h * (h.square().mean(1, keepdim=True) + ans.EPS).rsqrt() * n).backward(g_before @ d(end.hidden))
    top = h.grad.abs().amax(1, keepdim=True)
    assert_within(end.g_x, h.grad, 1e-4 * 4 * top, "g_x")
    assert_within(end.g_norm_weight, n.grad, 1e-4 * (4 * top * h.abs() * 2).sum(0).detach(), "g_norm_weight")


NAMES = ("g_x", "g_norm_weight", "g_hidden", "g_head", "g_before", "g_logits", "logprob")


@pytest.mark.parametrize("case", TRAINED)
def test_a_captured_step_beside_eager_ones(case):
    """Captured after an eager pass, replayed with eager passes of other inputs between: gradients are the eager ones each time."""
    end, x, labels = training(*case)
    end.gradients(x, labels)
    want = {n: getattr(end, n).clone() for n in NAMES}
    assert all(t.isfinite().all() for t in want.values())
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                       # (the products' library sets up its workspace of this stream)
        end.gradients(x, labels)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        end.gradients(x, labels)
    torch.cuda.synchronize()
    other = x.flip(0).contiguous() * 2
    for replay in range(3):
        end.gradients(other, labels)
        end.workspace.fill_(201)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(end, n), want[n]) for n in NAMES), replay


@pytest.mark.parametrize("case", TRAINED)
def test_training_on_a_busy_stream(case):
    end, x, labels = training(*case)
    end.gradients(x, labels)
    want = {n: getattr(end, n).clone() for n in NAMES}
    for _ in range(2):
        for n in NAMES:
            getattr(end, n).fill_(float("nan"))
        side = busy_stream()
        end.gradients(x, labels, stream=side)
        noise = [torch.full_like(end.g_logits, float("nan")) for _ in range(4)]
        side.synchronize()
        assert all(torch.equal(getattr(end, n), want[n]) for n in NAMES) and noise
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,inputs,width,classes,hidden,gated", [(1, 64, 32, 2, 33, False), (77, 100, 65, 9, 64, True), (301, 333, 130, 41, 128, False)])
def test_the_command_runs(rows, inputs, width, classes, hidden, gated):
    got = ans.run(rows=rows, inputs=inputs, width=width, classes=classes, steps=2, hidden=hidden, gated=gated, report=lambda line: None)
    assert abs(got["losses"][0] - math.log(classes)) < 1e-5             # (a classifier of zeros)
    assert math.isfinite(got["losses"][-1])
    if rows > 1:                                                        # (the only row's class is not the one learned: means over no rows, 0 / 0)
        assert math.isfinite(got["logprob"]) and 0 <= got["drawn"] <= 1


def test_the_4_bit_end_draws():
    """Draws from the 4-bit end's logits: the likeliest token at temperature 0, one of the three likeliest with top_k."""
    gen = generator(9)
    rows, width, classes = 40, 256, 300
    head = xnor.W4Weights.quantized(normal(gen, classes, width, scale=0.05).cuda(), 64, zeros=True)
    end = ans.Answer(torch.ones(width, device="cuda"), head, rows)
    end(normal(gen, rows, width).cuda(), torch.zeros((rows, 1), dtype=torch.int64, device="cuda"))
    uniform = torch.rand(rows, generator=gen).cuda()
    end.drawn(end.logits, uniform, torch.zeros(rows, device="cuda"))
    assert torch.equal(end.drawn.token, end.top_index[:, 0]) and bool((end.drawn.logprob == 0).all())
    end.drawn(end.logits, uniform, top_k=torch.full((rows,), 3, dtype=torch.int32, device="cuda"))
    assert bool((end.drawn.token[:, None] == end.top_index[:, :3]).any(1).all()) and bool((end.drawn.kept == 3).all())
