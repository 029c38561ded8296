"""The real end of a network as it is used: norm, 4-bit classifier and log probabilities behind a binary layer, trained, captured in a graph, on
a stream of its own."""
import math

import pytest
import torch

from paper_1603_05279_amd import answer as ans
from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, assert_within, generator, normal

pytestmark = pytest.mark.gpu


def test_training_then_answering():
    got = ans.run(rows=512, inputs=512, width=256, classes=100, steps=31, report=lambda line: None)
    assert abs(got["losses"][0] - math.log(100)) < 1e-5             # (a classifier of zeros)
    assert got["losses"][-1] < got["losses"][0] / 4
    assert got["right"] > 0.9 and got["same"] > 0.9


def make(rows, width, classes, group, dtype):
    gen = generator(rows)
    head = xnor.W4Weights.quantized(normal(gen, classes, width, scale=0.05).cuda(), group, zeros=True)
    end = ans.Answer((torch.rand(width, generator=gen) + 0.5).cuda(), head, rows, dtype)
    x, residual = (normal(gen, rows, width).to(dtype).cuda() for _ in range(2))
    return end, x, residual, torch.randint(0, classes, (rows, 1), generator=gen).cuda()


def results(end):
    return [t.clone() for t in (end.logits, end.logprob, end.entropy, end.top_index, end.top_logprob)]


def blank(end):
    for t in (end.logits, end.logprob, end.entropy, end.top_logprob, end.scale):
        t.fill_(float("nan"))
    end.q.fill_(-128)
    end.top_index.fill_(-77)
    end.workspace.fill_(201)


# one row, few rows, rows staged first, narrow and wide classifiers
CASES = [(1, 512, 1000, 64, torch.bfloat16), (37, 1003, 1000, 32, torch.float32), (200, 1030, 4000, 128, torch.bfloat16), (600, 500, 8200, 64, torch.float16),
         (3, 256, 33000, 128, torch.bfloat16)]


@pytest.mark.parametrize("case", CASES)
def test_graph_replays_reproduce_eager_results(case):
    end, x, residual, tokens = make(*case)
    end(x, tokens, residual)
    torch.cuda.synchronize()
    eager = results(end)
    assert all(t.isfinite().all() for t in eager)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        end(x, tokens, residual)
    torch.cuda.synchronize()
    for replay in range(4):
        blank(end)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(end), eager)), replay
        end(x, tokens, residual)                                        # eager work between replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("case", CASES[:3])
def test_on_a_side_stream(case):
    end, x, residual, tokens = make(*case)
    end(x, tokens, residual)
    eager = results(end)
    blank(end)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    end(x, tokens, residual, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results(end), eager))


def test_training_gradients_in_a_graph_and_against_64_bits():
    gen = generator(5)
    rows, width, classes = 70, 130, 45
    norm_weight, weight = (torch.rand(width, generator=gen) + 0.5).cuda(), normal(gen, classes, width, scale=0.1).cuda()
    x, labels = normal(gen, rows, width).cuda(), torch.randint(0, classes, (rows, 1), generator=gen).cuda()
    end = ans.EndTraining(norm_weight, weight, rows, 64)
    end.gradients(x, labels)
    values = end.values.double().cpu()
    w = weight.double().cpu().requires_grad_()
    v = values.clone().requires_grad_()
    torch.log_softmax(v @ w.t(), 1).gather(1, labels.cpu()).mean().neg().backward()
    # sums of `rows` and of `classes` float32 products, and what the log probabilities are off by
    assert_within(end.g_weight, w.grad, 2 * (rows * EPS32 + 2e-5) * (2 / rows) * values.abs().sum(0)[None], "g_weight")
    h = x.double().cpu()
    h.requires_grad_()
    n = torch.ones(width, dtype=torch.float64) * norm_weight.double().cpu()
    n.requires_grad_()
    (h * (h.square().mean(1, keepdim=True) + ans.EPS).rsqrt() * n).backward(v.grad)
    top = v.grad.abs().amax(1, keepdim=True) + 2e-5 / rows
    assert_within(end.g_x, h.grad, 1e-4 * top * 4, "g_x")
    assert_within(end.g_norm_weight, n.grad, 1e-4 * (top * h.abs() * 2).sum(0).detach(), "g_norm_weight")
