"""The training step and the making of 4-bit weights on a stream of their own, which is busy when they are called."""
import pytest
import torch

from paper_1603_05279_amd import answer as ans
from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import generator, normal

pytestmark = pytest.mark.gpu


def busy_stream():
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = torch.ones((4096, 4096), device="cuda")
        for _ in range(20):
            a = a @ a * 2.0 ** -12
    return side


def test_gradients_on_a_busy_stream():
    gen = generator(6)
    rows, width, classes = 300, 260, 2100
    norm_weight, weight = (torch.rand(width, generator=gen) + 0.5).cuda(), normal(gen, classes, width, scale=0.1).cuda()
    x, labels = normal(gen, rows, width).cuda(), torch.randint(0, classes, (rows, 1), generator=gen).cuda()
    end = ans.EndTraining(norm_weight, weight, rows, 64)
    names = ("g_x", "g_norm_weight", "g_weight", "g_logits", "logprob", "values")
    end.gradients(x, labels)
    want = {n: getattr(end, n).clone() for n in names}
    for n in names:
        getattr(end, n).fill_(float("nan"))
    for _ in range(3):
        side = busy_stream()
        end.gradients(x, labels, stream=side)
        noise = [torch.full((rows, classes), float("nan"), device="cuda") for _ in range(4)]        # (the current stream's memory is used again)
        side.synchronize()
        assert all(torch.equal(getattr(end, n), want[n]) for n in names) and noise
    torch.cuda.synchronize()


@pytest.mark.parametrize("raw", [False, True])
def test_weights_made_on_a_busy_stream(raw):
    class Handle:                               # what the library's calls take: anything with a stream's address
        def __init__(self, stream):
            self.cuda_stream = stream.cuda_stream

    w = normal(generator(7), 4000, 1003).cuda()
    want = xnor.W4Weights.quantized(w, 64, zeros=True).wimg.clone()
    for _ in range(3):
        side = busy_stream()
        made = xnor.W4Weights.quantized(w, 64, zeros=True, stream=Handle(side) if raw else side)
        noise = [torch.full((4000, 32 * 16), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        side.synchronize()
        assert torch.equal(made.wimg, want) and noise
    torch.cuda.synchronize()
