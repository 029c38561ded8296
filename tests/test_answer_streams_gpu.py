"""The making of 4-bit weights on a stream of its own, which is busy when it is called."""
import pytest
import torch

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
