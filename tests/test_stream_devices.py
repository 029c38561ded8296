"""A stream of another device than a call's tensors is refused before anything is launched: a kernel there would read memory that its device does not hold."""
import pytest
import torch

from paper_1603_05279_amd import xnor


class OtherStream:
    """A stream's handle and device, as torch.cuda.Stream has them."""
    cuda_stream = 0

    def __init__(self, index):
        self.device = torch.device("cuda", index)


@pytest.mark.gpu
def test_streams_of_other_devices():
    def new(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    x, q, scale, g_w, token = new(2, 64), new(2, 64, dtype=torch.int8), new(2), new(64, 64), new(2, dtype=torch.int32)
    work = new(xnor.q8_weight_gradient_workspace_bytes(2, 64, 64, 0, torch.float32, torch.float32), dtype=torch.uint8)
    calls = [lambda s: xnor.xnor_q8_rows(x, q, scale, 2, 64, 0, stream=s),
             lambda s: xnor.xnor_w8_linear(q, scale, q, scale, None, new(2, 2), None, 2, 64, 2, stream=s),
             lambda s: xnor.xnor_activation_q8(x, x, None, None, None, None, 2, 64, 0, 0, "relu", stream=s),
             lambda s: xnor.xnor_activation_backward(q, scale, x, x, 2, 64, 0, "relu", stream=s),
             lambda s: xnor.xnor_q8_weight_gradient(q, scale, x, g_w, None, work, 2, 64, 64, 0, stream=s),
             lambda s: xnor.xnor_sample(x, None, None, None, None, scale, token, None, None, None, 2, 64, stream=s)]
    here = x.device.index
    for call in calls:
        call(OtherStream(here))
        call(torch.cuda.current_stream())
        with pytest.raises(ValueError, match="device"):
            call(OtherStream(here + 1))
    torch.cuda.synchronize()
