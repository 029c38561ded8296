"""Workspaces of include/xnor_lowbit.h: one for the largest batch serves every smaller one."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import filled, generator, normal

ROWS = sorted(set(list(range(1, 700)) + [1000, 1023, 1024, 1025, 2048, 2049, 4095, 4097, 8191, 16384, 50000, 2 ** 20 - 1, 2 ** 20 + 1, 65535 * 64]))


@pytest.mark.parametrize("cin,out,group", [(4096, 16384, 128), (4096, 4096, 128), (9216, 4096, 32), (4097, 8192, 64), (1003, 1000, 32), (300, 500, 64), (1, 1, 32), (8538, 31744, 32)])
def test_products(cin, out, group):
    sizes = [xnor.w4_linear_workspace_bytes(r, cin, out, group) for r in ROWS]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("vocab", [1, 2048, 2049, 8192, 8193, 32000, 128000, 10 ** 6])
@pytest.mark.parametrize("top", [0, 1, 32])
def test_log_probabilities(vocab, top):
    sizes = [xnor.logprobs_workspace_bytes(r, vocab, top) for r in ROWS]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("cols", [1, 100, 512, 513, 4096, 4097, 9216, 32768])
def test_norm(cols):
    sizes = [xnor.rmsnorm_backward_workspace_bytes(r, cols) for r in ROWS]
    assert sizes == sorted(sizes)


def guarded(size):
    """A workspace of that size, and what must stay behind it."""
    whole = filled((size + 4096,), torch.uint8)
    return whole[:size], whole[size:]


@pytest.mark.gpu
@pytest.mark.parametrize("most,cin,out,group", [(128, 4096, 16384, 128), (300, 1030, 4000, 32), (260, 2048, 2050, 64)])
def test_fewer_rows_in_the_workspace_of_more(most, cin, out, group):
    gen = generator(most)
    packed = xnor.W4Weights.quantized(normal(gen, out, cin).cuda(), group)
    ws, behind = guarded(xnor.w4_linear_workspace_bytes(most, cin, out, group))
    for t in (torch.float32, torch.bfloat16):
        x = normal(gen, most, cin).to(t).cuda()
        for rows in (most, most - 1, most // 2 + 1, most // 2, 64, 65, 33, 1):
            y, alone = filled((rows, out), t), filled((rows, out), t)
            xnor.xnor_w4_linear(x[:rows], packed.wimg, y, ws, rows, cin, out, group)
            xnor.xnor_w4_linear(x[:rows], packed.wimg, alone, filled((xnor.w4_linear_workspace_bytes(rows, cin, out, group),), torch.uint8), rows, cin, out, group)
            assert torch.equal(y, alone) and (behind == 201).all()


@pytest.mark.gpu
def test_fewer_rows_of_log_probabilities_and_gradients_in_the_workspace_of_more():
    gen = generator(1)
    vocab, most = 20000, 600
    l, tokens = normal(gen, most, vocab).cuda(), torch.randint(0, vocab, (most, 1), generator=gen).cuda()
    for top in (0, 5):
        ws, behind = guarded(xnor.logprobs_workspace_bytes(most, vocab, top))
        for rows in (most, 512, 257, 256, 9, 1):
            lp, i, v = filled((rows, 1), torch.float32), filled((rows, top), torch.int32), filled((rows, top), torch.float32)
            xnor.xnor_logprobs(l[:rows], tokens[:rows], lp, None, None, None, i if top else None, v if top else None, ws, rows, vocab, 1, top)
            want = torch.log_softmax(l[:rows].double(), 1).gather(1, tokens[:rows])
            assert (lp - want).abs().max() < 2e-4 and (behind == 201).all()
    cols, most = 700, 3000
    h, rstd = normal(gen, most, cols).cuda(), torch.ones(most, device="cuda")
    ws, behind = guarded(xnor.rmsnorm_backward_workspace_bytes(most, cols))
    for rows in (most, 2049, 2048, 1025, 1024, 513, 3):
        g_h, g_w = filled((rows, cols), torch.float32), filled((cols,), torch.float32)
        xnor.xnor_rmsnorm_backward(h[:rows], rstd, None, h[:rows], None, g_h, g_w, ws, rows, cols)
        want = h[:rows].double().square().sum(0)
        assert ((g_w - want).abs() <= 1e-4 * want).all() and (behind == 201).all()
