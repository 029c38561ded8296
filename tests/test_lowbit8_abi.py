"""Refusals of the 8-bit layers and of the draw: status codes before anything is launched, and the binding's checks of tensors (no GPU)."""
import ctypes

import pytest
import torch

from paper_1603_05279_amd import xnor

NULL, SHAPE, UNSUPPORTED, ALIGN = -1, -2, -3, -4
FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)     # never dereferenced


def rows8(x=FAKE, xs=64, q=FAKE, s=FAKE, rows=2, cols=64, group=0, type=1):
    return xnor.lib().xnor_q8_rows(x, xs, q, s, rows, cols, group, type, None)


def product(q=FAKE, xs=FAKE, w=FAKE, ws=FAKE, b=None, y=FAKE, work=FAKE, rows=2, cin=64, out=4, type=0):
    return xnor.lib().xnor_w8_linear(q, xs, w, ws, b, y, work, rows, cin, out, type, None)


def activation(x=FAKE, xs=64, y=FAKE, q=None, s=None, k=None, ks=None, rows=2, cols=64, group=0, kept_group=0, f=0, gated=0, type=1):
    return xnor.lib().xnor_activation_q8(x, xs, y, q, s, k, ks, rows, cols, group, kept_group, f, gated, type, None)


def backward(k=FAKE, ks=FAKE, g=FAKE, gs=64, gx=FAKE, rows=2, cols=64, kept_group=0, f=0, gated=0, type=1):
    return xnor.lib().xnor_activation_backward(k, ks, g, gs, gx, rows, cols, kept_group, f, gated, type, None)


def gradient(q=FAKE, s=FAKE, g=FAKE, gs=4, gw=FAKE, gb=None, acc=0, work=FAKE, rows=2, cin=64, out=4, group=0, type=0, w_type=0):
    return xnor.lib().xnor_q8_weight_gradient(q, s, g, gs, gw, gb, acc, work, rows, cin, out, group, type, w_type, None)


def sample(l=FAKE, ls=64, t=None, k=None, p=None, m=None, u=FAKE, token=FAKE, lp=None, n=None, work=FAKE, rows=2, vocab=64, type=0):
    return xnor.lib().xnor_sample(l, ls, t, k, p, m, u, token, lp, n, work, rows, vocab, type, None)


MOST = 65535 * 64


@pytest.mark.parametrize("call,status,bad", [
    (rows8, NULL, dict(x=None)), (rows8, NULL, dict(q=None)), (rows8, NULL, dict(s=None)), (rows8, SHAPE, dict(rows=-1)), (rows8, SHAPE, dict(rows=MOST + 1)),
    (rows8, SHAPE, dict(cols=0)), (rows8, SHAPE, dict(cols=2 ** 24 + 1, xs=2 ** 25)), (rows8, SHAPE, dict(xs=63)), (rows8, UNSUPPORTED, dict(group=16)),
    (rows8, UNSUPPORTED, dict(group=-1)), (rows8, UNSUPPORTED, dict(type=3)), (rows8, ALIGN, dict(x=ODD)), (rows8, ALIGN, dict(q=ODD)), (rows8, ALIGN, dict(s=ODD)),
    (rows8, 0, dict(rows=0, x=None)),
    (product, NULL, dict(q=None)), (product, NULL, dict(xs=None)), (product, NULL, dict(w=None)), (product, NULL, dict(ws=None)), (product, NULL, dict(y=None)),
    (product, SHAPE, dict(rows=-1)), (product, SHAPE, dict(rows=MOST + 1)), (product, SHAPE, dict(cin=0)), (product, SHAPE, dict(out=-3)),
    (product, SHAPE, dict(out=2 ** 24 + 1)), (product, SHAPE, dict(cin=2 ** 24 + 1)), (product, UNSUPPORTED, dict(cin=131072)), (product, UNSUPPORTED, dict(type=-1)),
    (product, ALIGN, dict(q=ODD)), (product, ALIGN, dict(w=ODD)), (product, ALIGN, dict(ws=ODD)), (product, ALIGN, dict(b=ODD)), (product, ALIGN, dict(y=ODD)),
    (product, ALIGN, dict(work=ODD)), (product, 0, dict(rows=0, q=None, y=None)),
    (activation, NULL, dict(x=None)), (activation, NULL, dict(y=None)), (activation, NULL, dict(q=FAKE)), (activation, NULL, dict(k=FAKE)),
    (activation, SHAPE, dict(rows=-1)), (activation, SHAPE, dict(cols=0)), (activation, SHAPE, dict(cols=2 ** 23 + 1, xs=2 ** 24)), (activation, SHAPE, dict(xs=63)),
    (activation, SHAPE, dict(gated=1, xs=127)), (activation, UNSUPPORTED, dict(group=8)), (activation, UNSUPPORTED, dict(kept_group=256)),
    (activation, UNSUPPORTED, dict(f=3)), (activation, UNSUPPORTED, dict(f=-1)), (activation, UNSUPPORTED, dict(gated=2, xs=256)),
    (activation, UNSUPPORTED, dict(gated=-1)), (activation, UNSUPPORTED, dict(type=7)), (activation, ALIGN, dict(x=ODD)), (activation, ALIGN, dict(y=ODD)),
    (activation, ALIGN, dict(q=FAKE, s=ODD)), (activation, ALIGN, dict(k=ODD, ks=FAKE)), (activation, 0, dict(rows=0, x=None, y=None)),
    (backward, NULL, dict(k=None)), (backward, NULL, dict(ks=None)), (backward, NULL, dict(g=None)), (backward, NULL, dict(gx=None)), (backward, SHAPE, dict(gs=63)),
    (backward, SHAPE, dict(rows=MOST + 1)), (backward, SHAPE, dict(cols=-1)), (backward, UNSUPPORTED, dict(f=4)), (backward, UNSUPPORTED, dict(gated=3)),
    (backward, UNSUPPORTED, dict(kept_group=1)), (backward, UNSUPPORTED, dict(type=3)), (backward, ALIGN, dict(g=ODD)), (backward, ALIGN, dict(gx=ODD)),
    (backward, SHAPE, dict(rows=MOST, cols=2 ** 14, gs=2 ** 14)), (backward, 0, dict(rows=0, k=None)),
    (gradient, SHAPE, dict(cin=2 ** 24, out=2 ** 12, gs=2 ** 12)), (gradient, NULL, dict(q=None)), (gradient, NULL, dict(s=None)), (gradient, NULL, dict(g=None)), (gradient, NULL, dict(gw=None)), (gradient, NULL, dict(work=None)),
    (gradient, NULL, dict(rows=0, gw=None)), (gradient, SHAPE, dict(rows=-1)), (gradient, SHAPE, dict(cin=0)), (gradient, SHAPE, dict(out=0)),
    (gradient, SHAPE, dict(out=2 ** 24 + 1, gs=2 ** 25)), (gradient, SHAPE, dict(gs=3)), (gradient, UNSUPPORTED, dict(acc=2)), (gradient, UNSUPPORTED, dict(group=33)),
    (gradient, UNSUPPORTED, dict(type=3)), (gradient, UNSUPPORTED, dict(w_type=-1)), (gradient, ALIGN, dict(gw=ODD)), (gradient, ALIGN, dict(gb=ODD)),
    (gradient, ALIGN, dict(work=ODD)), (gradient, ALIGN, dict(q=ODD)), (gradient, 0, dict(rows=0, acc=1, gw=None)),
    (sample, NULL, dict(l=None)), (sample, NULL, dict(u=None)), (sample, NULL, dict(token=None)), (sample, SHAPE, dict(rows=-1)), (sample, SHAPE, dict(vocab=0)),
    (sample, SHAPE, dict(vocab=2 ** 30 + 1, ls=2 ** 31)), (sample, SHAPE, dict(ls=63)), (sample, UNSUPPORTED, dict(type=3)), (sample, ALIGN, dict(l=ODD)),
    (sample, ALIGN, dict(t=ODD)), (sample, ALIGN, dict(k=ODD)), (sample, ALIGN, dict(p=ODD)), (sample, ALIGN, dict(m=ODD)), (sample, ALIGN, dict(u=ODD)),
    (sample, ALIGN, dict(token=ODD)), (sample, ALIGN, dict(lp=ODD)), (sample, ALIGN, dict(n=ODD)), (sample, ALIGN, dict(work=ODD)), (sample, 0, dict(rows=0, l=None, u=None)),
])
def test_status(call, status, bad):
    assert call(**bad) == status


ROWS = sorted(set(list(range(1, 700)) + [1000, 1023, 1024, 1025, 2048, 2049, 4095, 4097, 8191, 16384, 50000, 2 ** 20 - 1, 2 ** 20 + 1, MOST]))


@pytest.mark.parametrize("cin,out", [(4096, 4096), (9216, 4096), (1003, 1000), (64, 16), (1, 1), (131071, 33), (256, 32000), (4100, 129)])
def test_workspaces_of_more_rows_serve_fewer(cin, out):
    sizes = [xnor.w8_linear_workspace_bytes(r, cin, out) for r in ROWS]
    assert sizes == sorted(sizes)
    for group in (0, 64):
        for t, wt in ((torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)):
            sizes = [xnor.q8_weight_gradient_workspace_bytes(r, cin, out, group, t, wt) for r in ROWS]
            assert sizes == sorted(sizes) and sizes[0] > 0
    sizes = [xnor.sample_workspace_bytes(r, cin) for r in ROWS]
    assert sizes == sorted(sizes)


def test_sizes_that_are_refused_need_nothing():
    assert xnor.w8_linear_workspace_bytes(0, 64, 64) == xnor.w8_linear_workspace_bytes(4, 131072, 64) == 0
    assert xnor.q8_weight_gradient_workspace_bytes(4, 64, 64, 16, torch.float32, torch.float32) == 0
    assert xnor.q8_weight_gradient_workspace_bytes(0, 64, 64, 32, torch.float32, torch.float32) == 0
    assert xnor.sample_workspace_bytes(-1, 64) == xnor.sample_workspace_bytes(4, 0) == 0


class _Stream:
    cuda_stream = 0


def test_tensors_on_the_host_or_of_another_type():
    x, q = torch.zeros((2, 64)), torch.zeros((2, 64), dtype=torch.int8)
    with pytest.raises(ValueError, match="device"):
        xnor.xnor_q8_rows(x, q, x, 2, 64, 0, stream=_Stream())
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        xnor.xnor_q8_rows(q, q, x, 2, 64, 0, stream=_Stream())
    with pytest.raises(ValueError, match="device"):
        xnor.xnor_w8_linear(q, x, q, x, None, x, None, 2, 64, 2, stream=_Stream())
    with pytest.raises(TypeError):
        xnor.xnor_sample(None, None, None, None, None, x, x, None, None, None, 2, 64, stream=_Stream())
    with pytest.raises(KeyError):
        xnor.xnor_activation_q8(x, x, None, None, None, None, 2, 64, 0, 0, "tanh", stream=_Stream())


@pytest.mark.gpu
def test_tensors_that_hold_less_than_the_sizes_say():
    def new(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    x, q, i8 = new(2, 64), new(2, 64, dtype=torch.int8), torch.int8
    short = pytest.raises(ValueError, match="holds less")
    for rows, cols, group in ((3, 64, 0), (2, 65, 0), (2, 64, 32)):
        with short:
            xnor.xnor_q8_rows(x, q, new(2), rows, cols, group)
    with short:
        xnor.xnor_w8_linear(q, new(2), new(3, 64, dtype=i8), new(4), None, new(2, 4), None, 2, 64, 4)
    with short:
        xnor.xnor_w8_linear(q, new(2), new(4, 64, dtype=i8), new(4), new(3), new(2, 4), None, 2, 64, 4)
    with short:
        xnor.xnor_activation_q8(x, new(2, 64), None, None, None, None, 2, 64, 0, 0, "relu", True)
    with short:
        xnor.xnor_activation_q8(x, None, None, None, q, new(2), 2, 64, 0, 32, "relu")
    with short:
        xnor.xnor_activation_backward(q, new(2), x, x, 2, 64, 64, "relu", True)
    work = new(xnor.q8_weight_gradient_workspace_bytes(2, 64, 8, 0, torch.float32, torch.float32) - 1, dtype=torch.uint8)
    with short:
        xnor.xnor_q8_weight_gradient(q, new(2), new(2, 8), new(8, 64), None, work, 2, 64, 8, 0)
    with short:
        xnor.xnor_sample(x, None, None, None, None, new(1), new(2, dtype=torch.int32), None, None, None, 2, 64)
    with pytest.raises(ValueError, match="Int"):
        xnor.xnor_sample(x, None, new(2), None, None, new(2), new(2, dtype=torch.int32), None, None, None, 2, 64)
    with pytest.raises(ValueError, match="densely"):
        xnor.xnor_w8_linear(q.t(), new(64), new(4, 2, dtype=i8), new(4), None, new(64, 4), None, 64, 2, 4)
