"""Refusals of include/xnor_lowbit.h: status codes before anything is launched, and the binding's checks of tensors (no GPU)."""
import ctypes

import pytest
import torch

from paper_1603_05279_amd import xnor

NULL, SHAPE, UNSUPPORTED, ALIGN = -1, -2, -3, -4
FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)     # never dereferenced


def norm(x=FAKE, xs=64, r=None, rs=0, w=None, s=None, q=FAKE, scale=FAKE, v=None, rstd=None, rows=2, cols=64, group=0, type=1, eps=1e-6):
    return xnor.lib().xnor_rmsnorm_q8(x, xs, r, rs, w, s, q, scale, v, rstd, rows, cols, group, type, eps, None)


def norm_backward(h=FAKE, hs=64, rstd=FAKE, w=None, g=FAKE, gs=64, s=None, ss=0, gh=FAKE, gw=None, ws=None, rows=2, cols=64, type=1):
    return xnor.lib().xnor_rmsnorm_backward(h, hs, rstd, w, g, gs, s, ss, gh, gw, ws, rows, cols, type, None)


def quantize(w=FAKE, ws=64, c=FAKE, s=FAKE, z=None, out=4, cin=64, group=32, type=0):
    return xnor.lib().xnor_w4_quantize(w, ws, c, s, z, out, cin, group, type, None)


def pack(c=FAKE, s=FAKE, z=None, img=FAKE, out=4, cin=64, group=32):
    return xnor.lib().xnor_w4_pack(c, s, z, img, out, cin, group, None)


def linear(x=FAKE, xs=64, img=FAKE, y=FAKE, ws=FAKE, rows=2, cin=64, out=4, group=32, type=0):
    return xnor.lib().xnor_w4_linear(x, xs, img, y, ws, rows, cin, out, group, type, None)


def linear_q8(q=FAKE, xs=FAKE, img=FAKE, y=FAKE, ws=FAKE, rows=2, cin=64, out=4, group=32, x_group=0, type=0):
    return xnor.lib().xnor_w4_linear_q8(q, xs, img, y, ws, rows, cin, out, group, x_group, type, None)


def logprobs(l=FAKE, ls=64, t=FAKE, tb=8, lp=FAKE, lse=None, shift=None, h=None, ti=None, tv=None, ws=FAKE, rows=2, vocab=64, given=1, top=0, type=0):
    return xnor.lib().xnor_logprobs(l, ls, t, tb, lp, lse, shift, h, ti, tv, ws, rows, vocab, given, top, type, None)


def logprobs_backward(l=FAKE, ls=64, t=FAKE, tb=8, shift=FAKE, h=None, gl=FAKE, gh=None, g=FAKE, rows=2, vocab=64, given=1, type=0):
    return xnor.lib().xnor_logprobs_backward(l, ls, t, tb, shift, h, gl, gh, g, rows, vocab, given, type, None)


@pytest.mark.parametrize("call,status,bad", [
    (norm, NULL, dict(x=None)), (norm, NULL, dict(q=None)), (norm, NULL, dict(scale=None)), (norm, SHAPE, dict(rows=-1)),
    (norm, SHAPE, dict(rows=65535 * 64 + 1)), (norm, SHAPE, dict(cols=0)), (norm, SHAPE, dict(xs=63)), (norm, SHAPE, dict(r=FAKE, rs=63)),
    (norm, SHAPE, dict(eps=0.0)), (norm, SHAPE, dict(eps=float("nan"))), (norm, SHAPE, dict(eps=float("inf"))), (norm, UNSUPPORTED, dict(group=16)),
    (norm, UNSUPPORTED, dict(group=-32)), (norm, UNSUPPORTED, dict(type=3)), (norm, UNSUPPORTED, dict(type=-1)),
    (norm, UNSUPPORTED, dict(cols=32769, xs=40000)), (norm, ALIGN, dict(x=ODD)), (norm, ALIGN, dict(q=ODD)), (norm, ALIGN, dict(w=ODD)),
    (norm, ALIGN, dict(rstd=ODD)), (norm, 0, dict(rows=0, x=None, q=None)),
    (norm_backward, NULL, dict(h=None)), (norm_backward, NULL, dict(rstd=None)), (norm_backward, NULL, dict(g=None)), (norm_backward, NULL, dict(gh=None)),
    (norm_backward, NULL, dict(gw=FAKE)), (norm_backward, SHAPE, dict(hs=63)), (norm_backward, SHAPE, dict(gs=63)), (norm_backward, SHAPE, dict(s=FAKE)),
    (norm_backward, SHAPE, dict(cols=-4)), (norm_backward, UNSUPPORTED, dict(type=9)), (norm_backward, ALIGN, dict(gw=ODD, ws=FAKE)),
    (norm_backward, ALIGN, dict(ws=ODD, gw=FAKE)), (norm_backward, 0, dict(rows=0, h=None)),
    (quantize, NULL, dict(w=None)), (quantize, NULL, dict(c=None)), (quantize, NULL, dict(s=None)), (quantize, SHAPE, dict(out=0)),
    (quantize, SHAPE, dict(ws=63)), (quantize, UNSUPPORTED, dict(group=0)), (quantize, UNSUPPORTED, dict(group=256)), (quantize, UNSUPPORTED, dict(type=5)),
    (quantize, ALIGN, dict(z=ODD)), (pack, NULL, dict(c=None)), (pack, NULL, dict(s=None)), (pack, NULL, dict(img=None)), (pack, SHAPE, dict(cin=0)),
    (pack, SHAPE, dict(cin=(1 << 24) + 1)), (pack, UNSUPPORTED, dict(group=48)), (pack, ALIGN, dict(img=ODD)),
    (linear, NULL, dict(x=None)), (linear, NULL, dict(img=None)), (linear, NULL, dict(y=None)), (linear, SHAPE, dict(rows=-2)), (linear, SHAPE, dict(xs=10)),
    (linear, SHAPE, dict(out=-1)), (linear, UNSUPPORTED, dict(type=3)), (linear, UNSUPPORTED, dict(group=0)), (linear, ALIGN, dict(y=ODD)),
    (linear, ALIGN, dict(ws=ODD)), (linear, 0, dict(rows=0, x=None)),
    (linear_q8, NULL, dict(q=None)), (linear_q8, NULL, dict(xs=None)), (linear_q8, UNSUPPORTED, dict(x_group=16)), (linear_q8, UNSUPPORTED, dict(group=64, x_group=32)),
    (linear_q8, UNSUPPORTED, dict(type=-2)), (linear_q8, ALIGN, dict(xs=ODD)), (linear_q8, SHAPE, dict(cin=0)), (linear_q8, 0, dict(rows=0, y=None)),
    (logprobs, NULL, dict(l=None)), (logprobs, NULL, dict(t=None)), (logprobs, NULL, dict(lp=None)), (logprobs, NULL, dict(top=1)),
    (logprobs, SHAPE, dict(vocab=0)), (logprobs, SHAPE, dict(ls=63)), (logprobs, SHAPE, dict(given=-1)), (logprobs, SHAPE, dict(top=-1)),
    (logprobs, UNSUPPORTED, dict(top=33, ti=FAKE, tv=FAKE)), (logprobs, UNSUPPORTED, dict(given=1025)), (logprobs, UNSUPPORTED, dict(tb=2)),
    (logprobs, UNSUPPORTED, dict(type=4)), (logprobs, NULL, dict(vocab=100000, ls=100000, ws=None)), (logprobs, ALIGN, dict(lse=ODD)), (logprobs, ALIGN, dict(shift=ODD)), (logprobs, 0, dict(rows=0, l=None)),
    (logprobs_backward, NULL, dict(l=None)), (logprobs_backward, NULL, dict(shift=None)), (logprobs_backward, NULL, dict(g=None)),
    (logprobs_backward, NULL, dict(gl=None)), (logprobs_backward, NULL, dict(gh=FAKE)), (logprobs_backward, NULL, dict(t=None)),
    (logprobs_backward, SHAPE, dict(ls=1)), (logprobs_backward, UNSUPPORTED, dict(tb=16)), (logprobs_backward, ALIGN, dict(g=ODD)),
    (logprobs_backward, SHAPE, dict(rows=65535 * 64, vocab=1 << 20, ls=1 << 20)), (logprobs_backward, 0, dict(rows=0, g=None)),
])
def test_status(call, status, bad):
    assert call(**bad) == status


def test_sizes_that_are_refused_need_nothing():
    assert xnor.w4_wimg_bytes(0, 64, 32) == xnor.w4_wimg_bytes(4, 64, 33) == 0
    assert xnor.w4_wimg_bytes(17, 129, 64) == 2 * 2 * 1024 + 2 * 3 * (64 + 16)
    assert xnor.rmsnorm_backward_workspace_bytes(0, 64) == xnor.logprobs_workspace_bytes(0, 64, 1) == xnor.w4_linear_workspace_bytes(-1, 64, 64, 32) == 0
    assert xnor.logprobs_workspace_bytes(4, 100, 8) == 0


class _Stream:
    cuda_stream = 0


def test_tensors_on_the_host_or_of_another_type():
    x = torch.zeros((2, 64))
    with pytest.raises(ValueError, match="device"):
        xnor.xnor_rmsnorm_q8(x, None, None, None, None, None, x, None, 2, 64, 0, 1e-6, stream=_Stream())
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        xnor.xnor_rmsnorm_q8(x.double(), None, None, None, None, None, x, None, 2, 64, 0, 1e-6, stream=_Stream())
    with pytest.raises(TypeError):
        xnor.xnor_w4_linear(None, x, x, None, 2, 64, 4, 32, stream=_Stream())


@pytest.mark.gpu
def test_tensors_that_hold_less_than_the_sizes_say():
    x, f = torch.zeros((2, 64), device="cuda"), torch.zeros(2, device="cuda")
    for rows, cols, group, scale in ((3, 64, 0, 3), (2, 65, 0, 2), (2, 64, 32, 2)):
        with pytest.raises(ValueError, match="holds less"):
            xnor.xnor_rmsnorm_q8(x, None, None, None, None, torch.zeros(scale, device="cuda"), x, None, rows, cols, group, 1e-6)
    with pytest.raises(ValueError, match="int32 or int64"):
        xnor.xnor_logprobs(x, x, f, f, None, f, None, None, None, 2, 64, 1, 0)
    with pytest.raises(ValueError, match="densely"):
        xnor.xnor_rmsnorm_q8(x.t(), None, None, None, None, None, x, None, 64, 2, 0, 1e-6)
    with pytest.raises(ValueError, match="holds less"):
        xnor.xnor_w4_linear(x, torch.zeros(100, dtype=torch.uint8, device="cuda"), x, None, 2, 64, 4, 32)
    with pytest.raises(ValueError, match="holds less"):
        xnor.xnor_logprobs(x, torch.zeros(1, dtype=torch.int64, device="cuda"), f, f, None, f, None, None, None, 2, 64, 1, 0)
    with pytest.raises(ValueError, match="holds less"):
        xnor.xnor_logprobs_backward(x, torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros((2, 2), device="cuda"), f, f, f[:1], x, 2, 64, 1)
