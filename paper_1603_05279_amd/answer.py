"""A binary layer and the real end of a network behind it: trained, rounded to few bits, and asked.

    python -m paper_1603_05279_amd.answer [--rows 1024] [--inputs 1024] [--width 512] [--classes 1000] [--steps 90] [--hidden 0]

The inputs are seeded noisy copies of one pattern per class.  A fixed binary fully connected layer makes features of their signs; behind it
stand a root-mean-square norm and a real classifier, as XNOR-Net leaves a network's last layer real (sec. 4.1).  `EndTraining` trains
those two through the norm's 8-bit rounding, `Answer` holds the classifier in 4 bits and answers in three library calls.

With `--hidden N` a hidden layer of N outputs and its activation stand between norm and classifier (`--gated` for the product of two halves).
`HiddenTraining` trains all of it in 8 bits: rows and weights of both products, what the activation keeps for the backward pass, and the rows
that the weight gradients read.  `HiddenAnswer` holds both layers in 8 bits.  Either answer draws one class per row, too.
"""
import argparse

import torch

from . import xnor

EPS = 1e-6


class Drawn:
    """One token per row of logits, drawn with given random numbers, on buffers of its own: token, its log probability, how many were left."""

    def __init__(self, rows, classes, device):
        self.rows, self.classes = rows, classes
        self.token, self.kept = (torch.empty(rows, dtype=torch.int32, device=device) for _ in range(2))
        self.logprob = torch.empty(rows, dtype=torch.float32, device=device)
        self.workspace = torch.empty(max(xnor.sample_workspace_bytes(rows, classes), 1), dtype=torch.uint8, device=device)

    def __call__(self, logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
        xnor.xnor_sample(logits, temperature, top_k, top_p, min_p, uniform, self.token, self.logprob, self.kept, self.workspace,
                         self.rows, self.classes, stream)


class Answer:
    """Norm -> 4-bit classifier -> log probabilities, for `rows` rows of `type`, on buffers of its own."""

    def __init__(self, norm_weight, head, rows, dtype=torch.float32, given=1, top=5):
        self.norm_weight, self.head = norm_weight, head
        self.rows, self.given, self.top = rows, given, top
        classes, width = head.shape
        device = norm_weight.device

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        self.q = empty(rows, width, dtype=torch.int8)
        self.scale = empty(rows, -(-width // head.group))
        self.logits = empty(rows, classes, dtype=dtype)
        self.logprob, self.entropy = empty(rows, given), empty(rows)
        self.top_index, self.top_logprob = empty(rows, top, dtype=torch.int32), empty(rows, top)
        nbytes = max(xnor.w4_linear_workspace_bytes(rows, width, classes, head.group), xnor.logprobs_workspace_bytes(rows, classes, top))
        self.workspace = empty(max(nbytes, 1), dtype=torch.uint8)
        self.drawn = Drawn(rows, classes, device)

    def __call__(self, x, tokens, residual=None, stream=None):
        """logprob of `tokens` [rows][given], entropy, top_index and top_logprob are filled; `drawn(logits, uniform, ...)` draws from these rows."""
        classes, width = self.head.shape
        group = self.head.group
        xnor.xnor_rmsnorm_q8(x, residual, self.norm_weight, None, self.q, self.scale, None, None, self.rows, width, group, EPS, stream)
        xnor.xnor_w4_linear_q8(self.q, self.scale, self.head.wimg, self.logits, self.workspace, self.rows, width, classes, group, group, stream)
        xnor.xnor_logprobs(self.logits, tokens, self.logprob, None, None, self.entropy, self.top_index, self.top_logprob, self.workspace,
                           self.rows, classes, self.given, self.top, stream)


class EndTraining:
    """Norm and classifier in float32, trained by plain gradient descent on the mean log probability of one label per row."""

    def __init__(self, norm_weight, weight, rows, group):
        self.norm_weight, self.weight, self.rows, self.group = norm_weight, weight, rows, group
        classes, width = weight.shape
        device = weight.device

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        self.values, self.rstd = empty(rows, width), empty(rows)
        self.logprob, self.shift = empty(rows, 1), empty(rows, 2)
        self.g_logprob = torch.full((rows, 1), -1.0 / rows, device=device)
        self.g_x, self.g_norm_weight, self.g_logits = empty(rows, width), empty(width), empty(rows, classes)
        self.g_weight = empty(classes, width)
        nbytes = max(xnor.rmsnorm_backward_workspace_bytes(rows, width), xnor.logprobs_workspace_bytes(rows, classes, 0))
        self.workspace = empty(max(nbytes, 1), dtype=torch.uint8)

    def gradients(self, x, labels, stream=None):
        """Loss = -mean logprob; fills g_x, g_norm_weight and g_weight, all on `stream`."""
        with xnor.on_stream(stream):
            self._gradients(x, labels)

    def _gradients(self, x, labels):
        classes, width = self.weight.shape
        rows = self.rows
        xnor.xnor_rmsnorm_q8(x, None, self.norm_weight, None, None, None, self.values, self.rstd, rows, width, self.group, EPS)
        logits = self.values @ self.weight.t()
        xnor.xnor_logprobs(logits, labels, self.logprob, None, self.shift, None, None, None, self.workspace, rows, classes, 1, 0)
        xnor.xnor_logprobs_backward(logits, labels, self.shift, None, self.g_logprob, None, self.g_logits, rows, classes, 1)
        torch.mm(self.g_logits.t(), self.values, out=self.g_weight)
        xnor.xnor_rmsnorm_backward(x, self.rstd, self.norm_weight, self.g_logits @ self.weight, None, self.g_x, self.g_norm_weight,
                                   self.workspace, rows, width)

    def step(self, x, labels, rate):
        self.gradients(x, labels)
        self.weight -= rate * self.g_weight
        self.norm_weight -= rate * self.g_norm_weight


class HiddenAnswer:
    """Norm -> 8-bit hidden layer -> activation -> 8-bit classifier -> log probabilities, for `rows` rows of `type`, on buffers of its own.

    `hidden` and `head` are `W8Weights`; with `gated` the hidden layer has two outputs for each input of the classifier."""

    def __init__(self, norm_weight, hidden, head, rows, function="gelu", gated=False, dtype=torch.float32, given=1, top=5):
        self.norm_weight, self.hidden, self.head, self.rows = norm_weight, hidden, head, rows
        self.function, self.gated, self.given, self.top = function, gated, given, top
        (wide, width), (classes, inner) = hidden.shape, head.shape
        device = norm_weight.device

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        self.q, self.scale = empty(rows, width, dtype=torch.int8), empty(rows, 1)
        self.inner_q, self.inner_scale = empty(rows, inner, dtype=torch.int8), empty(rows, 1)
        self.before, self.logits = empty(rows, wide, dtype=dtype), empty(rows, classes, dtype=dtype)
        self.logprob, self.entropy = empty(rows, given), empty(rows)
        self.top_index, self.top_logprob = empty(rows, top, dtype=torch.int32), empty(rows, top)
        nbytes = max(xnor.w8_linear_workspace_bytes(rows, width, wide), xnor.w8_linear_workspace_bytes(rows, inner, classes),
                     xnor.logprobs_workspace_bytes(rows, classes, top))
        self.workspace = empty(max(nbytes, 1), dtype=torch.uint8)
        self.drawn = Drawn(rows, classes, device)

    def __call__(self, x, tokens, residual=None, stream=None):
        """logprob of `tokens` [rows][given], entropy, top_index and top_logprob are filled; `drawn(logits, uniform, ...)` draws from these rows."""
        (wide, width), (classes, inner) = self.hidden.shape, self.head.shape
        rows, w = self.rows, self.workspace
        xnor.xnor_rmsnorm_q8(x, residual, self.norm_weight, None, self.q, self.scale, None, None, rows, width, 0, EPS, stream)
        xnor.xnor_w8_linear(self.q, self.scale, self.hidden.codes, self.hidden.scale, None, self.before, w, rows, width, wide, stream)
        xnor.xnor_activation_q8(self.before, None, self.inner_q, self.inner_scale, None, None, rows, inner, 0, 0, self.function, self.gated, stream)
        xnor.xnor_w8_linear(self.inner_q, self.inner_scale, self.head.codes, self.head.scale, None, self.logits, w, rows, inner, classes, stream)
        xnor.xnor_logprobs(self.logits, tokens, self.logprob, None, None, self.entropy, self.top_index, self.top_logprob, w,
                           rows, classes, self.given, self.top, stream)


class HiddenTraining:
    """Norm, hidden layer, activation and classifier, trained by plain gradient descent on the mean log probability of one label per row.

    The weights are float32; both products read them, and their rows, in 8 bits, and the backward pass takes these roundings for the identity:
    the gradients of the rows come from the float32 weights that are trained (a code's half step, 1 / 254 of an output's largest, from those
    that the products read), the gradients of the weights from the 8-bit rows, the only ones that are kept.
    Nothing of the forward pass is kept in more than 8 bits but the logits."""

    def __init__(self, norm_weight, hidden, head, rows, function="gelu", gated=False, kept_group=128):
        self.norm_weight, self.hidden, self.head, self.rows = norm_weight, hidden, head, rows
        self.function, self.gated, self.kept_group = function, gated, kept_group
        (wide, width), (classes, inner) = hidden.shape, head.shape
        device = hidden.device

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        self.hidden8, self.head8 = xnor.W8Weights(hidden), xnor.W8Weights(head)
        self.rstd, self.q, self.scale = empty(rows), empty(rows, width, dtype=torch.int8), empty(rows, 1)
        self.inner_q, self.inner_scale = empty(rows, inner, dtype=torch.int8), empty(rows, 1)
        self.kept, self.kept_scale = empty(rows, wide, dtype=torch.int8), empty(rows, -(-wide // kept_group) if kept_group else 1)
        self.before, self.logits = empty(rows, wide), empty(rows, classes)
        self.logprob, self.shift = empty(rows, 1), empty(rows, 2)
        self.g_logprob = torch.full((rows, 1), -1.0 / rows, device=device)
        self.g_logits, self.g_before, self.g_x, self.g_norm_weight = empty(rows, classes), empty(rows, wide), empty(rows, width), empty(width)
        self.g_hidden, self.g_head = empty(wide, width), empty(classes, inner)
        f32 = torch.float32
        nbytes = max(xnor.w8_linear_workspace_bytes(rows, width, wide), xnor.w8_linear_workspace_bytes(rows, inner, classes),
                     xnor.q8_weight_gradient_workspace_bytes(rows, width, wide, 0, f32, f32),
                     xnor.q8_weight_gradient_workspace_bytes(rows, inner, classes, 0, f32, f32),
                     xnor.rmsnorm_backward_workspace_bytes(rows, width), xnor.logprobs_workspace_bytes(rows, classes, 0))
        self.workspace = empty(max(nbytes, 1), dtype=torch.uint8)

    def gradients(self, x, labels, stream=None):
        """Loss = -mean logprob; fills g_x, g_norm_weight, g_hidden and g_head, all on `stream`."""
        with xnor.on_stream(stream):
            self._gradients(x, labels)

    def _gradients(self, x, labels):
        (wide, width), (classes, inner) = self.hidden.shape, self.head.shape
        rows, w = self.rows, self.workspace
        self.hidden8.quantize(self.hidden)
        self.head8.quantize(self.head)
        xnor.xnor_rmsnorm_q8(x, None, self.norm_weight, None, self.q, self.scale, None, self.rstd, rows, width, 0, EPS)
        xnor.xnor_w8_linear(self.q, self.scale, self.hidden8.codes, self.hidden8.scale, None, self.before, w, rows, width, wide)
        xnor.xnor_activation_q8(self.before, None, self.inner_q, self.inner_scale, self.kept, self.kept_scale, rows, inner, 0, self.kept_group,
                                self.function, self.gated)
        xnor.xnor_w8_linear(self.inner_q, self.inner_scale, self.head8.codes, self.head8.scale, None, self.logits, w, rows, inner, classes)
        xnor.xnor_logprobs(self.logits, labels, self.logprob, None, self.shift, None, None, None, w, rows, classes, 1, 0)
        xnor.xnor_logprobs_backward(self.logits, labels, self.shift, None, self.g_logprob, None, self.g_logits, rows, classes, 1)
        xnor.xnor_q8_weight_gradient(self.inner_q, self.inner_scale, self.g_logits, self.g_head, None, w, rows, inner, classes, 0)
        xnor.xnor_activation_backward(self.kept, self.kept_scale, self.g_logits @ self.head, self.g_before, rows, inner, self.kept_group,
                                      self.function, self.gated)
        xnor.xnor_q8_weight_gradient(self.q, self.scale, self.g_before, self.g_hidden, None, w, rows, width, wide, 0)
        xnor.xnor_rmsnorm_backward(x, self.rstd, self.norm_weight, self.g_before @ self.hidden, None, self.g_x, self.g_norm_weight, w, rows, width)

    def step(self, x, labels, rate):
        self.gradients(x, labels)
        self.hidden -= rate * self.g_hidden
        self.head -= rate * self.g_head
        self.norm_weight -= rate * self.g_norm_weight


def binary_features(x, weights):
    """float32 outputs of a binary fully connected layer: one binarise call, one product."""
    rows, inputs = x.shape
    desc = xnor.make_desc(rows, inputs, 1, 1, weights.shape[0], 1, 1)
    bufs = xnor.ConvBuffers(desc, x.device)
    xnor.xnor_binactiv(x, None, None, bufs.xbits, bufs.A, None, desc)
    out = torch.empty((rows, weights.shape[0]), dtype=torch.float32, device=x.device)
    xnor.xnor_linear(bufs.xbits, weights.wbits, weights.wmfma, bufs.A, weights.alpha, out, None, rows, inputs, weights.shape[0])
    return out


def run(rows=1024, inputs=1024, width=512, classes=1000, steps=90, group=64, rate=None, hidden=0, gated=False, report=print):
    """Trains on `rows` examples, answers `rows` others; what came of it as a dict.  `hidden` 0: no hidden layer."""
    gen = torch.Generator(device="cpu").manual_seed(2024)
    patterns = torch.randn((classes, inputs), generator=gen)
    layer = xnor.PackedWeights(torch.randn((width, inputs, 1, 1), generator=gen).cuda())
    labels = torch.randint(0, classes, (2, rows), generator=gen)
    x = patterns[labels] + torch.randn((2, rows, inputs), generator=gen)
    labels = [part.cuda().unsqueeze(1) for part in labels]              # (apart: each starts at 16 bytes, whatever the rows)
    train, held = (binary_features(part.cuda(), layer) for part in x)

    norm_weight, head = torch.ones(width, device="cuda"), torch.zeros((classes, hidden or width), device="cuda")
    if hidden:
        first = torch.randn((hidden * (2 if gated else 1), width), generator=gen).mul_(width ** -0.5).cuda()
        end = HiddenTraining(norm_weight, first, head, rows, gated=gated)
    else:
        end = EndTraining(norm_weight, head, rows, group)
    if rate is None:
        rate = 2.0 if hidden else 5.0
    losses = []
    for i in range(steps):
        end.step(train, labels[0], rate)
        if i % 30 == 0 or i == steps - 1:
            losses.append(-float(end.logprob.mean()))
            report(f"step {i:4d}  loss {losses[-1]:.4f}")

    h = held.double()
    exact = h * (h.square().mean(1, keepdim=True) + EPS).rsqrt() * end.norm_weight
    if hidden:
        answer = HiddenAnswer(end.norm_weight, xnor.W8Weights(end.hidden), xnor.W8Weights(end.head), rows, gated=gated)
        before = exact @ end.hidden.double().t()
        value = before[:, :hidden]
        value = 0.5 * value * torch.special.erfc(value * -0.5 ** 0.5)
        exact = (value * before[:, hidden:] if gated else value) @ end.head.double().t()
    else:
        answer = Answer(end.norm_weight, xnor.W4Weights.quantized(end.weight, group, zeros=True), rows)
        exact = exact @ end.weight.double().t()
    seen = torch.isin(labels[1].flatten(), labels[0].flatten())         # (a class without an example cannot be known)
    answer(held, labels[1])
    right = (answer.top_index[:, 0].long() == labels[1].flatten())[seen].float().mean()
    same = (exact.argmax(1) == answer.top_index[:, 0]).float().mean()
    answer.drawn(answer.logits, torch.rand(rows, generator=gen).cuda())
    drawn = (answer.drawn.token.long() == labels[1].flatten())[seen].float().mean()
    result = {"losses": losses, "right": float(right), "same": float(same), "logprob": float(answer.logprob[seen].mean()), "drawn": float(drawn)}
    report(f"held-out rows of known classes: {100 * result['right']:.1f} % right, {100 * result['drawn']:.1f} % when drawn, "
           f"mean log probability {result['logprob']:.3f}; {8 if hidden else 4}-bit and real ends agree on {100 * result['same']:.1f} % of all rows")
    return result


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("rows", 1024), ("inputs", 1024), ("width", 512), ("classes", 1000), ("steps", 90), ("hidden", 0)):
        parser.add_argument("--" + name, type=int, default=value)
    parser.add_argument("--gated", action="store_true")
    run(**vars(parser.parse_args()))


if __name__ == "__main__":
    main()
