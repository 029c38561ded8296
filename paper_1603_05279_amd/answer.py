"""A binary layer and the real end of a network behind it: trained, rounded to few bits, and asked.

    python -m paper_1603_05279_amd.answer [--rows 1024] [--inputs 1024] [--width 512] [--classes 1000] [--steps 90]

The inputs are seeded noisy copies of one pattern per class.  A fixed binary fully connected layer makes features of their signs; behind it
stand a root-mean-square norm and a real classifier, as XNOR-Net leaves a network's last layer real (sec. 4.1).  `EndTraining` trains
those two through the norm's 8-bit rounding, `Answer` holds the classifier in 4 bits and answers in three library calls.
"""
import argparse

import torch

from . import xnor

EPS = 1e-6


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

    def __call__(self, x, tokens, residual=None, stream=None):
        """logprob of `tokens` [rows][given], entropy, top_index and top_logprob are filled."""
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


def binary_features(x, weights):
    """float32 outputs of a binary fully connected layer: one binarise call, one product."""
    rows, inputs = x.shape
    desc = xnor.make_desc(rows, inputs, 1, 1, weights.shape[0], 1, 1)
    bufs = xnor.ConvBuffers(desc, x.device)
    xnor.xnor_binactiv(x, None, None, bufs.xbits, bufs.A, None, desc)
    out = torch.empty((rows, weights.shape[0]), dtype=torch.float32, device=x.device)
    xnor.xnor_linear(bufs.xbits, weights.wbits, weights.wmfma, bufs.A, weights.alpha, out, None, rows, inputs, weights.shape[0])
    return out


def run(rows=1024, inputs=1024, width=512, classes=1000, steps=90, group=64, rate=5.0, report=print):
    """Trains on `rows` examples, answers `rows` others; what came of it as a dict."""
    gen = torch.Generator(device="cpu").manual_seed(2024)
    patterns = torch.randn((classes, inputs), generator=gen)
    layer = xnor.PackedWeights(torch.randn((width, inputs, 1, 1), generator=gen).cuda())
    labels = torch.randint(0, classes, (2, rows), generator=gen)
    x = patterns[labels] + torch.randn((2, rows, inputs), generator=gen)
    labels = [part.cuda().unsqueeze(1) for part in labels]              # (apart: each starts at 16 bytes, whatever the rows)
    train, held = (binary_features(part.cuda(), layer) for part in x)

    end = EndTraining(torch.ones(width, device="cuda"), torch.zeros((classes, width), device="cuda"), rows, group)
    losses = []
    for i in range(steps):
        end.step(train, labels[0], rate)
        if i % 30 == 0 or i == steps - 1:
            losses.append(-float(end.logprob.mean()))
            report(f"step {i:4d}  loss {losses[-1]:.4f}")

    answer = Answer(end.norm_weight, xnor.W4Weights.quantized(end.weight, group, zeros=True), rows)
    seen = torch.isin(labels[1].flatten(), labels[0].flatten())         # (a class without an example cannot be known)
    answer(held, labels[1])
    right = (answer.top_index[:, 0].long() == labels[1].flatten())[seen].float().mean()
    h = held.double()
    exact = (h * (h.square().mean(1, keepdim=True) + EPS).rsqrt() * end.norm_weight) @ end.weight.double().t()
    same = (exact.argmax(1) == answer.top_index[:, 0]).float().mean()
    result = {"losses": losses, "right": float(right), "same": float(same), "logprob": float(answer.logprob[seen].mean())}
    report(f"held-out rows of known classes: {100 * result['right']:.1f} % right, mean log probability {result['logprob']:.3f}; "
           f"4-bit and real classifiers agree on {100 * result['same']:.1f} % of all rows")
    return result


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("rows", 1024), ("inputs", 1024), ("width", 512), ("classes", 1000), ("steps", 90)):
        parser.add_argument("--" + name, type=int, default=value)
    run(**vars(parser.parse_args()))


if __name__ == "__main__":
    main()
