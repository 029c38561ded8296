"""The low-bit layers around a network's binary blocks, as their users issue them (entry points of paper_1603_05279_amd.xnor).

XNOR-Net leaves a network's first and last layers real.  What a program runs there: the residual's addition and the root-mean-square norm with
8-bit outputs, the product with 4-bit weights under group scales, and the log probabilities of the answer with its alternatives; in training
the backward passes of the norm (straight through the rounding) and of the log probabilities.  Buffers belong to the caller and are kept, the
4-bit weights are laid out once.

Kinds of work (`kind`):
  norm        h = x + residual, RMS norm, 8-bit values and scales
  norm_train  the same with the values a layer is trained on, and its backward pass
  w4          product of real rows with 4-bit weights
  layer       norm, then the product of its 8-bit output with 4-bit weights
  head        layer with the vocabulary's rows as weights, then the log probabilities of its logits
  logp        log probabilities of given tokens, entropy, top alternatives
  logp_train  the same and its backward pass

Plain forms compute in 32 bits and round once at the end; every rounding that is part of the operator (8-bit values) is a comparison-free
sequence of single roundings, so the stored integers are the same on both sides.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = 2.0 ** -100          # a group whose largest magnitude is below has 8-bit values of zero


def listed():
    return [
        # one token in front of a layer of width 4096: latency of a single request
        {"name": "norm_4096_1", "kind": "norm", "rows": 1, "cols": 4096, "type": "bf16", "group": 0},
        # a prompt of 2048 tokens, scales in groups as the 4-bit products take them
        {"name": "norm_4096_2048", "kind": "norm", "rows": 2048, "cols": 4096, "type": "bf16", "group": 128},
        # a training step's batch over a wide layer (the width of AlexNet's first fully connected layer)
        {"name": "norm_train_9216_2048", "kind": "norm_train", "rows": 2048, "cols": 9216, "type": "bf16", "group": 0},
        # nothing a multiple of anything, in 32 bits
        {"name": "norm_train_1003_777", "kind": "norm_train", "rows": 777, "cols": 1003, "type": "f32", "group": 64},
        # AlexNet's first fully connected layer on a single request
        {"name": "w4_9216x4096_1", "kind": "w4", "rows": 1, "cin": 9216, "cout": 4096, "type": "bf16", "group": 128, "zeros": False},
        # a decoding batch of 16, zero points, small groups
        {"name": "w4_4096x4096_16", "kind": "w4", "rows": 16, "cin": 4096, "cout": 4096, "type": "f16", "group": 64, "zeros": True},
        # a ragged classifier in 32 bits
        {"name": "w4_1003x1000_37", "kind": "w4", "rows": 37, "cin": 1003, "cout": 1000, "type": "f32", "group": 32, "zeros": True},
        # a prompt through a wide product
        {"name": "w4_4096x8192_2048", "kind": "w4", "rows": 2048, "cin": 4096, "cout": 8192, "type": "bf16", "group": 128, "zeros": False},
        # the first fully connected layer at its benchmark batch, 8-bit inputs from the norm in front of it
        {"name": "layer_9216x4096_256", "kind": "layer", "rows": 256, "cin": 9216, "cout": 4096, "type": "bf16", "group": 128, "zeros": False},
        # the last layers of a decoding batch of 8: norm, vocabulary product, log probabilities of the answer
        {"name": "head_4096x32000_8", "kind": "head", "rows": 8, "cin": 4096, "cout": 32000, "type": "bf16", "group": 128, "zeros": False,
         "given": 1, "top": 8},
        # the answer to one request out of a long vocabulary, twenty alternatives
        {"name": "logp_128000_1", "kind": "logp", "rows": 1, "vocab": 128000, "type": "bf16", "given": 1, "top": 20, "masked": 0.0},
        # a training batch over a vocabulary: loss, entropy and their gradient
        {"name": "logp_train_32000_4096", "kind": "logp_train", "rows": 4096, "vocab": 32000, "type": "bf16", "given": 1, "top": 0, "masked": 0.0},
    ]


# ---- sizes ----------------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi, step):
    """Half of the widths are whole steps, the others any."""
    n = _log_int(rng, lo, hi)
    n = max(step, n // step * step) if rng.random() < 0.5 else n
    return n + 1 if n == 3 * 1024 else n


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "w4", "w4", "layer", "head", "logp", "logp", "logp_train"])
    case = {"kind": kind, "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
    if kind in ("norm", "norm_train"):
        cols = _width(rng, 64, 16384, 64)
        case.update(rows=_log_int(rng, 1, min(8192, 2048 * 9216 // cols)), cols=cols, group=rng.choice([0, 32, 64, 128]))
    elif kind in ("w4", "layer", "head"):
        cin, cout = _width(rng, 256, 9216, 128), _width(rng, 1000 if kind == "head" else 256, 32000 if kind == "head" else 8192, 64)
        most = 64 if kind == "head" else 2048
        case.update(rows=_log_int(rng, 1, most), cin=cin, cout=cout, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5)
        if case["type"] == "f32" or cin * cout * case["rows"] > 4096 * 8192 * 2048:     # (no dearer than the listed prompt)
            case["rows"] = _log_int(rng, 1, max(1, min(most, 4096 * 8192 * 2048 // 4 // (cin * cout))))
        if kind == "head":
            case.update(given=rng.choice([1, 1, 4]), top=rng.choice([0, 1, 5, 20]))
    else:
        vocab, top = _width(rng, 100, 160000, 8), rng.choice([0, 1, 5, 20, 32])
        most = 4096 * 32000 // (8 if top else 4 if case["type"] == "f32" else 2)
        case.update(rows=_log_int(rng, 1, min(4096, most // vocab)), vocab=vocab, given=rng.choice([1, 1, 3]), top=top,
                    masked=rng.choice([0.0, 0.0, 0.5, 0.999]))
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


def _norm_inputs(case, gen):
    rows, cols, t = case["rows"], case.get("cols") or case["cin"], TYPES[case["type"]]
    x = _normal(gen, rows, cols)
    x *= torch.where(_uniform(gen, cols) < 0.01, 12.0, 1.0)         # a few channels carry outliers
    s = {"x": x.to(t), "residual": (2 * _normal(gen, rows, cols)).to(t), "weight": 0.5 + _uniform(gen, cols)}
    if case["kind"] == "norm_train":
        s["g_values"], s["g_sum"] = _normal(gen, rows, cols).to(t), _normal(gen, rows, cols).to(t)
    return s


def _w4_inputs(case, gen):
    """Codes 0..15, two to a byte (the even input in the low half), rows of whole 32 inputs; a scale and a zero point per group."""
    cin, cout, group = case["cin"], case["cout"], case["group"]
    padded, groups = -(-cin // 32) * 32, -(-cin // group)
    u = (4 * _normal(gen, cout, padded) + 8).round_().clamp_(0, 15).to(torch.uint8)
    s = {"codes": u[:, 0::2] | (u[:, 1::2] << 4), "scale": (0.5 + _uniform(gen, cout, groups)) / (4 * math.sqrt(cin)), "zero": None}
    if case["zeros"]:
        s["zero"] = torch.randint(5, 11, (cout, groups), generator=gen, device="cuda", dtype=torch.uint8)
    return s


def _logits(case, gen):
    logits = 3 * _normal(gen, case["rows"], case["vocab"])
    if case["masked"]:                                              # every third row may answer with a part of the vocabulary
        logits[::3].masked_fill_(_uniform(gen, *logits[::3].shape) < case["masked"], -math.inf)
    return logits.to(TYPES[case["type"]])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, rows = case["kind"], case["rows"]
    s = {}
    if kind in ("norm", "norm_train", "layer", "head"):
        s.update(_norm_inputs(case, gen))
    if kind == "w4":
        s["x"] = _normal(gen, rows, case["cin"]).to(TYPES[case["type"]])
    if kind in ("w4", "layer", "head"):
        s.update(_w4_inputs(case, gen))
    if kind in ("logp", "logp_train"):
        s["logits"] = _logits(case, gen)
    if kind in ("head", "logp", "logp_train"):
        s["tokens"] = torch.randint(0, case.get("vocab") or case["cout"], (rows, case["given"]), generator=gen, device="cuda")
    if kind == "logp_train":
        s["g_logprob"], s["g_entropy"] = _normal(gen, rows, case["given"]), 0.01 * _normal(gen, rows)
    return s


def _groups(width, group):
    return -(-width // group) if group else 1


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _hold(case, s)
    return s


def _hold(case, s):
    """What a program of the framework's keeps from call to call: laid-out weights, results and workspaces."""
    from paper_1603_05279_amd import xnor
    kind, rows, t = case["kind"], case["rows"], TYPES[case["type"]]

    def new(*shape, dtype=t):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def scratch(size):
        return new(size, dtype=torch.uint8) if size else None

    f32 = torch.float32
    if "residual" in s:
        cols = case.get("cols") or case["cin"]
        group = 0 if kind == "head" else case["group"]
        s.update(sum=new(rows, cols), q=None if kind == "norm_train" else new(rows, cols, dtype=torch.int8),
                 values=new(rows, cols) if kind.startswith("norm") else None, qscale=new(rows, _groups(cols, group), dtype=f32),
                 rstd=new(rows, dtype=f32))
        if kind == "norm_train":
            s.update(g_x=new(rows, cols), g_weight=new(cols, dtype=f32), scratch=scratch(xnor.rmsnorm_backward_workspace_bytes(rows, cols)))
    if "codes" in s:
        cin, cout = case["cin"], case["cout"]
        s["w4"] = xnor.W4Weights(s["codes"], s["scale"], s["zero"], cin, case["group"])
        s.update(y=new(rows, cout, dtype=f32 if kind == "head" else t), w4_scratch=scratch(xnor.w4_linear_workspace_bytes(rows, cin, cout, case["group"])))
    if "tokens" in s:
        vocab, top = case.get("vocab") or case["cout"], case["top"]
        s.update(logprob=new(rows, case["given"], dtype=f32), lse=new(rows, dtype=f32), entropy=new(rows, dtype=f32),
                 shift=new(rows, 2, dtype=f32) if kind == "logp_train" else None,
                 top_index=new(rows, top, dtype=torch.int32) if top else None, top_logprob=new(rows, top, dtype=f32) if top else None,
                 lp_scratch=scratch(xnor.logprobs_workspace_bytes(rows, vocab, top)))
        if kind == "logp_train":
            s["g_logits"] = torch.empty_like(s["logits"])


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_norm(s, group):
    """h in 32 bits, 1/rms, the 8-bit integers (as real numbers) and their scales per group."""
    h = s["x"].float() + s["residual"].float()
    rstd = 1 / torch.sqrt(h.square().mean(-1) + EPS)
    t = h * s["weight"]
    rows, cols = t.shape
    group = group or cols
    t = torch.nn.functional.pad(t, (0, -cols % group)).view(rows, -1, group)
    top = t.abs().amax(-1)
    some = top >= TINY
    factor = torch.where(some, torch.full_like(top, 127.0) / top, 0.0)
    q = torch.round(t * factor[..., None])
    scale = torch.where(some, top, 0.0) * rstd[:, None] / 127
    return h, rstd, q, scale


def _plain_values(q, scale, cols):
    return (q * scale[..., None]).reshape(q.shape[0], -1)[:, :cols]


def _plain_norm_backward(s, h, rstd):
    h, g = h.float() * rstd[:, None], s["g_values"].float()
    gw = g * s["weight"]
    g_x = rstd[:, None] * (gw - h * (gw * h).mean(-1, keepdim=True)) + s["g_sum"].float()
    return g_x, (g * h).sum(0)


def _plain_weights(s, cin, group):
    u = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).flatten(1)[:, :cin].float()
    zero = s["zero"].float() if s["zero"] is not None else torch.full_like(s["scale"], 8.0)
    return (u - zero.repeat_interleave(group, 1)[:, :cin]) * s["scale"].repeat_interleave(group, 1)[:, :cin]


def _plain_logp(logits, tokens, top):
    l = logits.float()
    m = l.amax(-1, keepdim=True)
    some = m > -math.inf
    d = l - torch.where(some, m, 0.0)
    e = torch.exp(d)
    z = e.sum(-1, keepdim=True)
    lse = torch.where(some, m + torch.log(z), -math.inf)
    entropy = torch.where(some, torch.log(z) - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / z, 0.0)
    back = torch.where(some, lse, 0.0)
    r = {"logprob": l.gather(1, tokens) - back, "lse": lse[:, 0], "entropy": entropy[:, 0]}
    if top:
        v, i = torch.sort(l, dim=-1, descending=True, stable=True)          # ties: the lowest index
        v, i = v[:, :top], i[:, :top]
        r["top_index"] = torch.where(v > -math.inf, i, -1).int()
        r["top_logprob"] = v - back
    return r


def _plain_logp_backward(s, lse, entropy):
    l = s["logits"].float()
    seen = l > -math.inf                    # a masked logit is no variable: its gradient is zero
    lp = torch.where(seen, l - lse[:, None], 0.0)
    p = torch.exp(lp)
    g = -p * s["g_logprob"].sum(-1, keepdim=True) - s["g_entropy"][:, None] * p * (lp + entropy[:, None])
    return torch.where(seen, g.scatter_add_(1, s["tokens"], s["g_logprob"]), 0.0)


def _plain(s):
    case = s["case"]
    kind, t = case["kind"], TYPES[case["type"]]
    if kind in ("norm", "norm_train"):
        h, rstd, q, scale = _plain_norm(s, case["group"])
        total = h.to(t)
        r = {"sum": total, "values": _plain_values(q, scale, case["cols"]).to(t), "scale": scale, "rstd": rstd}
        if kind == "norm_train":
            g_x, g_weight = _plain_norm_backward(s, total, rstd)
            r.update(g_x=g_x.to(t), g_weight=g_weight)
        return r
    if kind in ("w4", "layer", "head"):
        w = _plain_weights(s, case["cin"], case["group"])
        if kind == "w4":
            return {"y": (s["x"].float() @ w.t()).to(t)}
        h, _, q, scale = _plain_norm(s, 0 if kind == "head" else case["group"])
        y = _plain_values(q, scale, case["cin"]) @ w.t()
        if kind == "layer":
            return {"sum": h.to(t), "y": y.to(t)}
        r = _plain_logp(y, s["tokens"], case["top"])
        r.pop("top_index", None)            # (the order of computed logits that nearly tie is no property of the operator)
        return dict(r, sum=h.to(t), logits=y)
    r = _plain_logp(s["logits"], s["tokens"], case["top"])
    if kind == "logp_train":
        r["g_logits"] = _plain_logp_backward(s, r["lse"], r["entropy"]).to(t)
    return r


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _own_logp(xnor, s, logits, rows, vocab):
    case = s["case"]
    xnor.xnor_logprobs(logits, s["tokens"], s["logprob"], s["lse"], s["shift"], s["entropy"], s["top_index"], s["top_logprob"], s["lp_scratch"],
                       rows, vocab, case["given"], case["top"])
    r = {"logprob": s["logprob"], "lse": s["lse"], "entropy": s["entropy"]}
    return dict(r, top_index=s["top_index"], top_logprob=s["top_logprob"]) if case["top"] else r


def _own(s):
    from paper_1603_05279_amd import xnor
    case = s["case"]
    kind, rows = case["kind"], case["rows"]
    if kind == "w4":
        xnor.xnor_w4_linear(s["x"], s["w4"].wimg, s["y"], s["w4_scratch"], rows, case["cin"], case["cout"], case["group"])
        return {"y": s["y"]}
    if kind in ("logp", "logp_train"):
        r = _own_logp(xnor, s, s["logits"], rows, case["vocab"])
        if kind == "logp_train":
            xnor.xnor_logprobs_backward(s["logits"], s["tokens"], s["shift"], s["entropy"], s["g_logprob"], s["g_entropy"], s["g_logits"], rows,
                                        case["vocab"], case["given"])
            r["g_logits"] = s["g_logits"]
        return r
    cols, group = case.get("cols") or case["cin"], 0 if kind == "head" else case["group"]
    xnor.xnor_rmsnorm_q8(s["x"], s["residual"], s["weight"], s["sum"], s["q"], s["qscale"], s["values"], s["rstd"], rows, cols, group, EPS)
    if kind in ("norm", "norm_train"):
        r = {"sum": s["sum"], "values": s["values"], "scale": s["qscale"], "rstd": s["rstd"]}
        if kind == "norm_train":
            xnor.xnor_rmsnorm_backward(s["sum"], s["rstd"], s["weight"], s["g_values"], s["g_sum"], s["g_x"], s["g_weight"], s["scratch"], rows, cols)
            r.update(g_x=s["g_x"], g_weight=s["g_weight"])
        return r
    xnor.xnor_w4_linear_q8(s["q"], s["qscale"], s["w4"].wimg, s["y"], s["w4_scratch"], rows, cols, case["cout"], case["group"], group)
    if kind == "layer":
        return {"sum": s["sum"], "y": s["y"]}
    r = _own_logp(xnor, s, s["y"], rows, case["cout"])
    r.pop("top_index", None)
    return dict(r, sum=s["sum"], logits=s["y"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    kind, rows, size = case["kind"], case["rows"], TYPES[case["type"]].itemsize
    moved = flops = 0
    if kind in ("norm", "norm_train"):
        n, groups = rows * case["cols"], _groups(case["cols"], case["group"])
        moved += n * 4 * size + case["cols"] * 4 + rows * (4 * groups + 4)          # x, residual; sum, values
        flops += 8 * n
        if kind == "norm_train":                                                    # sum, the two gradients; g_x
            moved, flops = moved + n * 4 * size + rows * 4 + case["cols"] * 8, flops + 10 * n
    if kind in ("layer", "head"):
        moved += rows * case["cin"] * 3 * size + case["cin"] * 4                    # x, residual; sum
        flops += 8 * rows * case["cin"]
    if kind in ("w4", "layer", "head"):
        cin, cout = case["cin"], case["cout"]
        moved += cout * (cin / 2 + _groups(cin, case["group"]) * (5 if case["zeros"] else 4))
        moved += rows * cin * size if kind == "w4" else 0
        moved += rows * cout * (4 if kind == "head" else size)
        flops += 2 * rows * cin * cout
    if kind in ("logp", "logp_train"):
        n = rows * case["vocab"]
        moved, flops = moved + n * size, flops + 6 * n
        if kind == "logp_train":
            moved, flops = moved + 2 * n * size + rows * 4 * (case["given"] + 3), flops + 8 * n
    if kind in ("head", "logp", "logp_train"):
        moved += rows * (case["given"] * 12 + 8 + case["top"] * 8)
    return {"bytes": moved, "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_norm(s, group):
    h = s["x"].double().add(s["residual"])
    rms = (h.pow(2).sum(1) / h.shape[1] + EPS).sqrt()
    y = h / rms[:, None] * s["weight"].double()
    group = group or h.shape[1]
    scale, values = [], []
    for part in y.split(group, 1):
        top = part.abs().max(1, keepdim=True).values
        scale.append(top / 127)
        values.append(torch.round(part / top * 127) * top / 127)
    return h, 1 / rms, torch.cat(scale, 1), torch.cat(values, 1)


def _exact_logp(l, tokens, top):
    lp = torch.log_softmax(l, -1)
    none = torch.isneginf(l).all(1)
    lp[none] = -math.inf
    r = {"logprob": torch.take_along_dim(lp, tokens, 1), "lse": torch.logsumexp(l, 1), "entropy": torch.special.entr(lp.exp()).sum(1)}
    if top:
        v, i = torch.sort(lp, dim=1, descending=True, stable=True)
        r["top_index"], r["top_logprob"] = i[:, :top].masked_fill(v[:, :top] == -math.inf, -1).int(), v[:, :top]
    return lp, r


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_train"):
        h, rstd, scale, values = _exact_norm(s, case["group"])
        r = {"sum": h, "values": values, "scale": scale, "rstd": rstd}
        if kind == "norm_train":
            # of the stored sum, with the stored 1/rms, as the backward pass is given them
            n, g = h.to(TYPES[case["type"]]).double() * rstd[:, None], s["g_values"].double()
            dot = (g * s["weight"] * n).sum(1, keepdim=True) / case["cols"]
            r["g_x"] = (g * s["weight"] - n * dot) * rstd[:, None] + s["g_sum"]
            r["g_weight"] = torch.sum(g * n, 0)
        return r
    if kind in ("w4", "layer", "head"):
        cin, group = case["cin"], case["group"]
        k = torch.arange(cin, device="cuda")
        u = (s["codes"][:, k // 2] >> (4 * (k % 2))) & 15
        w = u.double() - (8.0 if s["zero"] is None else s["zero"][:, k // group].double())
        w *= s["scale"][:, k // group]
        if kind == "w4":
            return {"y": s["x"].double() @ w.t()}
        h, _, _, values = _exact_norm(s, 0 if kind == "head" else group)
        y = values @ w.t()
        if kind == "layer":
            return {"sum": h, "y": y}
        _, r = _exact_logp(y, s["tokens"], case["top"])
        r.pop("top_index", None)
        return dict(r, sum=h, logits=y)
    lp, r = _exact_logp(s["logits"].double(), s["tokens"], case["top"])
    if kind == "logp_train":
        p = lp.exp()
        g = -p * s["g_logprob"].double().sum(1, keepdim=True)
        g += s["g_entropy"].double()[:, None] * (torch.special.entr(p) - p * r["entropy"][:, None])
        r["g_logits"] = g.scatter_add(1, s["tokens"], s["g_logprob"].double()).masked_fill_(torch.isneginf(s["logits"]), 0)
    return r
