"""Real layers in 8 bits, their training from 8-bit rows, and the drawn answer, as their users issue them (entry points of paper_1603_05279_amd.xnor).

What a program runs around a network's binary blocks: products of 8-bit rows with 8-bit weights, one scale for each row (token) and output channel;
activation functions that keep their input in 8 bits for the backward pass and hand 8-bit rows to the next product; the gradient of a weight from the
8-bit rows that its product read; and a token drawn from the logits by temperature, top-k, top-p and min-p with random numbers that are given.
Buffers belong to the caller and are kept; 8-bit weights are made once.

Kinds of work (`kind`):
  product     8-bit rows by 8-bit weights
  layer       real rows: to 8 bits, then the product
  activation  activation function with its input kept in 8 bits, and its backward pass
  hidden      layer, activation to 8-bit rows, product
  gradient    gradients of weights and biases from 8-bit rows
  sample      tokens drawn from rows of logits

Plain forms compute in 32 bits and round once at the end (draws in 64, where a probability next to a border decides); what is stored in 8 bits is made by
single roundings, so the stored integers are the same on both sides.  In `hidden` the rows of the second product are rounded from a computed function,
whose last bit may differ: its result is compared, which holds a few of them.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = 2.0 ** -100          # a row or group whose largest magnitude is below has 8-bit values of zero


def listed():
    return [
        # AlexNet's first fully connected layer on a single request
        {"name": "product_9216x4096_1", "kind": "product", "rows": 1, "cin": 9216, "cout": 4096, "type": "bf16", "bias": False},
        # a decoding batch of 16
        {"name": "product_4096x4096_16", "kind": "product", "rows": 16, "cin": 4096, "cout": 4096, "type": "f16", "bias": True},
        # a ragged classifier in 32 bits
        {"name": "layer_1003x1000_37", "kind": "layer", "rows": 37, "cin": 1003, "cout": 1000, "type": "f32", "bias": True},
        # a prompt of 2048 tokens through a wide layer
        {"name": "layer_4096x8192_2048", "kind": "layer", "rows": 2048, "cin": 4096, "cout": 8192, "type": "bf16", "bias": False},
        # nothing a multiple of anything, in 32 bits
        {"name": "activation_1003_777", "kind": "activation", "rows": 777, "cols": 1003, "type": "f32", "group": 64, "function": "gelu", "gated": False},
        # a training step's batch through a gated activation
        {"name": "activation_gated_4096_2048", "kind": "activation", "rows": 2048, "cols": 4096, "type": "bf16", "group": 128, "function": "silu",
         "gated": True},
        # AlexNet's two wide fully connected layers at their benchmark batch
        {"name": "hidden_9216x4096_256", "kind": "hidden", "rows": 256, "cin": 9216, "width": 4096, "cout": 4096, "type": "bf16", "function": "relu",
         "gated": False, "bias": True},
        # the first of those layers in training, gradients for weights held in 32 bits
        {"name": "gradient_9216x4096_256", "kind": "gradient", "rows": 256, "cin": 9216, "cout": 4096, "type": "bf16", "wtype": "f32", "group": 0},
        # a ragged one in 32 bits throughout
        {"name": "gradient_1003x1000_777", "kind": "gradient", "rows": 777, "cin": 1003, "cout": 1000, "type": "f32", "wtype": "f32", "group": 64},
        # a training step's batch through a wide layer, all in 16 bits
        {"name": "gradient_4096x8192_2048", "kind": "gradient", "rows": 2048, "cin": 4096, "cout": 8192, "type": "bf16", "wtype": "bf16", "group": 128},
        # the answer to one request out of a long vocabulary
        {"name": "sample_128000_1", "kind": "sample", "rows": 1, "vocab": 128000, "type": "bf16", "top_k": 0, "top_p": 0.95, "min_p": 0.0, "masked": 0.0},
        # a serving batch, every request with settings of its own
        {"name": "sample_32000_256", "kind": "sample", "rows": 256, "vocab": 32000, "type": "bf16", "top_k": 64, "top_p": 0.9, "min_p": 0.05,
         "masked": 0.0},
    ]


# ---- sizes ----------------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi, step):
    """Half of the widths are whole steps, the others any."""
    n = _log_int(rng, lo, hi)
    return max(step, n // step * step) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["product", "product", "layer", "activation", "hidden", "gradient", "gradient", "sample", "sample"])
    case = {"kind": kind, "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
    most = 2048 * 4096 * 8192
    if kind in ("product", "layer"):
        cin, cout = _width(rng, 256, 9216, 64), _width(rng, 256, 8192, 64)
        case.update(rows=_log_int(rng, 1, min(2048, most // (cin * cout))), cin=cin, cout=cout, bias=rng.random() < 0.5)
    elif kind == "activation":
        cols, gated = _width(rng, 64, 9216, 64), rng.random() < 0.5
        case.update(rows=_log_int(rng, 1, min(4096, 2048 * 4096 // cols)), cols=cols, group=rng.choice([0, 32, 64, 128]),
                    function=rng.choice(["relu", "gelu", "silu"]), gated=gated)
    elif kind == "hidden":
        case["type"] = rng.choice(["bf16", "f16"])
        cin, width, cout, gated = _width(rng, 256, 4096, 64), _width(rng, 256, 4096, 64), _width(rng, 256, 4096, 64), rng.random() < 0.5
        case.update(rows=_log_int(rng, 1, 1024), cin=cin, width=width, cout=cout, function=rng.choice(["relu", "gelu", "silu"]), gated=gated,
                    bias=rng.random() < 0.5)
    elif kind == "gradient":
        cin, cout = _width(rng, 128, 9216, 64), _width(rng, 128, 8192, 64)
        case.update(wtype=rng.choice(["f32", case["type"]]), group=rng.choice([0, 32, 64, 128]), cin=cin, cout=cout)
        if case["wtype"] != "bf16":                                     # (no dearer than the listed batch)
            most //= 4
        case["rows"] = _log_int(rng, 1, min(2048, max(1, most // (cin * cout))))
    else:
        vocab = _width(rng, 100, 160000, 8)
        case.update(rows=_log_int(rng, 1, min(512, max(1, 256 * 32000 // vocab))), vocab=vocab, top_k=rng.choice([0, 0, 1, 50, 400]),
                    top_p=rng.choice([1.0, 0.95, 0.8]), min_p=rng.choice([0.0, 0.0, 0.02]), masked=rng.choice([0.0, 0.0, 0.5, 0.999]))
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


def _to_8_bits(x, group):
    """Integers (as real numbers) and scales of a 32-bit matrix, one scale for a row (group 0) or a group of its columns."""
    rows, cols = x.shape
    group = group or cols
    t = torch.nn.functional.pad(x, (0, -cols % group)).view(rows, -1, group)
    top = t.abs().amax(-1)
    some = top >= TINY
    factor = torch.where(some, torch.full_like(top, 127.0) / top, 0.0)
    q = torch.round(t * factor[..., None])
    return q.view(rows, -1)[:, :cols], torch.where(some, top, 0.0) / 127


def _weights(gen, cout, cin):
    q, scale = _to_8_bits(_normal(gen, cout, cin) / math.sqrt(cin), 0)
    return q.to(torch.int8), scale[:, 0].contiguous()


def _rows(gen, rows, cols):
    x = _normal(gen, rows, cols)
    return x * torch.where(_uniform(gen, cols) < 0.01, 12.0, 1.0)           # a few channels carry outliers


def _setting(gen, rows, values):
    """One of `values` for each request."""
    return values[torch.randint(0, len(values), (rows,), generator=gen, device="cuda")]


def _sample_inputs(case, gen):
    rows, vocab = case["rows"], case["vocab"]
    logits = 3 * _normal(gen, rows, vocab)
    if case["masked"]:                                                      # every third row may answer with a part of the vocabulary
        logits[::3].masked_fill_(_uniform(gen, *logits[::3].shape) < case["masked"], -math.inf)
    s = {"logits": logits.to(TYPES[case["type"]]), "uniform": _uniform(gen, rows), "temperature": 0.6 + 0.8 * _uniform(gen, rows)}
    for name, off in (("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)):
        v, t = case[name], torch.int32 if name == "top_k" else torch.float32
        s[name] = None
        if v != off:            # a half of the requests leave it out
            s[name] = _setting(gen, rows, torch.tensor([v, off], dtype=t, device="cuda")) if rows > 1 else torch.tensor([v], dtype=t, device="cuda")
    return s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, rows, t = case["kind"], case["rows"], TYPES[case["type"]]
    if kind == "sample":
        return _sample_inputs(case, gen)
    if kind == "activation":
        wide = case["cols"] * (2 if case["gated"] else 1)
        return {"x": _rows(gen, rows, wide).to(t), "g_y": _normal(gen, rows, case["cols"]).to(t)}
    if kind == "gradient":
        q, scale = _to_8_bits(_rows(gen, rows, case["cin"]), case["group"])
        g = _normal(gen, rows, case["cout"]) * torch.exp(_normal(gen, rows, 1)) / 64        # tokens differ in what they have to say
        return {"q": q.to(torch.int8), "scale": scale.contiguous(), "g_y": g.to(t)}
    s, cin = {}, case["cin"]
    if kind == "product":
        q, scale = _to_8_bits(_rows(gen, rows, cin), 0)
        s["q"], s["scale"] = q.to(torch.int8), scale[:, 0].contiguous()
    else:
        s["x"] = _rows(gen, rows, cin).to(t)
    first = case["width"] * (2 if case["gated"] else 1) if kind == "hidden" else case["cout"]
    s["w"], s["w_scale"] = _weights(gen, first, cin)
    s["bias"] = _normal(gen, first) if case["bias"] else None
    if kind == "hidden":
        s["w2"], s["w2_scale"] = _weights(gen, case["cout"], case["width"])
        s["bias2"] = _normal(gen, case["cout"]) if case["bias"] else None
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
    """What a program of the framework's keeps from call to call: results and workspaces."""
    from paper_1603_05279_amd import xnor
    kind, rows, t = case["kind"], case["rows"], TYPES[case["type"]]

    def new(*shape, dtype=t):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def scratch(size):
        return new(size, dtype=torch.uint8) if size else None

    f32, i8 = torch.float32, torch.int8
    if kind == "sample":
        s.update(token=new(rows, dtype=torch.int32), logprob=new(rows, dtype=f32), kept=new(rows, dtype=torch.int32),
                 scratch=scratch(xnor.sample_workspace_bytes(rows, case["vocab"])))
    elif kind == "activation":
        wide = s["x"].shape[1]
        s.update(y=new(rows, case["cols"]), kept=new(rows, wide, dtype=i8), kept_scale=new(rows, _groups(wide, case["group"]), dtype=f32), g_x=new(rows, wide))
    elif kind == "gradient":
        cin, cout, wt = case["cin"], case["cout"], TYPES[case["wtype"]]
        s.update(g_w=new(cout, cin, dtype=wt), g_bias=new(cout, dtype=f32),
                 scratch=scratch(xnor.q8_weight_gradient_workspace_bytes(rows, cin, cout, case["group"], t, wt)))
    else:
        cin, cout, wide = case["cin"], case["cout"], s["w"].shape[0]
        if kind != "product":
            s.update(q=new(rows, cin, dtype=i8), scale=new(rows, 1, dtype=f32))
        s.update(y=new(rows, wide), scratch=scratch(xnor.w8_linear_workspace_bytes(rows, cin, wide)))
        if kind == "hidden":
            width = case["width"]
            s.update(q2=new(rows, width, dtype=i8), scale2=new(rows, 1, dtype=f32), y2=new(rows, cout),
                     scratch2=scratch(xnor.w8_linear_workspace_bytes(rows, width, cout)))


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_product(q, scale, w, w_scale, bias):
    y = (q.float() @ w.float().t()) * (scale.view(-1, 1) * w_scale)
    return y if bias is None else y + bias


def _function(x, name):
    if name == "relu":
        return torch.clamp(x, min=0.0)
    if name == "gelu":
        return x * 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
    return x / (1 + torch.exp(-x))


def _derivative(x, name):
    if name == "relu":
        return (x > 0).to(x.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-x))
    return s * (1 + x * (1 - s))


def _activation(x, name, gated):
    if not gated:
        return _function(x, name)
    a, b = x.chunk(2, 1)
    return _function(a, name) * b


def _activation_gradient(x, g, name, gated):
    if not gated:
        return g * _derivative(x, name)
    a, b = x.chunk(2, 1)
    return torch.cat((g * b * _derivative(a, name), g * _function(a, name)), 1)


def _values(q, scale, group):
    return q * (scale.repeat_interleave(group, 1)[:, :q.shape[1]] if group else scale)


def _plain_sample(s):
    l = s["logits"].double()
    v, index = torch.sort(l, dim=1, descending=True, stable=True)           # ties: the lowest index
    place = torch.arange(l.shape[1], device=l.device)
    keep = v > -math.inf
    some = keep[:, :1]
    w = torch.where(keep, torch.exp((v - torch.where(some, v[:, :1], 0.0)) / s["temperature"].double()[:, None]), 0.0)
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep = keep & ((place < k) | (k <= 0))
    if s["top_p"] is not None:
        kept = torch.where(keep, w, 0.0)
        before = torch.cumsum(kept, 1) - kept
        p = s["top_p"].double()[:, None]
        keep = keep & ((before < p * kept.sum(1, keepdim=True)) | (p >= 1) | (place == 0))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double()[:, None])
    w = torch.where(keep, w, 0.0)
    total = torch.cumsum(w, 1)
    chosen = (total <= s["uniform"].double()[:, None] * total[:, -1:]).sum(1, keepdim=True)
    count = keep.sum(1, keepdim=True)
    chosen = torch.minimum(chosen, (count - 1).clamp(min=0))
    logprob = torch.log(w.gather(1, chosen) / total[:, -1:])
    token = torch.where(some, index.gather(1, chosen), -1)
    return {"token": token[:, 0].int(), "logprob": torch.where(some, logprob, -math.inf)[:, 0].float(), "kept": count[:, 0].int()}


def _plain(s):
    case = s["case"]
    kind, t = case["kind"], TYPES[case["type"]]
    if kind == "sample":
        return _plain_sample(s)
    if kind == "activation":
        x = s["x"].float()
        kept, scale = _to_8_bits(x, case["group"])
        g_x = _activation_gradient(_values(kept, scale, case["group"]), s["g_y"].float(), case["function"], case["gated"])
        return {"y": _activation(x, case["function"], case["gated"]).to(t), "kept_scale": scale, "g_x": g_x.to(t)}
    if kind == "gradient":
        g = s["g_y"].float()
        g_w = g.t() @ _values(s["q"].float(), s["scale"], case["group"])
        return {"g_w": g_w.to(TYPES[case["wtype"]]), "g_bias": g.sum(0)}
    if kind == "product":
        return {"y": _plain_product(s["q"], s["scale"], s["w"], s["w_scale"], s["bias"]).to(t)}
    q, scale = _to_8_bits(s["x"].float(), 0)
    y = _plain_product(q, scale, s["w"], s["w_scale"], s["bias"]).to(t)
    if kind == "layer":
        return {"scale": scale, "y": y}
    q, scale = _to_8_bits(_activation(y.float(), case["function"], case["gated"]), 0)
    return {"y": _plain_product(q, scale, s["w2"], s["w2_scale"], s["bias2"]).to(t)}


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _own(s):
    from paper_1603_05279_amd import xnor
    case = s["case"]
    kind, rows = case["kind"], case["rows"]
    if kind == "sample":
        xnor.xnor_sample(s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["token"], s["logprob"], s["kept"], s["scratch"],
                         rows, case["vocab"])
        return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}
    if kind == "activation":
        cols, group, function, gated = case["cols"], case["group"], case["function"], case["gated"]
        xnor.xnor_activation_q8(s["x"], s["y"], None, None, s["kept"], s["kept_scale"], rows, cols, 0, group, function, gated)
        xnor.xnor_activation_backward(s["kept"], s["kept_scale"], s["g_y"], s["g_x"], rows, cols, group, function, gated)
        return {"y": s["y"], "kept_scale": s["kept_scale"], "g_x": s["g_x"]}
    if kind == "gradient":
        xnor.xnor_q8_weight_gradient(s["q"], s["scale"], s["g_y"], s["g_w"], s["g_bias"], s["scratch"], rows, case["cin"], case["cout"], case["group"])
        return {"g_w": s["g_w"], "g_bias": s["g_bias"]}
    cin, wide = case["cin"], s["w"].shape[0]
    if kind != "product":
        xnor.xnor_q8_rows(s["x"], s["q"], s["scale"], rows, cin, 0)
    xnor.xnor_w8_linear(s["q"], s["scale"], s["w"], s["w_scale"], s["bias"], s["y"], s["scratch"], rows, cin, wide)
    if kind == "product":
        return {"y": s["y"]}
    if kind == "layer":
        return {"scale": s["scale"], "y": s["y"]}
    width = case["width"]
    xnor.xnor_activation_q8(s["y"], None, s["q2"], s["scale2"], None, None, rows, width, 0, 0, case["function"], case["gated"])
    xnor.xnor_w8_linear(s["q2"], s["scale2"], s["w2"], s["w2_scale"], s["bias2"], s["y2"], s["scratch2"], rows, width, case["cout"])
    return {"y": s["y2"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    kind, rows, size = case["kind"], case["rows"], TYPES[case["type"]].itemsize
    if kind == "sample":
        n = rows * case["vocab"]
        return {"bytes": n * size + rows * 32, "flops": 8 * n}
    if kind == "activation":
        n, wide = rows * case["cols"], 2 if case["gated"] else 1
        groups = rows * _groups(case["cols"] * wide, case["group"])
        # x; y, the 8-bit rows and scales; those and the gradient; its result
        return {"bytes": n * size * (wide + 1) + 2 * (n * wide + 4 * groups) + n * size * (1 + wide), "flops": 30 * n * wide}
    if kind == "gradient":
        cin, cout = case["cin"], case["cout"]
        moved = rows * (cin + 4 * _groups(cin, case["group"]) + cout * size) + cout * (cin * TYPES[case["wtype"]].itemsize + 4)
        return {"bytes": moved, "flops": 2 * rows * cin * cout + rows * cout}
    cin, cout = case["cin"], case["cout"]
    moved = rows * (cin + 4 if kind == "product" else cin * size) + rows * cout * size
    wide = case["width"] * (2 if case["gated"] else 1) if kind == "hidden" else cout
    moved += wide * (cin + (8 if case["bias"] else 4))
    flops = 2 * rows * cin * wide
    if kind == "hidden":
        moved += cout * (case["width"] + (8 if case["bias"] else 4))
        flops += 2 * rows * case["width"] * cout
    return {"bytes": moved, "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_8_bits(x, group):
    """What the 8 bits of a matrix stand for, and the scales."""
    parts = [part / (part.abs().max(1, keepdim=True).values / 127) for part in x.split(group or x.shape[1], 1)]
    scales = [part.abs().max(1, keepdim=True).values / 127 for part in x.split(group or x.shape[1], 1)]
    return torch.cat([part.round() * scale for part, scale in zip(parts, scales)], 1), torch.cat(scales, 1)


def _exact_activation(x, name, gated):
    """The function's values and, by differentiation, what a gradient is multiplied by."""
    x = x.detach().requires_grad_(True)
    a, b = torch.tensor_split(x, 2, 1) if gated else (x, None)
    f = {"relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[name](a)
    return x, f * b if gated else f


def _exact_product(values, s, name, bias):
    y = values @ (s[name].double() * s[name + "_scale"].double()[:, None]).t()
    return y if s[bias] is None else y + s[bias].double()


def _exact_logprob(s):
    """Log probability, under the tokens that may be drawn, of the one that is."""
    l = s["logits"].double().cpu()
    found = []
    for r in range(l.shape[0]):
        some = torch.isfinite(l[r]).nonzero()[:, 0]
        if not len(some):
            found.append(-math.inf)
            continue
        z = l[r][some] / float(s["temperature"][r])
        z = z[torch.argsort(-l[r][some], stable=True)]
        k = int(s["top_k"][r]) if s["top_k"] is not None else 0
        z = z[:k] if k > 0 else z
        p = torch.softmax(z, 0)
        top_p = float(s["top_p"][r]) if s["top_p"] is not None else 1.0
        if top_p < 1:
            p = p[:int((p.cumsum(0) < top_p).sum()) + 1]
        if s["min_p"] is not None:
            p = p[p >= float(s["min_p"][r]) * p[0]]
        p = p / p.sum()
        at = min(int(torch.searchsorted(p.cumsum(0), float(s["uniform"][r]), right=True)), len(p) - 1)
        found.append(float(p[at].log()))
    return torch.tensor(found, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return {"token": None, "logprob": _exact_logprob(s), "kept": None}
    if kind == "activation":
        with torch.enable_grad():
            _, y = _exact_activation(s["x"].double(), case["function"], case["gated"])
            values, scale = _exact_8_bits(s["x"].double(), case["group"])
            x, again = _exact_activation(values, case["function"], case["gated"])
            g_x, = torch.autograd.grad(again, x, s["g_y"].double())
        return {"y": y.detach(), "kept_scale": scale, "g_x": g_x}
    if kind == "gradient":
        g, columns = s["g_y"].double(), torch.arange(case["cin"], device="cuda")
        scale = s["scale"].double()[:, columns // case["group"]] if case["group"] else s["scale"].double()
        return {"g_w": torch.matmul(g.t(), s["q"].double().mul(scale)), "g_bias": torch.sum(g, 0)}
    if kind == "product":
        return {"y": _exact_product(s["q"].double() * s["scale"].double().view(-1, 1), s, "w", "bias")}
    values, scale = _exact_8_bits(s["x"].double(), 0)
    y = _exact_product(values, s, "w", "bias")
    if kind == "layer":
        return {"scale": scale, "y": y}
    _, h = _exact_activation(y.to(TYPES[case["type"]]).double(), case["function"], case["gated"])
    return {"y": _exact_product(_exact_8_bits(h.detach(), 0)[0], s, "w2", "bias2")}
