"""xnor_logprobs and its backward pass against log_softmax in 64 bits.

Bounds: exp and log to a few 2^-24, a sum of positive terms added by up to 512 additions per thread (each term off by at most 512 roundings,
3e-5; in the mean their square root: 1e-5 is several standard deviations), and the roundings of log p itself."""
import math

import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import HALF_ULP, SMALLEST, TYPES, apart, assert_within, filled, generator, normal

pytestmark = pytest.mark.gpu
INF = math.inf


def reference(l, tokens, top):
    l = l.double()
    lse = torch.logsumexp(l, 1)
    empty = torch.isneginf(lse)
    lp = torch.where(empty[:, None], l, torch.log_softmax(l, 1))
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    valid = (tokens >= 0) & (tokens < l.shape[1])
    logprob = torch.where(valid, lp.gather(1, tokens.clamp(0, l.shape[1] - 1).long()), torch.zeros(tokens.shape, dtype=torch.float64))
    v, i = torch.sort(l, dim=1, descending=True, stable=True)
    n = min(top, l.shape[1])
    index, value = torch.full((l.shape[0], top), -1), torch.full((l.shape[0], top), -INF, dtype=torch.float64)
    index[:, :n] = torch.where(v[:, :n] > -INF, i[:, :n], torch.tensor(-1))
    value[:, :n] = lp.gather(1, i[:, :n])
    return lse, entropy, logprob, index, value


def run(l, tokens, top, extra=0, entropy=True):
    rows, vocab = l.shape
    given = tokens.shape[1]
    out = {"lse": filled((rows,), torch.float32), "shift": filled((rows, 2), torch.float32), "entropy": filled((rows,), torch.float32) if entropy else None,
           "logprob": filled((rows, given), torch.float32), "top_index": filled((rows, top), torch.int32), "top_logprob": filled((rows, top), torch.float32)}
    size = xnor.logprobs_workspace_bytes(rows, vocab, top)
    xnor.xnor_logprobs(apart(l, extra), tokens.cuda(), out["logprob"], out["lse"], out["shift"], out["entropy"], out["top_index"] if top else None,
                       out["top_logprob"] if top else None, filled((size,), torch.uint8) if size else None, rows, vocab, given, top)
    torch.cuda.synchronize()
    return out


def check(l, tokens, top, extra=0):
    lse, entropy, logprob, index, value = reference(l, tokens, top)
    got = run(l, tokens, top, extra)
    assert torch.equal(got["top_index"].cpu().long(), index), "alternatives"
    assert_within(got["lse"], lse, 1e-5 + 2.0 ** -23 * lse.abs().nan_to_num(posinf=0), "lse")
    assert torch.equal(got["shift"][:, 0].cpu(), l.float().amax(1)) and ((got["shift"].sum(1) - got["lse"]).abs().nan_to_num() <= 2.0 ** -23 * got["lse"].abs()).all()
    for name, want in (("entropy", entropy), ("logprob", logprob), ("top_logprob", value)):
        assert_within(got[name], want, 1e-5 * (1 + want.abs().nan_to_num(posinf=0)), name)
    return got


SIZES = [(1, 1), (1, 2), (3, 7), (5, 100), (2, 1000), (1, 8192), (3, 8193), (1, 16001), (2, 32000), (1, 128000), (600, 513), (520, 9001), (9, 20011), (40, 50257)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_sizes(t, rows, vocab):
    gen = generator(rows + vocab)
    l = normal(gen, rows, vocab, scale=3).to(TYPES[t])
    for given, top in ((1, 0), (3, 1), (0, 5), (2, 20), (1, 32)):
        check(l, torch.randint(0, vocab, (rows, given), generator=gen), top)


@pytest.mark.parametrize("extra", [1, 3, 8])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_rows_that_lie_apart_and_short_tokens(t, extra):
    gen = generator(extra)
    check(normal(gen, 5, 9003).to(TYPES[t]), torch.randint(0, 9003, (5, 2), generator=gen, dtype=torch.int32), 7, extra)


@pytest.mark.parametrize("vocab", [50, 3000, 20000, 128000])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "two values", "one thread", "lowest", "zeros of both signs", "large"])
def test_orders_and_ties(kind, vocab):
    """Rows that put all alternatives into one place, or everywhere."""
    i = torch.arange(vocab)
    l = {"rising": i / vocab * 8, "falling": -i / vocab * 8, "equal": torch.full((vocab,), 2.5), "two values": (i % 3 == 0).float(),
         "one thread": (i // 8 % 256 == 17).float() * (5 + i / vocab), "lowest": torch.full((vocab,), torch.finfo(torch.float32).min),
         "zeros of both signs": torch.where(i % 2 == 0, -0.0, 0.0), "large": 3e4 + 100 * torch.sin(i.float())}[kind].float()
    rows = torch.stack([l, l.flip(0), torch.where(i % 7 == 3, -INF, l.double()).float()])
    for top in (1, 20, 32):
        check(rows, torch.tensor([[0, vocab - 1]] * 3), top)


@pytest.mark.parametrize("vocab", [40, 3000, 40000])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("low", [-INF, None])
def test_masks(vocab, t, low):
    """Rows of which a few logits, one, or none are left; masked by -inf or by the type's lowest value."""
    gen = generator(vocab)
    low = torch.finfo(TYPES[t]).min if low is None else low
    l = normal(gen, 6, vocab).to(TYPES[t])
    for row, left in enumerate((vocab, vocab // 2, 9, 3, 1, 0)):
        hidden = torch.randperm(vocab, generator=gen)[: vocab - left]
        l[row, hidden] = low
    tokens = torch.randint(0, vocab, (6, 4), generator=gen)
    tokens[:, 3] = l.float().argmax(1)
    got = check(l, tokens, 12)
    if low == -INF:
        assert got["lse"][5] == -INF and got["entropy"][5] == 0 and (got["logprob"][5] == -INF).all()


def test_tokens_that_are_none():
    gen = generator(2)
    check(normal(gen, 4, 300), torch.tensor([[-1, 5], [300, 299], [-(2 ** 40), 0], [2 ** 40, 7]]), 0)


@pytest.mark.parametrize("vocab", [70, 9000, 40000])
@pytest.mark.parametrize("bad", [math.nan, INF])
def test_rows_with_a_nan_or_an_infinity(vocab, bad):
    gen = generator(3)
    l = normal(gen, 3, vocab)
    l[1, vocab // 2] = bad
    got = run(l, torch.tensor([[0], [1], [2]]), 5)
    for name in ("lse", "entropy", "logprob", "top_logprob"):
        assert got[name][1].isnan().all() and got[name][[0, 2]].isfinite().all(), name
    assert (got["top_index"][1] == -1).all() and (got["top_index"][[0, 2]] >= 0).all()


def test_results_that_are_not_wanted():
    gen = generator(4)
    for vocab in (500, 30000):
        l = normal(gen, 2, vocab).cuda()
        full = run(l.cpu(), torch.tensor([[3], [4]]), 6)
        lp = filled((2, 1), torch.float32)
        ws = filled((xnor.logprobs_workspace_bytes(2, vocab, 0),), torch.uint8)
        xnor.xnor_logprobs(l, torch.tensor([[3], [4]]).cuda(), lp, None, None, None, None, None, ws, 2, vocab, 1, 0)
        assert_within(lp, full["logprob"], 1e-6, "logprob alone")
        i, v = filled((2, 6), torch.int32), filled((2, 6), torch.float32)
        ws = filled((xnor.logprobs_workspace_bytes(2, vocab, 6),), torch.uint8)
        xnor.xnor_logprobs(l, None, None, None, None, None, i, v, ws, 2, vocab, 0, 6)
        assert torch.equal(i, full["top_index"])


def reference_backward(l, tokens, g_lp, g_h):
    l = l.double()
    m = l.amax(1, keepdim=True)
    seen = l > -INF
    log_s = torch.where(torch.isneginf(m), torch.zeros_like(m), (l - m).exp().sum(1, keepdim=True).log())
    lp = torch.where(seen, (l - m) - log_s, torch.zeros_like(l))
    p = torch.where(seen, lp.exp(), torch.zeros_like(l))
    entropy = -(p * lp).sum(1, keepdim=True)
    valid = (tokens >= 0) & (tokens < l.shape[1])
    g = g_lp.double() * valid if g_lp is not None else torch.zeros(tokens.shape, dtype=torch.float64)
    h = g_h.double()[:, None] if g_h is not None else torch.zeros(l.shape[0], 1, dtype=torch.float64)
    out = -p * g.sum(1, keepdim=True) - h * p * (lp + entropy)
    own = torch.zeros_like(l).scatter_add_(1, tokens.clamp(0, l.shape[1] - 1).long(), g)
    size = p * (g.abs().sum(1, keepdim=True) + h.abs() * (lp.abs() + entropy))
    return torch.where(seen, out + own, torch.zeros_like(l)), torch.where(seen, size, torch.zeros_like(l)), own.abs(), entropy[:, 0], torch.cat((m, log_s), 1)


def backward(l, tokens, g_lp, g_h, t, extra=0):
    rows, vocab = l.shape
    want, size, own, entropy, shift = reference_backward(l, tokens, g_lp, g_h)
    g = filled((rows, vocab), TYPES[t])
    xnor.xnor_logprobs_backward(apart(l, extra), tokens.cuda(), shift.float().cuda(), entropy.float().cuda(), g_lp.cuda() if g_lp is not None else None,
                                g_h.cuda() if g_h is not None else None, g, rows, vocab, tokens.shape[1])
    # log p is off by its own roundings and by that of its shift (2e-5 covers differences up to 100), the sums by a few 2^-24
    assert_within(g, want, 2e-5 * size + 2.0 ** -22 * own + HALF_ULP[t] * want.abs() + SMALLEST[t], "g_logits")
    return g


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,given", [(1, 1, 1), (3, 9, 2), (2, 1000, 1), (5, 8191, 3), (2, 8200, 40), (3, 33000, 1)])
def test_backward(t, rows, vocab, given):
    gen = generator(rows + vocab)
    l = normal(gen, rows, vocab, scale=2).to(TYPES[t])
    tokens = torch.randint(0, vocab, (rows, given), generator=gen)
    tokens[0, -1] = tokens[0, 0]                     # the same token twice
    if given > 2:
        tokens[-1, 1] = -1
    g_lp, g_h = normal(gen, rows, given), normal(gen, rows)
    backward(l, tokens, g_lp, g_h, t)
    backward(l, tokens, g_lp, None, t, extra=5)
    backward(l, tokens, None, g_h, t)


def test_backward_of_masked_rows():
    gen = generator(1)
    l = normal(gen, 4, 500)
    l[0, 10:] = -INF
    l[1, 1:] = -INF
    l[2] = -INF
    l[3] = torch.finfo(torch.float32).min
    g = backward(l, torch.tensor([[3, 400], [0, 1], [5, 6], [7, 8]]), normal(gen, 4, 2), normal(gen, 4), "f32")
    assert not g[2].any() and not g[0, 10:].any()


def test_backward_keeps_a_nan_row_nan():
    l = normal(generator(2), 2, 300)
    l[1, 4] = math.nan
    shift = torch.tensor([[0.0, float(torch.logsumexp(l[0], 0))], [1.0, math.nan]]).cuda()
    g = filled((2, 300), torch.float32)
    xnor.xnor_logprobs_backward(l.cuda(), torch.tensor([[1], [2]]).cuda(), shift, None, torch.ones(2, 1).cuda(), None, g, 2, 300, 1)
    assert g[1].isnan().all() and g[0].isfinite().all()


def test_backward_against_differences():
    gen = generator(5)
    l, tokens = normal(gen, 2, 12).double(), torch.tensor([[3, 4], [0, 0]])
    g_lp, g_h = normal(gen, 2, 2).double(), normal(gen, 2).double()

    def loss(l):
        lp = torch.log_softmax(l, 1)
        return (lp.gather(1, tokens) * g_lp).sum() - (g_h * (lp.exp() * lp).sum(1)).sum()

    want = torch.empty_like(l)
    for i in range(2):
        for j in range(12):
            d = torch.zeros_like(l)
            d[i, j] = 1e-5
            want[i, j] = (loss(l + d) - loss(l - d)) / 2e-5
    got = backward(l.float(), tokens, g_lp.float(), g_h.float(), "f32")
    assert_within(got, want, 2e-5 * (1 + want.abs()), "g_logits")


def test_backward_in_place():
    gen = generator(6)
    l = normal(gen, 7, 9100).to(torch.bfloat16)
    tokens, g_lp, g_h = torch.randint(0, 9100, (7, 3), generator=gen), normal(gen, 7, 3), normal(gen, 7)
    want = backward(l, tokens, g_lp, g_h, "bf16")
    _, _, _, entropy, shift = reference_backward(l, tokens, g_lp, g_h)
    same = l.cuda()
    xnor.xnor_logprobs_backward(same, tokens.cuda(), shift.float().cuda(), entropy.float().cuda(), g_lp.cuda(), g_h.cuda(), same, 7, 9100, 3)
    assert torch.equal(same, want)


def test_offsets_past_32_bits():
    """Rows 2^30 elements apart: the third starts 4 GiB behind the first."""
    gap, vocab = 2 ** 30, 9000
    base = torch.empty(2 * gap + vocab, dtype=torch.bfloat16, device="cuda")
    l = base.as_strided((3, vocab), (gap, 1))
    gen = generator(7)
    rows = normal(gen, 3, vocab).to(torch.bfloat16)
    l.copy_(rows.cuda())
    tokens = torch.randint(0, vocab, (3, 1), generator=gen)
    lp, i, v = filled((3, 1), torch.float32), filled((3, 4), torch.int32), filled((3, 4), torch.float32)
    ws = filled((xnor.logprobs_workspace_bytes(3, vocab, 4),), torch.uint8)
    xnor.xnor_logprobs(l, tokens.cuda(), lp, None, None, None, i, v, ws, 3, vocab, 1, 4)
    _, _, logprob, index, _ = reference(rows, tokens, 4)
    assert torch.equal(i.cpu().long(), index)
    assert_within(lp, logprob, 1e-5 * (1 + logprob.abs()), "logprob")


def test_no_rows():
    empty = torch.empty((0, 10), device="cuda")
    xnor.xnor_logprobs(empty, None, None, None, None, None, None, None, None, 0, 10, 0, 0)
    xnor.xnor_logprobs_backward(empty, None, empty, empty, None, empty, empty, 0, 10, 0)
