"""xnor_logprobs where one logit is all that counts: a log probability is never above 0 and an entropy never below."""
import math

import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import TYPES, filled, generator, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 40, 1000, 3000, 20000])
@pytest.mark.parametrize("others", [-math.inf, -200.0, "lowest"])
@pytest.mark.parametrize("top", [0, 2])
def test_a_single_survivor(t, vocab, others, top):
    """Rows of one logit of any size among masks: its log probability and the entropy are 0, to the bit."""
    gen = generator(vocab)
    rows = 500
    others = torch.finfo(TYPES[t]).min if others == "lowest" else others
    l = torch.full((rows, vocab), others)
    at = torch.randint(0, vocab, (rows,), generator=gen)
    l[torch.arange(rows), at] = normal(gen, rows, scale=20) + 40
    out = {"logprob": filled((rows, 1), torch.float32), "lse": filled((rows,), torch.float32), "shift": filled((rows, 2), torch.float32),
           "entropy": filled((rows,), torch.float32), "index": filled((rows, top), torch.int32), "value": filled((rows, top), torch.float32)}
    size = xnor.logprobs_workspace_bytes(rows, vocab, top)
    l = l.to(TYPES[t])
    xnor.xnor_logprobs(l.cuda(), at[:, None].cuda(), out["logprob"], out["lse"], out["shift"], out["entropy"], out["index"] if top else None,
                       out["value"] if top else None, filled((size,), torch.uint8) if size else None, rows, vocab, 1, top)
    kept = l.float().amax(1)
    assert not out["logprob"].any() and not out["entropy"].any() and not out["shift"][:, 1].any()
    assert torch.equal(out["lse"].cpu(), kept) and torch.equal(out["shift"][:, 0].cpu(), kept)
    if top:
        assert torch.equal(out["index"][:, 0].cpu().long(), at) and not out["value"][:, 0].any() and (out["value"][:, 1] <= -100).all()


@pytest.mark.parametrize("vocab", [3, 700, 30000])
def test_signs_near_a_single_survivor(vocab):
    """The others' share falls from all to nothing: still no log probability above 0, no entropy below."""
    gen = generator(vocab)
    rows = 400
    l = normal(gen, rows, vocab)
    at = torch.randint(0, vocab, (rows,), generator=gen)
    l[torch.arange(rows), at] = torch.linspace(0, 60, rows)
    lp, entropy = filled((rows, 1), torch.float32), filled((rows,), torch.float32)
    index, value = filled((rows, 3), torch.int32), filled((rows, 3), torch.float32)
    ws = filled((xnor.logprobs_workspace_bytes(rows, vocab, 3),), torch.uint8)
    xnor.xnor_logprobs(l.cuda(), at[:, None].cuda(), lp, None, None, entropy, index, value, ws, rows, vocab, 1, 3)
    assert (lp <= 0).all() and (entropy >= 0).all() and (value <= 0).all()
