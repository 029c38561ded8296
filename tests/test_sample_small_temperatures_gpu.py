"""Draws at temperatures that float32 hardly holds, from logits as close together: a logit's distance in temperatures is what counts, and how many there are of it."""
import pytest
import torch

from tests.lowbit_helpers import generator
from tests.test_sample_gpu import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("step", [0.02, 1.0, 30.0, 900.0, 2e4, 3e6])
@pytest.mark.parametrize("temperature", [1e-44, 3e-41, 1e-39, 3e-38, 4e-37, 1e-35])
@pytest.mark.parametrize("rows,vocab", [(24, 3000), (1, 60001)])
def test_logits_a_few_temperatures_apart(rows, vocab, temperature, step):
    gen = generator(vocab + int(step * 100))
    place = torch.stack([torch.randperm(vocab, generator=gen) for _ in range(rows)])
    logits = (-(place.double() * step * temperature)).float()                # (of the smallest temperatures a few differ by nothing: subnormal numbers)
    u = torch.rand(rows, generator=gen)
    check(logits, u, temperature=temperature)
    check(logits, u, temperature=temperature, top_p=0.9)
    check(logits, u, temperature=temperature, top_k=2000, top_p=0.999)
    check(logits, u, temperature=temperature, min_p=1e-3)


def test_a_row_with_larger_ones_beside_them():
    """Logits of ordinary size below, and above, ones that differ by less than float32's smallest normal number."""
    gen = generator(5)
    rows, vocab = 16, 4000
    logits = 1e-39 * torch.randint(0, 50, (rows, vocab), generator=gen).float()
    logits[:, ::3] = -torch.rand((rows, len(range(0, vocab, 3))), generator=gen) * 10.0 ** torch.randint(-38, 38, (rows, 1), generator=gen)
    u = torch.rand(rows, generator=gen)
    for temperature in (1e-45, 1e-40, 2e-39, 1e-38, 1e-20):
        check(logits, u, temperature=temperature)
        check(logits, u, temperature=temperature, top_p=0.7)
    logits[:, 5], logits[:, 6] = 3e30, -3e38
    for temperature in (1e-45, 1e-40, 1e-20, 1e30):
        check(logits, u, temperature=temperature)
