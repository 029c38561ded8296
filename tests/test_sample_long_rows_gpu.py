"""Draws from single rows of vocabularies past a quarter of a million: parts of a row in workgroups of their own, up to 64 of them, and the row in one workgroup beyond."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import TYPES, generator, normal
from tests.test_sample_gpu import check

PART_TOKENS, MOST_PARTS = 8184, 64


@pytest.mark.parametrize("vocab", [261888, 261889, 262144, 300000, PART_TOKENS * MOST_PARTS])
def test_a_long_row_is_taken_in_parts(vocab):
    """(without a GPU) One row needs what its parts hand on, and a few rows as much each; from 256 workgroups on there is nothing to hand on."""
    parts = -(-vocab // PART_TOKENS)
    one = xnor.sample_workspace_bytes(1, vocab)
    assert one > 0 and one % parts == 0
    most = 256 // parts
    assert [xnor.sample_workspace_bytes(rows, vocab) for rows in (most, most + 1, 5000)] == [most * one] * 3
    assert xnor.sample_workspace_bytes(1, PART_TOKENS * MOST_PARTS + 1) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("name,rows,vocab", [("bf16", 1, 262144), ("f32", 2, 262145), ("f16", 5, 300007), ("f32", 4, PART_TOKENS * MOST_PARTS), ("bf16", 1, PART_TOKENS * MOST_PARTS - 9),
                                             ("f32", 5, PART_TOKENS * MOST_PARTS), ("f32", 1, PART_TOKENS * MOST_PARTS + 1)])
def test_long_rows(name, rows, vocab):
    gen = generator(vocab)
    logits = (3 * normal(gen, rows, vocab)).to(TYPES[name])
    if rows > 1:
        logits[1, : vocab // 2] = -float("inf")
    for u in (torch.rand(rows, generator=gen), torch.full((rows,), 0.999)):
        check(logits, u)
        check(logits, u, top_p=0.95)
        check(logits, u, temperature=0.7, top_p=0.9, min_p=0.002)
        check(logits, u, temperature=1.5, top_k=20000, min_p=1e-4)


@pytest.mark.gpu
def test_long_rows_all_alike():
    """More tokens of one size than a list holds: found by their places."""
    vocab = 300000
    check(torch.zeros((1, vocab), dtype=torch.bfloat16), torch.tensor([0.7]), top_p=0.5)
    check(torch.zeros((2, vocab)), torch.tensor([0.1, 0.9999999]))
