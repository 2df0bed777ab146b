"""What a sweep's training step is said to move and compute, part by part, against a count of it."""
import os
import sys
from types import SimpleNamespace

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import sweep_step  # noqa: E402


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rows,vocab,width,left_out", [(7, 11, 24, 0), (100, 40, 8, 25), (64, 64, 16, 64)])
def test_work_of_the_parts(rows, vocab, width, left_out, bits):
    tokens = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(rows))
    targets = torch.arange(rows) % vocab
    targets[:left_out] = -1
    got = sweep_step.SweepStep.work(SimpleNamespace(rows=rows, vocab=vocab, width=width, bits=bits, tokens=tokens, targets=targets))
    moved = 0
    for _ in range(rows):                       # a token there and back, a looked-up row written, its gradient read
        moved += 2 * 8 + 2 * width * 2
    for _ in set(tokens.tolist()):              # a row of the table read; of its gradient read and written
        moved += 3 * width * 2
    assert got["lookup"] == moved
    product = lambda n: 2 * n * vocab * width                                           # noqa: E731
    assert got["loss"] == product(rows) + 3 * product(rows - left_out)
    # master and gradient read, master and copy written, two states read and written
    assert got["update"] == vocab * width * (4 + 2 + 4 + 2 + 2 * 2 * (4 if bits == 32 else 1))
