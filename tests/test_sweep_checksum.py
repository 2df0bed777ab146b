"""The checksum of a sweep's training step sees every word of everything that the step leaves behind."""
import os
import sys
from types import SimpleNamespace

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import sweep_step  # noqa: E402


def left_behind():
    g = torch.Generator().manual_seed(1)
    master = torch.randn((131, 1027), generator=g)                     # 134 537 words, two words 65 536 apart among them
    hidden = torch.randn((7, 33), generator=g).to(torch.bfloat16)      # 462 bytes: the last word is half there
    codes = torch.randint(0, 127, (1001,), generator=g, dtype=torch.uint8)
    return SimpleNamespace(master=master, weight=master.to(torch.bfloat16), hidden=hidden,
                           grad={"hidden": hidden.clone(), "weight": master.to(torch.bfloat16)},
                           out={"loss": torch.randn(7, generator=g), "mean": torch.ones(2)},
                           state={"m": [codes], "m_exp": [codes[:5].clone()]})


def checksum(s):
    return sweep_step.SweepStep.checksum(s)


@pytest.mark.parametrize("bit", [1, 1 << 30])
@pytest.mark.parametrize("word", [0, 1, 12345, 65534, 65535, 65536, 131070, 131071, 131072, 134536])
def test_one_wrong_bit_of_any_word(word, bit):
    s = left_behind()
    first = checksum(s)
    assert checksum(left_behind()) == first
    s.master.view(-1).view(torch.int32)[word] ^= bit
    assert checksum(s) != first


def test_the_last_bytes_of_every_tensor():
    first = checksum(left_behind())
    for find in (lambda s: s.weight, lambda s: s.hidden, lambda s: s.grad["hidden"], lambda s: s.grad["weight"], lambda s: s.out["loss"],
                 lambda s: s.out["mean"], lambda s: s.state["m"][0], lambda s: s.state["m_exp"][0]):
        s = left_behind()
        find(s).view(-1).view(torch.uint8)[-1] ^= 1
        assert checksum(s) != first


def test_words_that_change_places():
    s = left_behind()
    first = checksum(s)
    w = s.master.view(-1)
    w[[5, 65541]] = w[[65541, 5]]
    assert checksum(s) != first
