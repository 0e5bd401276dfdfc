"""Decoder layers' own arguments (no GPU is touched)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2410_14740_amd import decoder


@pytest.mark.parametrize("budget", [1, 2, 3, 7])
def test_evict_keeps_within_any_budget(budget):
    layer = object.__new__(decoder.DecoderLayer)
    calls = []
    layer.budget = budget
    layer.cache = SimpleNamespace(evict=lambda *a: calls.append(a))
    layer.evict()
    layer.evict(first=budget, recent=budget)
    (keep, first, recent), (_, most, rest) = calls
    assert keep == budget and first == 1 and recent == min(2, budget - 1)
    assert most == budget and rest == 0


def test_a_negative_budget_is_refused():
    with pytest.raises(ValueError, match="budget -1"):
        decoder.DecoderLayer(None, 1, 1, 0, 1, 8, 2, 64, (None, None), budget=-1)


def test_a_prompt_without_tokens_is_refused():
    with pytest.raises(ValueError, match="without tokens"):
        decoder.run([], [torch.zeros(3, 8), torch.zeros(0, 8)], 1)


def test_a_negative_number_of_tokens_is_refused(capsys):
    with pytest.raises(SystemExit):
        decoder.main(["--tokens", "-1"])
    assert "--tokens -1" in capsys.readouterr().err
