"""The binding's part of drafted tokens, where no GPU is needed."""
import types

import pytest
import torch

from paper_2504_12526_amd import binding


def test_children_of_trees_are_not_passed_over_unsaid(monkeypatch):
    """A tree without a number of children to try is refused, where all but the first of a row would be lost; a chain has one."""
    asked = []

    class Library:
        def mom_verify_drafts(self, *args):
            asked.append(args[8])
            return 0

    monkeypatch.setattr(binding, "_lib", Library())
    rows, counts, u = torch.zeros(6, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(6)
    call = lambda **more: binding.mom_verify_drafts(torch.zeros(6, 50), rows, u, rows, rows, counts, torch.zeros(9, dtype=torch.uint8), stream=types.SimpleNamespace(cuda_stream=None), **more)
    with pytest.raises(ValueError, match="max_children"):
        call(parents=rows)
    assert asked == []
    call(parents=rows, max_children=3)
    call(parents=rows, max_children=1)
    call()
    assert asked == [3, 1, 1]
