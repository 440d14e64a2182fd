"""Which stream a call of the binding goes to, where no GPU is needed."""
import importlib.util

import pytest
import torch

from paper_2504_12526_amd import binding


class _Stream:
    cuda_stream = 1234


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_a_torch_without_the_unnamed_questions(monkeypatch, missing):
    """The functions that torch has no public names for may go: the current stream is asked in public then."""
    monkeypatch.delattr(torch._C, missing, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _Stream())
    spec = importlib.util.spec_from_file_location("another_binding", binding.__file__)
    another = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(another)
    assert another._stream(None) == 1234


def test_a_stream_that_is_given_is_taken():
    assert binding._stream(_Stream()) == 1234
