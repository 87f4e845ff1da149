"""Which pairs of outputs and inputs of one shape the op-level wrappers take: the same rows, or
rows that share no memory."""
import pytest
import torch

from paper_2608_10362_gb300.engine import _same_or_apart


def _at(offset, rows, n, ld, raw=torch.zeros(4096)):
    return torch.as_strided(raw, (rows, n), (ld, 1), offset)


@pytest.mark.parametrize("a,b", [
    ((0, 3, 10, 12), (0, 3, 10, 12)),        # the same rows
    ((0, 3, 10, 24), (12, 3, 10, 24)),       # beside one another in the rows of one tensor
    ((12, 3, 10, 24), (0, 3, 10, 24)),
    ((0, 3, 10, 12), (36, 3, 10, 17)),       # apart
    ((5, 1, 10, 10), (5, 1, 10, 64)),        # one row: its stride says nothing
    ((5, 1, 10, 0), (5, 1, 10, 10)),
    ((0, 1, 10, 0), (10, 1, 10, 0)),
])
def test_taken(a, b):
    _same_or_apart("out", _at(*a), "logits", _at(*b))


@pytest.mark.parametrize("a,b", [
    ((0, 3, 10, 12), (1, 3, 10, 12)), ((0, 3, 10, 12), (0, 3, 10, 13)), ((0, 3, 10, 24), (15, 3, 10, 24)),
    ((0, 3, 10, 24), (12, 3, 10, 25)), ((5, 1, 10, 10), (6, 1, 10, 10)), ((5, 1, 10, 0), (6, 1, 10, 0)),
    ((5, 1, 10, 30), (6, 1, 10, 30)), ((6, 1, 10, 0), (5, 1, 10, 64)),
])
def test_refused(a, b):
    with pytest.raises(ValueError):
        _same_or_apart("out", _at(*a), "logits", _at(*b))


def test_one_column():
    raw = torch.zeros(64)
    a, b = torch.as_strided(raw, (3, 1), (5, 1), 0), torch.as_strided(raw, (3, 1), (5, 7), 0)
    _same_or_apart("out", a, "logits", b)
    _same_or_apart("out", a, "logits", torch.as_strided(raw, (3, 1), (5, 1), 2))
