"""Objects that count the same dropout numbers drop the same elements: the second one to do so warns.  CPU only; calls that would enqueue work are written down instead."""
import gc
import warnings

import pytest
import torch

import paper_2506_01352_amd as tahq
from paper_2506_01352_amd import binding
from test_classes_host import library  # noqa: F401


@pytest.fixture
def dropout(library, monkeypatch):  # noqa: F811
    monkeypatch.setattr(binding, "_whole", lambda where, name, t, *rest: t.data_ptr())
    gc.collect()
    return lambda seed=0, offset=0, **more: tahq.Dropout(tahq.make_dropout_config(64, tahq.F32, 0.5, seed, offset), device="cpu", **more)


X = torch.zeros(64)


def test_the_same_numbers_twice(dropout):
    first, second = dropout(), dropout()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        first.forward(X)
        first.forward(X)
    with pytest.warns(UserWarning, match="under seed 0"):
        second.forward(X)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        second.forward(X)                                # once


def test_numbers_of_their_own(dropout):
    """Other seeds, other offsets, offsets that the caller counts, an object that is gone, a graph's offset of its own."""
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        kept = [dropout(), dropout(seed=1), dropout(offset=1 << 32), dropout(graph_offset=torch.zeros(1, dtype=torch.int64))]
        for drop in kept:
            drop.forward(X)
        again = dropout()
        again.forward(X, offset=0)
        again.backward(X, offset=0)
        del kept, drop
        gc.collect()
        again.forward(X)
