"""The binding of the INT8 product and of beam search: each refusal is the one that is meant."""

import ctypes

import numpy as np
import pytest

from paper_2608_02703_gb300 import archead


class _Library:
    """Stands in for the library: keeps what it is called with and answers OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return archead.OK

        return call


@pytest.fixture
def library(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(archead, "load", lambda: lib)
    return lib


@pytest.mark.parametrize("codes", [
    np.array([[200, 1]], np.int16), np.array([[-129, 0]], np.int64), np.array([[128, 0]], np.uint8),
    np.array([[1.5, 0]], np.float32), np.array([[np.nan, 0]], np.float32), np.array([[np.inf, 0]]),
], ids=str)
def test_codes_that_int8_does_not_hold_are_refused(library, codes):
    with pytest.raises(ValueError, match="int8 does not hold"):
        archead.archead_int8_weight_create(codes, np.ones(1, np.float32), stream=0)
    assert not library.calls


@pytest.mark.parametrize("dtype", [np.int8, np.int16, np.int64, np.float32])
def test_codes_that_int8_holds_are_taken(library, dtype):
    codes = np.array([[-128, 127, 0], [5, -6, 7]], dtype)
    for given in (codes, np.asfortranarray(codes)):
        archead.archead_int8_weight_create(given, np.ones(2, np.float32), stream=0)
    assert len(library.calls) == 2
