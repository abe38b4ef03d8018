"""The binding of the INT8 product and of beam search: each refusal is the one that is meant."""

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


class _OnGpu:
    """A tensor of the host that says it is on the GPU (its address goes to the stand-in library only)."""

    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0

    def view(self, *args):
        return _OnGpu(self.t.view(*args))


def _t(*shape, dtype="float32"):
    import torch

    return _OnGpu(torch.zeros(shape, dtype=getattr(torch, dtype)))


def _quantize(**kw):
    a = dict(x=_t(3, 6), codes=_t(3, 6, dtype="int8"), scales=_t(3)) | kw
    archead.archead_int8_quantize_tokens(a["x"], a["codes"], a["scales"], stream=0)


def _matmul(**kw):
    a = dict(codes=_t(3, 6, dtype="int8"), scales=_t(3), M=3, y=_t(3, 10)) | kw
    archead.archead_int8_matmul(archead.Int8Weight(None, 10, 6), a["codes"], a["scales"], a["M"], a["y"], stream=0)


def _select(**kw):
    a = dict(logits=_t(6, 9), scores=_t(2, 3), out_scores=_t(2, 4), out_parents=_t(2, 4, dtype="int32"),
             out_tokens=_t(2, 4, dtype="int32"), ended=None) | kw
    archead.archead_beam_select(archead.Beam(None), **a, stream=0)


ELEMENTS = "contiguous elements"


@pytest.mark.parametrize("call,kw", [
    (_quantize, dict(codes=_t(3, 7, dtype="int8"))), (_quantize, dict(x=_t(3, 1), codes=_t(3, 6, dtype="int8"))),
    (_matmul, dict(codes=_t(3, 8, dtype="int8"))), (_matmul, dict(codes=_t(4, 5, dtype="int8"))),
    (_select, dict(out_parents=_t(2, 5, dtype="int32"))), (_select, dict(out_tokens=_t(3, 3, dtype="int32"))),
    (_select, dict(ended=_t(2, 4, dtype="uint8"))),
])
def test_larger_matrices_of_other_rows_are_refused(library, call, kw):
    with pytest.raises(ValueError, match=ELEMENTS):
        call(**kw)
    assert not library.calls


@pytest.mark.parametrize("call,kw", [
    (_quantize, dict()), (_quantize, dict(codes=_t(5, 6, dtype="int8"))), (_quantize, dict(codes=_t(100, dtype="int8"))),
    (_quantize, dict(codes=_t(9, 2, dtype="int8"))), (_matmul, dict()), (_matmul, dict(codes=_t(4, 6, dtype="int8"))),
    (_matmul, dict(codes=_t(3, 2, 3, dtype="int8"))), (_matmul, dict(M=0)), (_select, dict()),
    (_select, dict(out_parents=_t(5, 4, dtype="int32"), out_tokens=_t(50, dtype="int32"))),
    (_select, dict(ended=_t(2, 3, dtype="uint8"))), (_select, dict(ended=_t(2, 3, dtype="bool"))),
    (_select, dict(ended=_t(4, 3, dtype="uint8"))),
])
def test_matrices_with_room_to_spare_are_taken(library, call, kw):
    """More rows than the call needs, a flat buffer, or the same elements in another shape."""
    call(**kw)
    assert len(library.calls) == 1


@pytest.mark.parametrize("kw", [dict(row_dim=4), dict(row_dim=-5), dict(length_dim=4), dict(length_dim=-5)], ids=str)
def test_dimensions_that_a_state_has_not_are_refused(kw):
    import torch

    t = torch.empty((2, 6, 8, 10))
    with pytest.raises(ValueError, match="has no dimension"):
        archead.archead_beam_state(t, **kw)
    with pytest.raises(ValueError, match="has no dimension"):
        archead.archead_beam_state(torch.tensor(1.0))
    a, b = archead.archead_beam_state(t, row_dim=-3, length_dim=-2), archead.archead_beam_state(t, row_dim=1, length_dim=2)
    assert (a.rows, a.room) == (b.rows, b.room) == (6, 8)


def _linear(**kw):
    a = dict(x=_t(3, 6), M=3, y=_t(3, 10)) | kw
    archead.archead_int8_linear(archead.Int8Weight(None, 10, 6), a["x"], a["M"], a["y"], stream=0)


def _on_host(*shape, dtype="float32"):
    return _t(*shape, dtype=dtype).t


def _transposed(*shape, dtype="float32"):
    return _OnGpu(_t(*shape, dtype=dtype).t.t())


ROWS = "adjacent elements"
HOST = "not on the GPU"
TYPE = "bf16, fp16 or fp32"


@pytest.mark.parametrize("call,kw,message", [
    (_linear, dict(x=_t(3, 7)), ROWS), (_linear, dict(x=_t(2, 6)), ROWS), (_linear, dict(M=4), ROWS),
    (_linear, dict(x=_t(18)), ROWS), (_linear, dict(x=_transposed(6, 3)), ROWS), (_linear, dict(y=_t(3, 9)), ROWS),
    (_linear, dict(y=_transposed(10, 3)), ROWS), (_linear, dict(x=_t(3, 6, dtype="float64")), TYPE),
    (_linear, dict(y=_t(3, 10, dtype="float64")), TYPE), (_linear, dict(y=_t(3, 10, dtype="int32")), TYPE),
    (_linear, dict(x=_on_host(3, 6)), HOST), (_linear, dict(y=_on_host(3, 10)), HOST),
    (_matmul, dict(codes=_t(3, 6)), ELEMENTS), (_matmul, dict(codes=_t(2, 6, dtype="int8")), ELEMENTS),
    (_matmul, dict(codes=_transposed(6, 3, dtype="int8")), ELEMENTS), (_matmul, dict(scales=_t(2)), ELEMENTS),
    (_matmul, dict(scales=_t(3, dtype="float64")), ELEMENTS), (_matmul, dict(y=_t(3, 11)), ROWS),
    (_matmul, dict(M=4), ROWS), (_matmul, dict(y=_t(3, 10, dtype="int8")), TYPE),
    (_matmul, dict(codes=_on_host(3, 6, dtype="int8")), HOST), (_matmul, dict(scales=_on_host(3)), HOST),
    (_matmul, dict(y=_on_host(3, 10)), HOST),
    (_quantize, dict(codes=_t(3, 6, dtype="uint8")), ELEMENTS), (_quantize, dict(codes=_t(2, 6, dtype="int8")), ELEMENTS),
    (_quantize, dict(scales=_t(2)), ELEMENTS), (_quantize, dict(x=_transposed(6, 3)), ROWS),
    (_quantize, dict(x=_t(3, 6, dtype="int32")), TYPE), (_quantize, dict(x=_on_host(3, 6)), HOST),
    (_quantize, dict(codes=_on_host(3, 6, dtype="int8")), HOST), (_quantize, dict(scales=_on_host(3)), HOST),
    (_select, dict(logits=_t(5, 9)), ROWS), (_select, dict(logits=_transposed(9, 6)), ROWS),
    (_select, dict(logits=_t(6, 9, dtype="float64")), TYPE), (_select, dict(scores=_t(2, 3, dtype="float64")), ELEMENTS),
    (_select, dict(scores=_transposed(3, 2)), ELEMENTS), (_select, dict(scores=_t(3, 3)), ROWS),
    (_select, dict(out_scores=_t(2, 4, dtype="float16")), ELEMENTS), (_select, dict(out_scores=_t(1, 4)), ELEMENTS),
    (_select, dict(out_scores=_t(2, 5)), ELEMENTS), (_select, dict(out_parents=_t(2, 4, dtype="int64")), ELEMENTS),
    (_select, dict(out_parents=_t(1, 4, dtype="int32")), ELEMENTS), (_select, dict(out_tokens=_t(2, 4)), ELEMENTS),
    (_select, dict(out_tokens=_t(2, 3, dtype="int32")), ELEMENTS), (_select, dict(ended=_t(2, 2, dtype="uint8")), ELEMENTS),
    (_select, dict(ended=_t(2, 3, dtype="int32")), ELEMENTS), (_select, dict(logits=_on_host(6, 9)), HOST),
    (_select, dict(scores=_on_host(2, 3)), HOST), (_select, dict(ended=_on_host(2, 3, dtype="uint8")), HOST),
    (_select, dict(out_scores=_on_host(2, 4)), HOST), (_select, dict(out_tokens=_on_host(2, 4, dtype="int32")), HOST),
])
def test_one_wrong_argument_is_refused_for_what_is_wrong(library, call, kw, message):
    call()
    assert len(library.calls) == 1  # the same call with the right argument
    with pytest.raises(ValueError, match=message):
        call(**kw)
    assert len(library.calls) == 1


@pytest.mark.parametrize("codes,scales,message", [
    (np.zeros((3, 4), np.int8), np.zeros(4, np.float32), "a scale for each"),
    (_on_host(3, 4), _on_host(3), "codes in int8"), (_on_host(3, 4, dtype="int8"), _on_host(3, dtype="float64"), "codes in int8"),
    (_on_host(3, 4, dtype="int8"), _on_host(4), "a scale for each"),
])
def test_weights_are_refused_for_what_is_wrong(library, codes, scales, message):
    with pytest.raises(ValueError, match=message):
        archead.archead_int8_weight_create(codes, scales, stream=0)
    assert not library.calls
    archead.archead_int8_weight_create(_on_host(3, 4, dtype="int8"), _on_host(3), stream=0)
    assert len(library.calls) == 1


def _reorder(states, parents, length):
    archead.archead_beam_reorder(states, parents, length, stream=0)


def test_reorderings_are_refused_for_what_is_wrong(library):
    def states(*t):
        s = archead.archead_beam_states([archead.archead_beam_state(a, length_dim=2) for a in t])
        s.on_gpu = True
        return s

    cache, parents = _on_host(4, 6, 8, 10), _t(2, 2, dtype="int32")
    good = states(cache, cache)
    _reorder(good, parents, 8)
    assert len(library.calls) == 1
    _, args = library.calls[0]
    assert args[1:3] == (2, parents.data_ptr()) and args[3:6] == (2, 2, 8)
    for bad, message in ((lambda: _reorder(good, parents, 9), "positions"),
                         (lambda: _reorder(good, _t(3, 2, dtype="int32"), 8), "rows"),
                         (lambda: _reorder(states(cache, cache[:3]), parents, 8), "rows"),
                         (lambda: _reorder(good, _t(2, 2, dtype="int64"), 8), ELEMENTS),
                         (lambda: _reorder(good, _transposed(2, 2, dtype="int32"), 8), ELEMENTS),
                         (lambda: _reorder(good, _on_host(2, 2, dtype="int32"), 8), HOST),
                         (lambda: _reorder(archead.archead_beam_states([archead.archead_beam_state(cache)]), parents, 8),
                          "a state is not on the GPU")):
        with pytest.raises(ValueError, match=message):
            bad()
    assert len(library.calls) == 1
