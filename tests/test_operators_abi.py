"""Refusals of the INT8 product and of beam search: argument checks answer
before any work is queued (no device is needed)."""

import ctypes

import numpy as np
import pytest

from paper_2608_02703_gb300 import archead
from paper_2608_02703_gb300.build import build

BAD = archead.ERR_INVALID_ARG
P = ctypes.c_void_p  # addresses below are never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    build()
    return archead.load()


@pytest.mark.parametrize("codes,scales,N,K,want", [
    (None, P(16), 4, 8, BAD), (P(16), None, 4, 8, BAD), (P(16), P(16), 0, 8, BAD), (P(16), P(16), -1, 8, BAD),
    (P(16), P(16), 4, 0, BAD), (P(16), P(16), 4, 1 << 17, archead.ERR_UNSUPPORTED),
    (P(16), P(16), 1 << 31, 8, archead.ERR_UNSUPPORTED),
])
def test_int8_weight_create_refuses(lib, codes, scales, N, K, want):
    out = P(1234)
    assert lib.archead_int8_weight_create(codes, scales, N, K, None, ctypes.byref(out)) == want
    assert out.value is None
    assert lib.archead_int8_weight_create(codes, scales, N, K, None, None) == BAD


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(dtype=3), BAD), (dict(dtype=-1), BAD),
    (dict(M=-1), BAD), (dict(K=0), BAD), (dict(ldx=7), BAD), (dict(x=P(17)), BAD), (dict(x=P(18), dtype=1), BAD),
    (dict(codes=P(24)), BAD), (dict(scales=P(24)), BAD), (dict(M=0), archead.OK),
    (dict(M=0, x=None, codes=None, scales=None), archead.OK), (dict(M=(1 << 30) + 1), archead.ERR_UNSUPPORTED),
])
def test_int8_quantize_refuses(lib, kw, want):
    a = dict(x=P(16), dtype=0, M=4, K=8, ldx=8, codes=P(32), scales=P(48)) | kw
    st = lib.archead_int8_quantize_tokens(a["x"], a["dtype"], a["M"], a["K"], a["ldx"], a["codes"], a["scales"], None)
    assert st == want


def test_null_handles(lib):
    assert lib.archead_int8_matmul(None, P(16), P(16), 1, P(16), 0, 8, None) == BAD
    assert lib.archead_int8_matmul_path(None, P(16), P(16), 1, P(16), 0, 8, 0, None) == BAD
    assert lib.archead_int8_linear(None, P(16), 0, 1, 8, P(16), 0, 8, None) == BAD
    assert lib.archead_int8_sync_status(None, None) == BAD
    assert lib.archead_int8_set_wait_budget(None, 5) == BAD
    assert lib.archead_int8_device_bytes(None) == -1
    lib.archead_int8_weight_destroy(None)
    lib.archead_beam_destroy(None)
    assert lib.archead_beam_select(None, P(16), 0, 1, 1, 4, 4, P(16), None, 0, 1, P(16), P(16), P(16), None) == BAD


@pytest.mark.parametrize("rows,vocab,n,want", [
    (0, 8, 1, BAD), (1, 0, 1, BAD), (1, 8, 0, BAD), (1, 8, 65, BAD), ((1 << 20) + 1, 8, 1, archead.ERR_UNSUPPORTED),
    (1, (1 << 30) + 1, 1, archead.ERR_UNSUPPORTED),
])
def test_beam_create_refuses(lib, rows, vocab, n, want):
    out = P(1234)
    assert lib.archead_beam_create(rows, vocab, n, ctypes.byref(out)) == want
    assert out.value is None
    assert lib.archead_beam_create(rows, vocab, n, None) == BAD


def _state(**kw):
    a = dict(data=4096, out=None, outer=2, outer_stride=1024, row_stride=256, inner=2, inner_stride=128, bytes=64,
             bytes_per_position=0) | kw
    return archead.archead_beam_state_t(**a)


@pytest.mark.parametrize("kw", [
    dict(data=None), dict(out=4096), dict(outer=-1), dict(inner=-1), dict(bytes=-1), dict(bytes_per_position=-1),
    dict(outer_stride=-1024), dict(row_stride=-256), dict(inner_stride=-128), dict(inner_stride=63),
    dict(row_stride=63), dict(outer_stride=63), dict(bytes=129), dict(bytes=0, bytes_per_position=13),
    dict(bytes_per_position=1 << 62), dict(bytes=1 << 62), dict(outer=1 << 40, inner=1 << 30), dict(inner=1 << 32),
    dict(outer=1 << 58, inner=1 << 2, outer_stride=1 << 50),
])
def test_beam_reorder_refuses_states(lib, kw):
    states = (archead.archead_beam_state_t * 2)(_state(), _state(**kw))  # (the first one is not moved either)
    assert lib.archead_beam_reorder(states, 2, P(16), 1, 4, 10, None) == BAD


@pytest.mark.parametrize("kw,want", [
    (dict(states=None), BAD), (dict(count=-1), BAD), (dict(parents=None), BAD), (dict(parents=P(18)), BAD),
    (dict(batch=-1), BAD), (dict(beams=0), BAD), (dict(beams=65), BAD), (dict(length=-1), BAD),
    (dict(batch=(1 << 30) + 1), archead.ERR_UNSUPPORTED),
    (dict(count=0), archead.OK), (dict(batch=0), archead.OK), (dict(count=0, states=None), archead.OK),
])
def test_beam_reorder_refuses(lib, kw, want):
    states = (archead.archead_beam_state_t * 1)(_state())
    a = dict(states=states, count=1, parents=P(16), batch=1, beams=4, length=10) | kw
    st = lib.archead_beam_reorder(a["states"], a["count"], a["parents"], a["batch"], a["beams"], a["length"], None)
    assert st == want


def test_states_that_move_nothing_are_accepted(lib):
    states = (archead.archead_beam_state_t * 3)(_state(outer=0), _state(inner=0), _state(bytes=0, data=None))
    assert lib.archead_beam_reorder(states, 3, P(16), 1, 4, 0, None) == archead.OK


# ------------------------------------------------------------------------
# The binding's own checks and descriptions (CPU tensors: addresses only).
# ------------------------------------------------------------------------
def _fields(s):
    return {k: getattr(s.desc, k) for k, _ in s.desc._fields_[2:]}


def test_state_descriptions():
    import torch

    cache = torch.empty((3, 8, 4, 20, 6), dtype=torch.float16)  # layer, row, head, position, element
    s = archead.archead_beam_state(cache, row_dim=1, length_dim=3)
    assert _fields(s) == dict(outer=3, outer_stride=8 * 4 * 20 * 6 * 2, row_stride=4 * 20 * 6 * 2, inner=4,
                              inner_stride=20 * 6 * 2, bytes=0, bytes_per_position=12)
    assert (s.rows, s.room) == (8, 20)
    s = archead.archead_beam_state(cache[:, :, 1:3], row_dim=1, length_dim=3)  # some heads
    assert (s.desc.inner, s.desc.row_stride) == (2, 4 * 20 * 6 * 2)
    s = archead.archead_beam_state(cache[0, :, 0, 0])  # rows a distance apart
    assert _fields(s) == dict(outer=1, outer_stride=0, row_stride=960, inner=1, inner_stride=0, bytes=12,
                              bytes_per_position=0)
    s = archead.archead_beam_state(torch.empty((5, 7, 3), dtype=torch.int32))
    assert (s.desc.bytes, s.desc.inner, s.desc.row_stride) == (84, 1, 84)
    s = archead.archead_beam_state(torch.empty((5, 7), dtype=torch.int32), length_dim=1)
    assert (s.desc.bytes, s.desc.bytes_per_position, s.room) == (0, 4, 7)
    s = archead.archead_beam_state(torch.empty((7, 5, 3)).transpose(0, 1))  # rows in the middle
    assert _fields(s) == dict(outer=1, outer_stride=0, row_stride=12, inner=7, inner_stride=60, bytes=12,
                              bytes_per_position=0)
    s = archead.archead_beam_state(torch.empty(6))
    assert (s.desc.bytes, s.desc.row_stride) == (4, 4)


def test_state_descriptions_refuse():
    import torch

    t = torch.empty((4, 6, 8, 10))
    for bad in (lambda: archead.archead_beam_state(t, out=torch.empty((4, 6, 8, 11))),
                lambda: archead.archead_beam_state(t, out=torch.empty((4, 6, 8, 10), dtype=torch.float16)),
                lambda: archead.archead_beam_state(t, row_dim=2, length_dim=1),
                lambda: archead.archead_beam_state(t[..., ::2], length_dim=2),
                lambda: archead.archead_beam_state(t[:, :, ::2], length_dim=2),
                lambda: archead.archead_beam_state(t[:, ::2].transpose(1, 2), row_dim=3),
                lambda: archead.archead_beam_state(t.permute(0, 2, 1, 3)[:, ::3, :, ::3], row_dim=0)):
        with pytest.raises(ValueError):
            bad()
    states = archead.archead_beam_states([archead.archead_beam_state(t, length_dim=2)])
    parents = torch.zeros((2, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        archead.archead_beam_reorder(states, parents, 9)  # more positions than there is room for
    with pytest.raises(ValueError):
        archead.archead_beam_reorder(states, torch.zeros((3, 2), dtype=torch.int32), 3)  # more rows
    with pytest.raises(ValueError):
        archead.archead_beam_reorder(states, parents.long(), 3)


def test_binding_refuses_shapes_and_types():
    import torch

    w = archead.Int8Weight(None, 10, 6)
    f32 = torch.float32
    y = torch.empty((3, 10))
    for bad in (lambda: archead.archead_int8_linear(w, torch.empty((3, 7)), 3, y),
                lambda: archead.archead_int8_linear(w, torch.empty((2, 6)), 3, y),
                lambda: archead.archead_int8_linear(w, torch.empty((3, 6)), 3, torch.empty((10, 3)).t()),
                lambda: archead.archead_int8_linear(w, torch.empty((3, 6), dtype=torch.float64), 3, y),
                lambda: archead.archead_int8_matmul(w, torch.empty((3, 6)), torch.empty(3), 3, y),
                lambda: archead.archead_int8_matmul(w, torch.empty((3, 6), dtype=torch.int8), torch.empty(2), 3, y),
                lambda: archead.archead_int8_quantize_tokens(y, torch.empty(30, dtype=torch.uint8), torch.empty(3)),
                lambda: archead.archead_int8_quantize_tokens(y.t(), torch.empty(30, dtype=torch.int8), torch.empty(10)),
                lambda: archead.archead_int8_weight_create(np.zeros((3, 4), np.int8), np.zeros(4, np.float32)),
                lambda: archead.archead_int8_weight_create(torch.zeros(3, 4), torch.zeros(3))):
        with pytest.raises(ValueError):
            bad()
    beam = archead.Beam(None)
    i = torch.empty((2, 4), dtype=torch.int32)
    good = dict(logits=torch.empty((6, 9)), scores=torch.empty((2, 3)), out_scores=torch.empty((2, 4)), out_parents=i,
                out_tokens=i)
    for kw in (dict(logits=torch.empty((5, 9))), dict(logits=torch.empty((9, 6)).t()),
               dict(scores=torch.empty((2, 3), dtype=torch.float64)), dict(out_parents=i.long()),
               dict(ended=torch.zeros((2, 2), dtype=torch.uint8)), dict(ended=torch.zeros((2, 3), dtype=torch.int32))):
        with pytest.raises(ValueError):
            archead.archead_beam_select(beam, **(good | kw))
    assert f32 == y.dtype


def test_binding_refuses_tensors_on_the_host():
    import torch

    w, beam = archead.Int8Weight(None, 10, 6), archead.Beam(None)
    x, y, c, s = torch.empty((3, 6)), torch.empty((3, 10)), torch.empty((3, 6), dtype=torch.int8), torch.empty(3)
    i = torch.zeros((2, 4), dtype=torch.int32)
    states = archead.archead_beam_states([archead.archead_beam_state(torch.empty((8, 5)))])
    for bad in (lambda: archead.archead_int8_linear(w, x, 3, y), lambda: archead.archead_int8_matmul(w, c, s, 3, y),
                lambda: archead.archead_int8_quantize_tokens(x, c, s),
                lambda: archead.archead_beam_select(beam, torch.empty((8, 9)), torch.empty((2, 4)), torch.empty((2, 4)),
                                                    i, i),
                lambda: archead.archead_beam_reorder(states, i)):
        with pytest.raises(ValueError, match="GPU"):
            bad()
