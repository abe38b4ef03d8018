"""Beam selection and reordering against plain implementations in 64 bits.

Selection: parents and tokens are equal to those of the definition wherever
the values of different beams are further apart than the kernels' rounding
(asserted of the inputs), in one beam always (its order is that of the
logits).  Values: the sum of exponentials of fewer than 2^18 terms, in partial
sums of at most 2^11 terms in turn, is within 2^-12 of its size in the worst
case, and three more roundings are 2^-24 of at most 128 each: 3e-4 in all.
Reordering moves bytes: equal."""

import numpy as np
import pytest

from paper_2608_02703_gb300 import archead

pytestmark = pytest.mark.gpu

VALUE = 3e-4
GAP = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _build():
    from paper_2608_02703_gb300.build import build

    build()


def _torch():
    import torch

    return torch


def _dtype(name):
    torch = _torch()
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def _definition(logits, scores, ended, end, n):
    """(scores, parents, tokens) in 64 bits, and the least distance of values of different beams among the n + 1 best."""
    batch, beams = scores.shape
    V = logits.shape[1]
    out = np.full((batch, n), -np.inf), np.full((batch, n), -1), np.full((batch, n), -1)
    gap = np.inf
    for b in range(batch):
        cands = []
        for k in range(beams):
            score = float(scores[b, k])
            if not np.isfinite(score):
                continue
            if ended is not None and ended[b, k]:
                cands.append((-score, k, 0, end))
                continue
            row = logits[b * beams + k].astype(np.float64)
            if np.isnan(row).any() or row.max() == np.inf or row.max() == -np.inf:
                continue
            lse = row.max() + np.log(np.exp(row - row.max()).sum())
            best = np.lexsort((np.arange(V), -(row + 0.0)))[:n + 1]
            for i, v in enumerate(best):
                if row[v] > -np.inf:
                    cands.append((-(score - lse + row[v]), k, i, int(v)))
        cands.sort()
        for i, c in enumerate(cands[:n]):
            out[0][b, i], out[1][b, i], out[2][b, i] = -c[0], c[1], c[3]
        for c, d in zip(cands[:n], cands[1:n + 1]):
            if c[1] != d[1]:
                gap = min(gap, d[0] - c[0])
    return out, gap


def _select(logits, scores, n, ended=None, end=0, beam=None, **kw):
    torch = _torch()
    batch, beams = scores.shape
    own = beam is None
    if own:
        beam = archead.archead_beam_create(batch * beams, logits.shape[1], n)
    o = torch.full((batch, n), float("nan"), device="cuda")
    p = torch.full((batch, n), -7, dtype=torch.int32, device="cuda")
    t = torch.full((batch, n), -7, dtype=torch.int32, device="cuda")
    archead.archead_beam_select(beam, logits, scores, o, p, t, ended=ended, end_token=end, **kw)
    torch.cuda.synchronize()
    if own:
        beam.close()
    return o.cpu().numpy(), p.cpu().numpy(), t.cpu().numpy()


def _compare(got, want):
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[2], want[2])
    none = np.isneginf(want[0])
    np.testing.assert_array_equal(np.isneginf(got[0]), none)
    assert not np.isnan(got[0]).any()
    off = np.abs(np.where(none, 0, got[0]) - np.where(none, 0, want[0]))
    assert off.max(initial=0) <= VALUE, off.max()


def _logits(rows, V, dtype, seed, spread=3.0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, V), generator=g) * spread).to(_dtype(dtype))


SIZES = [(1, 1, 1, 1), (1, 1, 7, 3), (1, 4, 1000, 8), (2, 3, 129, 6), (3, 5, 4096, 10), (1, 4, 50001, 8),
         (2, 8, 32768, 16), (5, 2, 3000, 1), (1, 16, 2049, 32), (1, 64, 500, 64), (2, 33, 70, 64), (40, 4, 1025, 4),
         (1, 1, 151936, 64), (1, 12, 151937, 24), (9, 16, 9000, 17)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("batch,beams,V,n", SIZES, ids=str)
def test_select(dtype, batch, beams, V, n):
    torch = _torch()
    logits = _logits(batch * beams, V, dtype, seed=V + n)
    scores = -10 * torch.rand((batch, beams), generator=torch.Generator().manual_seed(n))
    want, gap = _definition(logits.float().numpy(), scores.numpy(), None, 0, n)
    assert gap > GAP
    _compare(_select(logits.cuda(), scores.cuda(), n), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("batch,beams,V,n", [(1, 4, 300, 8), (4, 6, 5000, 12), (30, 3, 700, 6)], ids=str)
def test_ended_beams_and_masked_tokens(dtype, batch, beams, V, n):
    torch = _torch()
    logits = _logits(batch * beams, V, dtype, seed=V)
    logits[:, 3::5] = -float("inf")
    g = torch.Generator().manual_seed(n)
    scores = -3 * torch.rand((batch, beams), generator=g)
    ended = (torch.rand((batch, beams), generator=g) < 0.4).to(torch.uint8)
    scores[0, 0] = -float("inf")
    scores[-1, -1] = -1.5
    ended[-1, -1] = 1
    logits[-1] = float("nan")  # (an ended beam's logits are not looked at)
    want, gap = _definition(logits.float().numpy(), scores.numpy(), ended.numpy(), 17, n)
    assert gap > GAP
    for flags in (ended, ended.bool()):
        _compare(_select(logits.cuda(), scores.cuda(), n, flags.cuda(), 17), want)


def test_rows_without_candidates():
    """Empty rows, rows that hold a NaN or +inf, dead beams; then nothing at all."""
    torch = _torch()
    inf, nan = float("inf"), float("nan")
    beams, V, n = 6, 5000, 9
    logits = _logits(2 * beams, V, "fp32", seed=4)
    logits[0] = -inf
    logits[1, 4321] = nan
    logits[2, 17] = inf
    logits[3] = -inf
    logits[3, 4999], logits[3, 2500] = 2.0, 2.0  # two candidates only
    scores = torch.linspace(-1, -2, 2 * beams).reshape(2, beams)
    scores[0, 4] = nan
    scores[0, 5] = inf
    logits[beams:beams + 5] = -inf
    logits[beams + 5] = nan
    want, gap = _definition(logits.numpy(), scores.numpy(), None, 0, n)
    assert gap > GAP and (want[1][0] == 3).sum() == 2 and (want[1][1] == -1).all()
    _compare(_select(logits.cuda(), scores.cuda(), n), want)


def test_more_places_than_candidates():
    torch = _torch()
    logits = _logits(6, 3, "bf16", seed=5)
    scores = torch.tensor([[-0.5, -1.0, -2.5], [-0.25, -3.0, -0.75]])
    ended = torch.tensor([[0, 1, 0], [1, 1, 1]], dtype=torch.uint8)
    want, gap = _definition(logits.float().numpy(), scores.numpy(), ended.numpy(), 2, 20)
    assert gap > GAP and (want[1] == -1).any()
    _compare(_select(logits.cuda(), scores.cuda(), 20, ended.cuda(), 2), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V", [5, 100, 20000])
def test_ties(dtype, V):
    """Equal beams: the lower beam first; equal logits: the lower token first; the two zeros are equal."""
    torch = _torch()
    n, beams = 12, 3
    row = torch.zeros(V)
    row[1::2] = -0.0
    logits = row.to(_dtype(dtype)).repeat(beams, 1).cuda()
    got = _select(logits, torch.full((1, beams), -2.0).cuda(), n)
    m = min(n, V)
    np.testing.assert_array_equal(got[1][0, :m], 0)
    np.testing.assert_array_equal(got[2][0, :m], np.arange(m))
    # Equal rows of few distinct values: in each beam by value and token, and of equal values beam by beam.
    row = torch.randint(0, 4, (V,), generator=torch.Generator().manual_seed(V)).float()
    got = _select(row.to(_dtype(dtype)).repeat(beams, 1).cuda(), torch.full((1, beams), -2.0).cuda(), n)
    order = np.lexsort((np.arange(V), -row.numpy()))
    want = sorted((-float(row[v]), k, v) for k in range(beams) for v in order[:n])[:n]
    np.testing.assert_array_equal(got[1][0], [w[1] for w in want])
    np.testing.assert_array_equal(got[2][0], [w[2] for w in want])


def test_values_that_round_together_keep_the_order_of_the_logits():
    """A score so large that neighbouring logits give one value: the larger logit comes first."""
    torch = _torch()
    V = 600
    row = torch.linspace(0, 1e-3, V)  # ascending: the last token is the best
    got = _select(row[None].cuda(), torch.tensor([[-1e6]]).cuda(), 5)
    np.testing.assert_array_equal(got[2][0], np.arange(V - 1, V - 6, -1))
    assert (got[0] == got[0][0, 0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("pad,start", [(0, 0), (1, 0), (3, 1), (8, 0), (8, 3), (5, 2)])
def test_rows_apart_and_out_of_line(dtype, pad, start):
    """Row distances and first addresses of every alignment; equal rows stay equal whatever their alignment."""
    torch = _torch()
    batch, beams, V, n = 2, 4, 6001, 8
    data = _logits(batch * beams, V, dtype, seed=8)
    data[1] = data[0]
    whole = torch.full((batch * beams, V + pad + start), 99.0, dtype=data.dtype, device="cuda")
    flat = torch.full((whole.numel() + 16,), 99.0, dtype=data.dtype, device="cuda")
    view = flat[start:start + batch * beams * (V + pad)].view(batch * beams, V + pad)[:, :V]
    view.copy_(data)
    scores = -3 * torch.rand((batch, beams), generator=torch.Generator().manual_seed(1))
    scores[0, 1] = scores[0, 0]
    want, gap = _definition(data.float().numpy(), scores.numpy(), None, 0, n)
    _compare(_select(view, scores.cuda(), n), want)
    assert gap > GAP or gap == 0


def test_large_values():
    """Logits and scores so large that their rounding shows: score - lse and the value are rounded at up to 1.5e5
    (half a unit in the last place: 2^-7 each), the lse at up to 4.5e4 (2^-9)."""
    torch = _torch()
    logits = _logits(4, 3000, "fp32", seed=3, spread=1e4)
    scores = torch.tensor([[-1e5, -2e5], [-1.0, -2.0]])
    want, gap = _definition(logits.numpy(), scores.numpy(), None, 0, 6)
    got = _select(logits.cuda(), scores.cuda(), 6)
    off = 2.0 ** -6 + 2.0 ** -8
    assert gap > 2 * off
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[2], want[2])
    assert np.abs(got[0] - want[0]).max() <= off
    low = torch.finfo(torch.float32).min
    logits = torch.full((1, 3000), low)
    logits[0, 40] = 0.0  # masked with the type's lowest value instead of -inf
    got = _select(logits.cuda(), torch.tensor([[-1.0]]).cuda(), 3)
    assert got[2][0, 0] == 40 and abs(got[0][0, 0] + 1) < 1e-6
    logits[0, 40] = low  # nothing else: a uniform row
    got = _select(logits.cuda(), torch.tensor([[-1.0]]).cuda(), 3)
    np.testing.assert_array_equal(got[2][0], [0, 1, 2])


def test_handle_serves_smaller_calls_and_streams():
    torch = _torch()
    beam = archead.archead_beam_create(64, 20000, 16)
    side = torch.cuda.Stream()
    for i, (batch, beams, V, n) in enumerate([(1, 4, 20000, 8), (16, 4, 300, 4), (2, 2, 20000, 16), (8, 8, 1999, 16),
                                               (1, 1, 1, 1)]):
        logits = _logits(batch * beams, V, "bf16", seed=i)
        scores = -torch.rand((batch, beams), generator=torch.Generator().manual_seed(i))
        want, gap = _definition(logits.float().numpy(), scores.numpy(), None, 0, n)
        assert gap > GAP
        a, b = logits.cuda(), scores.cuda()
        torch.cuda.synchronize()
        _compare(_select(a, b, n, beam=beam, stream=side if i % 2 else None), want)
    for batch, beams, V, n in [(17, 4, 10, 2), (1, 1, 20001, 2), (1, 1, 10, 17)]:
        with pytest.raises(archead.ArcheadError) as e:
            _select(_logits(batch * beams, V, "bf16", 0).cuda(), torch.zeros((batch, beams)).cuda(), n, beam=beam)
        assert e.value.status == archead.ERR_UNSUPPORTED
    beam.close()


def test_many_rows():
    """More rows than a grid's second dimension takes."""
    torch = _torch()
    batch, beams, V, n = 35000, 2, 20, 2
    logits = _logits(batch * beams, V, "fp32", seed=1)
    scores = -torch.rand((batch, beams), generator=torch.Generator().manual_seed(1))
    got = _select(logits.cuda(), scores.cuda(), n)
    value = (scores.double().reshape(-1, 1) + torch.log_softmax(logits.double(), dim=1)).reshape(batch, -1)
    top = value.topk(n + 1, dim=1)
    clear = (top.values[:, :-1] - top.values[:, 1:] > GAP).all(dim=1).numpy()
    assert clear.mean() > 0.99
    np.testing.assert_array_equal(got[1][clear], (top.indices[:, :n] // V).numpy()[clear])
    np.testing.assert_array_equal(got[2][clear], (top.indices[:, :n] % V).numpy()[clear])
    assert np.abs(got[0] - top.values[:, :n].numpy()).max() <= VALUE


def test_select_in_a_graph_and_again():
    torch = _torch()
    logits = _logits(8, 30000, "bf16", seed=2).cuda()
    scores = -torch.rand((2, 4), generator=torch.Generator().manual_seed(2)).cuda()
    first = _select(logits, scores, 8)
    beam = archead.archead_beam_create(8, 30000, 8)
    o = torch.empty((2, 8), device="cuda")
    p, t = torch.empty((2, 8), dtype=torch.int32, device="cuda"), torch.empty((2, 8), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        archead.archead_beam_select(beam, logits, scores, o, p, t)
    for _ in range(3):
        o.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((o, p, t), first):
            np.testing.assert_array_equal(a.cpu().numpy(), b)
    beam.close()


# ------------------------------------------------------------------------
# Reordering
# ------------------------------------------------------------------------
def _reordered(src, parents, index, out=None):
    """The definition on a CPU copy whose first dimension is the rows: their contents at `index`."""
    batch, beams = parents.shape
    new = (src if out is None else out).clone()
    for b in range(batch):
        for k in range(beams):
            q = int(parents[b, k])
            got = src[b * beams + q] if 0 <= q < beams else None
            new[b * beams + k][index] = got[index] if got is not None else 0
    return new


def _parents(kind, batch, beams, seed=0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(0, beams, (batch, beams), generator=g)
    if kind == "same":
        p[:] = torch.arange(beams)
    elif kind == "cycle":
        p[:] = (torch.arange(beams) + 1) % beams
    elif kind == "swap":
        p[:] = torch.arange(beams).flip(0)
    elif kind == "one":
        p[:] = beams - 1
    elif kind == "none":
        p[0, 0], p[-1, -1] = -1, beams
        p[0, beams // 2] = 1 << 30
    return p.to(torch.int32)


def _any(shape, dtype, seed):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    return torch.randint(0, 256, (n,), generator=g, dtype=torch.uint8).view(dtype).reshape(shape)


@pytest.mark.parametrize("place", [True, False], ids=["in_place", "out"])
@pytest.mark.parametrize("kind", ["random", "same", "cycle", "swap", "one", "none"])
@pytest.mark.parametrize("batch,beams", [(1, 1), (1, 4), (3, 5), (2, 8), (1, 16), (2, 17), (1, 33), (1, 64)], ids=str)
def test_reorder(batch, beams, kind, place):
    torch = _torch()
    rows = batch * beams
    parents = _parents(kind, batch, beams)
    cache = _any((2, rows, 3, 11, 24), torch.int16, 1)   # layer, row, head, position, element
    history = _any((rows, 37), torch.int32, 2)
    state = _any((rows, 5, 7), torch.uint8, 3)
    length = 9
    given = [t.cuda() for t in (cache, history, state)]
    outs = [None] * 3 if place else [torch.full_like(t, 5) for t in given]
    states = archead.archead_beam_states([
        archead.archead_beam_state(given[0], row_dim=1, length_dim=3, out=outs[0]),
        archead.archead_beam_state(given[1], length_dim=1, out=outs[1]), archead.archead_beam_state(given[2], out=outs[2])])
    archead.archead_beam_reorder(states, parents.cuda(), length)
    fill = [None] * 3 if place else [torch.full_like(t, 5) for t in (cache, history, state)]
    layers = [_reordered(cache[i], parents, (slice(None), slice(0, length)), None if place else fill[0][i])
              for i in range(2)]
    want = [torch.stack(layers), _reordered(history, parents, slice(0, length), fill[1]),
            _reordered(state, parents, ..., fill[2])]
    for got, w, src, before in zip(given if place else outs, want, given, (cache, history, state)):
        assert torch.equal(got.cpu(), w)
        if not place:
            assert torch.equal(src.cpu(), before)


@pytest.mark.parametrize("start,size,pad", [(0, 1, 0), (1, 1, 2), (3, 5, 1), (2, 6, 4), (4, 12, 0), (8, 24, 8),
                                            (16, 48, 16), (16, 4096, 16), (7, 1000, 1), (0, 70000, 3)])
def test_reorder_alignments(start, size, pad):
    """Chunks of any size, address and distance; what lies between and around them is not touched."""
    torch = _torch()
    batch, beams = 2, 4
    buf = _any((64 + batch * beams * (size + pad),), torch.uint8, 5)
    dev = buf.cuda()
    view = lambda t: t[start:start + batch * beams * (size + pad)].view(batch * beams, size + pad)[:, :size]  # noqa: E731
    parents = _parents("random", batch, beams, seed=size)
    archead.archead_beam_reorder(archead.archead_beam_states([archead.archead_beam_state(view(dev), length_dim=1)]),
                                 parents.cuda(), size)
    want = buf.clone()
    view(want).copy_(_reordered(view(buf), parents, ...))
    assert torch.equal(dev.cpu(), want)


def test_reorder_many_states_and_lengths():
    """More states than one launch takes, in place and not, some without positions; no positions; one position."""
    torch = _torch()
    batch, beams = 2, 3
    parents = _parents("random", batch, beams, seed=3)
    for length in (0, 1, 4):
        cpu = [_any((batch * beams, 4 + i % 3, 6), torch.int16, i) for i in range(110)]
        dev = [t.cuda() for t in cpu]
        outs = [torch.zeros_like(t) if i % 7 == 3 else None for i, t in enumerate(dev)]
        states = [archead.archead_beam_state(t, length_dim=1 if i % 5 else None, out=o)
                  for i, (t, o) in enumerate(zip(dev, outs))]
        archead.archead_beam_reorder(archead.archead_beam_states(states), parents.cuda(), length)
        for i, (t, c, o) in enumerate(zip(dev, cpu, outs)):
            index = slice(0, length) if i % 5 else ...
            want = _reordered(c, parents, index, None if o is None else torch.zeros_like(c))
            assert torch.equal((t if o is None else o).cpu(), want), i
    archead.archead_beam_reorder(archead.archead_beam_states([]), parents.cuda(), 3)


def test_reorder_other_orders():
    """Rows in the middle or last but one; heads before the rows; a slice of the heads."""
    torch = _torch()
    batch, beams = 1, 4
    parents = _parents("swap", batch, beams)
    a = _any((9, 4, 16), torch.int16, 1)           # position, row, element: every position is a chunk
    b = _any((4, 6, 10, 8), torch.int32, 2)
    da, db = a.cuda(), b.cuda()
    states = archead.archead_beam_states([
        archead.archead_beam_state(da[:7], row_dim=1),
        archead.archead_beam_state(db[:, 1:4], length_dim=2)])
    archead.archead_beam_reorder(states, parents.cuda(), 5)
    want = a.clone()
    want[:7] = a[:7][:, parents[0].long()]
    assert torch.equal(da.cpu(), want)
    want = b.clone()
    want[:, 1:4, :5] = b[parents[0].long()][:, 1:4, :5]
    assert torch.equal(db.cpu(), want)


def test_reorder_far_apart():
    """Rows whose offsets pass 32 bits."""
    torch = _torch()
    beams, far = 3, (1 << 32) + 4096
    buf = torch.zeros(far * 2 + 4096, dtype=torch.uint8, device="cuda")
    view = torch.as_strided(buf, (beams, 4096), (far, 1))
    cpu = _any((beams, 4096), torch.uint8, 1)
    view.copy_(cpu)
    parents = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    archead.archead_beam_reorder(archead.archead_beam_states([archead.archead_beam_state(view)]), parents.cuda())
    assert torch.equal(view.cpu(), cpu[parents[0].long()])


def test_reorder_on_a_stream_and_in_a_graph():
    torch = _torch()
    cpu = _any((8, 2, 300, 64), torch.int16, 1)
    dev = cpu.cuda()
    parents = _parents("random", 2, 4, seed=1)
    on = parents.cuda()
    states = archead.archead_beam_states([archead.archead_beam_state(dev, length_dim=2)])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    archead.archead_beam_reorder(states, on, 300, stream=side)
    side.synchronize()
    want = _reordered(cpu, parents, ...)
    assert torch.equal(dev.cpu(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        archead.archead_beam_reorder(states, on, 300)
    parents = _parents("cycle", 2, 4)
    on.copy_(parents)
    graph.replay()
    assert torch.equal(dev.cpu(), _reordered(want, parents, ...))


@pytest.mark.parametrize("start", [0, 1])
def test_reorder_more_vectors_than_31_bits(start):
    """Rows of 2^31 + some single bytes (nothing is aligned): they are moved in parts."""
    torch = _torch()
    n, beams = (1 << 31) + 4097, 2
    buf = torch.empty(beams * n + 16, dtype=torch.uint8, device="cuda")
    view = buf[start:start + beams * n].view(beams, n)
    for k in range(beams):
        view[k] = 0
        view[k, ::9973] = k + 1
        view[k, -1] = 100 + k
    want = [(int((view[k] == k + 1).sum()), 100 + k) for k in range(beams)]
    parents = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    archead.archead_beam_reorder(archead.archead_beam_states([archead.archead_beam_state(view)]), parents)
    for k in range(beams):
        assert (int((view[k] == 2 - k).sum()), int(view[k, -1])) == want[1 - k]
        assert bool((view[k, ::9973][:-1] == 2 - k).all())
