"""The beam-search example against a plain search that takes the same logits: every step's choice, state and history."""

import importlib.util
import os

import pytest

from paper_2608_02703_gb300 import archead
from synth import HeadShape, make_head

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2608_02703_gb300.build import build

    build()
    spec = importlib.util.spec_from_file_location("beam_search_example", os.path.join(ROOT, "examples", "beam_search.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _plain(example, head, embedding, first, beams, steps, end):
    """The same search with lists and 64-bit sums; returns the tokens, the scores and the least distance of a choice."""
    import torch

    batch, rows = first.numel(), first.numel() * beams
    decoder = example.Decoder(embedding, rows)
    logits = torch.empty((rows, head.vocab), device="cuda")
    history = [[[] for _ in range(beams)] for _ in range(batch)]
    scores = torch.full((batch, beams), -float("inf"), dtype=torch.float64)
    scores[:, 0] = 0
    ended = [[False] * beams for _ in range(batch)]
    tokens = first.to(torch.int32)[:, None].expand(batch, beams).contiguous()
    gap = float("inf")
    for _ in range(steps):
        decoder.step(tokens)
        head.logits(decoder.h, logits)
        logp = torch.log_softmax(logits.double(), dim=1).cpu().view(batch, beams, -1)
        h = decoder.h.clone().view(batch, beams, -1)
        new_tokens = tokens.clone()
        for b in range(batch):
            found = []
            for k in range(beams):
                if scores[b, k] == -float("inf"):
                    continue
                if ended[b][k]:
                    found.append((-float(scores[b, k]), k, end))
                else:
                    top = torch.topk(logp[b, k], beams + 1)
                    found += [(-float(scores[b, k] + v), k, int(t)) for v, t in zip(top.values, top.indices)]
            found.sort()
            gap = min([gap] + [y[0] - x[0] for x, y in zip(found[:beams], found[1:])])
            old_history, old_ended = history[b], ended[b]
            history[b] = [old_history[k] + [t] for _, k, t in found[:beams]]
            ended[b] = [old_ended[k] or t == end for _, k, t in found[:beams]]
            for i, (v, k, t) in enumerate(found[:beams]):
                scores[b, i] = -v
                decoder.h.view(batch, beams, -1)[b, i] = h[b, k]
                new_tokens[b, i] = t
        tokens = new_tokens
    return torch.tensor(history), scores, gap


@pytest.mark.parametrize("kind", ["packed", "int8"])
@pytest.mark.parametrize("beams,end", [(1, 0), (3, 0), (4, 7), (8, 0)])
def test_search_equals_plain_search(example, kind, beams, end):
    import torch

    shape = HeadShape(V=1500, d=256, core_rank=16, corr_rank=8, group_size=64)
    first, steps = torch.tensor([3, 100], device="cuda"), 9
    for seed in range(40):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        embedding = torch.randn((shape.V, shape.d), generator=gen, device="cuda").to(torch.bfloat16)
        if kind == "packed":
            head = example.PackedHead(archead.archead_pack_create(make_head(shape, seed=3), shape))
        else:
            head = example.RowInt8Head(torch.randn((shape.V, shape.d), generator=gen, device="cuda") * 0.1)
        want, want_scores, gap = _plain(example, head, embedding, first, beams, steps, end)
        # Sums of 1500 terms, nine rounded sums of at most 128: far below 1e-4.  The first inputs on which the plain
        # search never has to choose between candidates as near as that.
        if gap > 1e-4:
            break
    assert gap > 1e-4
    tokens, scores = example.search(head, embedding, first, beams, steps, end)
    assert torch.equal(tokens.cpu().long(), want)
    assert float((scores.cpu().double() - want_scores).abs().max()) < 1e-4


def test_example_runs(example, capsys):
    example.main()
    out = capsys.readouterr().out
    assert "packed head" in out and "Row-INT8 head" in out and out.count("score") == 6
