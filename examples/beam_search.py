"""Beam search over an output head: the packed head or its Row-INT8 form.

A step of the search, for batch x beams rows:
  1. the decoder's hidden states give logits: archead_forward on a packed head, or archead_int8_linear on the rows'
     8-bit codes (it quantises the states itself);
  2. archead_beam_select takes the best (beam, token) candidates of each batch entry;
  3. archead_beam_reorder moves the decoder's state and the token histories to their new beams, in place.

The decoder here is a stand-in, a decaying average of token embeddings; a model's caches are reordered the same way
(length_dim names the dimension of their positions).

    python examples/beam_search.py            # builds the library if needed; needs the GPU
"""

from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2608_02703_gb300 import archead


class PackedHead:
    """Logits of a packed head (fp32)."""

    def __init__(self, pack):
        self.pack = pack
        self.vocab, self.hidden = pack.shape.V, pack.shape.d

    def logits(self, h, out):
        archead.archead_forward(self.pack, h, h.shape[0], out, archead.OUT_FP32)


class RowInt8Head:
    """Logits of a head of 8-bit rows, a scale each: made from a dense matrix with the quantiser of the tokens."""

    def __init__(self, dense):
        self.vocab, self.hidden = dense.shape
        codes = torch.empty(dense.shape, dtype=torch.int8, device=dense.device)
        scales = torch.empty(self.vocab, dtype=torch.float32, device=dense.device)
        archead.archead_int8_quantize_tokens(dense, codes, scales)
        self.weight = archead.archead_int8_weight_create(codes, scales)

    def logits(self, h, out):
        archead.archead_int8_linear(self.weight, h, h.shape[0], out)


class Decoder:
    """The stand-in: h <- decay h + embedding(token), of each row."""

    def __init__(self, embedding, rows, decay=0.7):
        self.embedding, self.decay = embedding, decay
        self.h = torch.zeros((rows, embedding.shape[1]), dtype=torch.bfloat16, device=embedding.device)

    def step(self, tokens):
        self.h.mul_(self.decay).add_(self.embedding[tokens.reshape(-1).long()])


def search(head, embedding, first, beams, steps, end_token):
    """The beams' tokens [batch, beams, steps], best first, and their scores [batch, beams].

    first: one token for each batch entry.  An ended beam keeps its score and repeats the end token."""
    batch, rows, device = first.numel(), first.numel() * beams, first.device
    decoder = Decoder(embedding, rows)
    history = torch.full((rows, steps), end_token, dtype=torch.int32, device=device)
    logits = torch.empty((rows, head.vocab), dtype=torch.float32, device=device)
    scores = torch.zeros((batch, beams), device=device)
    scores[:, 1:] = -float("inf")  # the beams start alike: only the first counts
    new_scores = torch.empty_like(scores)
    parents = torch.empty((batch, beams), dtype=torch.int32, device=device)
    tokens = first.to(torch.int32)[:, None].expand(batch, beams).contiguous()
    ended = torch.zeros((batch, beams), dtype=torch.uint8, device=device)
    selection = archead.archead_beam_create(rows, head.vocab, beams)
    states = archead.archead_beam_states([archead.archead_beam_state(decoder.h),
                                          archead.archead_beam_state(ended.view(rows, 1)),
                                          archead.archead_beam_state(history, length_dim=1)])
    for step in range(steps):
        decoder.step(tokens)
        head.logits(decoder.h, logits)
        archead.archead_beam_select(selection, logits, scores, new_scores, parents, tokens, ended=ended,
                                    end_token=end_token)
        archead.archead_beam_reorder(states, parents, step)
        scores, new_scores = new_scores, scores
        # (Where candidates ran out the token is -1: the beam is dead, its score -inf.)
        tokens.clamp_(min=0)
        history[:, step] = tokens.reshape(-1)
        ended |= (tokens == end_token).to(torch.uint8)
    return history.view(batch, beams, steps), scores


def main():
    from paper_2608_02703_gb300.build import build
    from synth import SHAPES, make_head

    build()
    torch.cuda.set_device(0)
    shape = SHAPES["tiny"]
    pack = archead.archead_pack_create(make_head(shape, seed=0), shape)
    gen = torch.Generator(device="cuda").manual_seed(0)
    embedding = torch.randn((shape.V, shape.d), generator=gen, device="cuda").to(torch.bfloat16)
    dense = torch.randn((shape.V, shape.d), generator=gen, device="cuda") * 0.2
    first = torch.tensor([5, 77, 901], device="cuda")
    for name, head in (("packed head", PackedHead(pack)), ("Row-INT8 head", RowInt8Head(dense))):
        tokens, scores = search(head, embedding, first, beams=4, steps=12, end_token=0)
        torch.cuda.synchronize()
        print(name)
        for b in range(first.numel()):
            print(f"  {int(first[b])}: score {float(scores[b, 0]):.3f}, tokens {tokens[b, 0].tolist()}")
    pack.close()


if __name__ == "__main__":
    main()
