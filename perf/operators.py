"""The operators of a beam-search step on an INT8 head, as measurable cases.

One step of beam search holds the hidden states of batch x beams rows.  They
are quantised to 8-bit integers with a scale for each token, multiplied with a
weight matrix in 8-bit integers with a scale for each output channel (the
"Row INT8" head that the packed head is compared with, or a projection before
it), the next beams are selected over beams x vocabulary, and the decoder's
states follow their parents.

  linear    y = dequantised(quantised(x)) W^T from activations
  matmul    the same from codes and scales
  quantize  codes and scales of activations
  select    the n best (beam, token) candidates of each batch entry
  reorder   rows of caches and token histories follow their parent beams
"""

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def _product(op, M, N, K, x="bf16", out="bf16"):
    return dict(op=op, M=M, N=N, K=K, x=x, out=out)


def _quantize(M, K, x="bf16"):
    return dict(op="quantize", M=M, K=K, x=x)


def _select(batch, beams, V, n, x="bf16", ended=0, banned=0):
    """ended: beams of each batch entry that have finished; banned: tokens with logit -inf in every row."""
    return dict(op="select", batch=batch, beams=beams, V=V, n=n, x=x, ended=ended, banned=banned)


def _reorder(batch, beams, layers, heads, dim, length, room, keep, place=True):
    """Key and value caches [rows][heads][room][dim] of each layer with `length` positions in use, and the token
    history [rows][room]; keep: beams of each batch entry that stay where they are (0: all move in a cycle)."""
    return dict(op="reorder", batch=batch, beams=beams, layers=layers, heads=heads, dim=dim, length=length, room=room,
                keep=keep, place=place)


def listed():
    named = [
        # One token on the package's tiny head: launches and latency only.
        ("linear, 1 token, tiny head", _product("linear", 1, 4096, 512)),
        # One user's eight beams on the Row-INT8 form of the Qwen3-8B-shaped head: the weights are streamed once.
        ("linear, 8 beams, wide head", _product("linear", 8, 151936, 4096)),
        # A projection of sizes that divide by nothing, for a batch of beams, from codes.
        ("matmul, 100 tokens, odd sizes", _product("matmul", 100, 10007, 2501, out="fp16")),
        # A prompt chunk through a square projection at the Qwen3-8B width.
        ("linear, 512 tokens, projection", _product("linear", 512, 4096, 4096)),
        # Scoring a window of text on the Row-INT8 head: all logits (the largest product).
        ("matmul, 2048 tokens, wide head", _product("matmul", 2048, 151936, 4096)),
        # Activations of one user's beams.
        ("quantize 8 tokens", _quantize(8, 4096)),
        # Activations of a prompt, from an fp32 residual stream of the Gemma-shaped width.
        ("quantize 4096 tokens", _quantize(4096, 2560, x="fp32")),
        # One user with four beams, two candidates for each of them.
        ("select, 4 beams", _select(1, 4, 151936, 8)),
        # A serving batch whose sampler takes fp32 logits.
        ("select, 16 x 8 beams, fp32", _select(16, 8, 151936, 16, x="fp32")),
        # A batch near its end: ended beams, banned tokens, wide vocabulary.
        ("select, 32 x 5 beams, some ended", _select(32, 5, 262144, 10, ended=2, banned=100)),
        # One user's short history: small states, latency.
        ("reorder, 4 beams, short", _reorder(1, 4, 4, 8, 64, 131, 160, 1)),
        # A batch with long caches, in place: two of four beams die in a step.
        ("reorder, 8 x 4 beams, long", _reorder(8, 4, 8, 8, 128, 3001, 4096, 2)),
    ]
    return [dict(c, name=n) for n, c in named]


def draw(rng):
    """One more case: sizes spread over the ranges that the listed cases stand for."""

    def log_int(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v + 1 if v == 3072 else v

    op = rng.choice(["linear", "linear", "matmul", "matmul", "quantize", "select", "select", "reorder"])
    if op in ("linear", "matmul"):
        M, N, K = log_int(1, 2048), log_int(64, 151936), log_int(33, 8192)
        if rng.random() < 0.5:  # widths of models are mostly multiples of 64
            K = max(64, K // 64 * 64)
            K += 64 if K == 3072 else 0
        while M > 1 and M * N * K > 2048 * 151936 * 4096:
            M = M // 2
        return _product(op, M, N, K, x=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                        out=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if op == "quantize":
        M, K = log_int(1, 8192), log_int(20, 16384)
        while M * K > 4096 * 2560:
            M = max(1, M // 2)
        return _quantize(M, K, x=rng.choice(["bf16", "fp16", "fp32"]))
    if op == "select":
        beams, V, x = rng.randint(1, 16), log_int(200, 262144), rng.choice(["bf16", "bf16", "fp16", "fp32"])
        batch = log_int(1, 64)
        while batch > 1 and batch * beams * V * _BYTES[x] > 16 * 8 * 151936 * 4:
            batch //= 2
        return _select(batch, beams, V, rng.randint(beams, 2 * beams), x=x, ended=rng.randint(0, beams // 2),
                       banned=rng.choice([0, 0, 30]))
    beams, heads, dim = rng.randint(2, 12), rng.choice([1, 2, 4, 8]), rng.choice([40, 64, 80, 128])
    batch, layers, length = log_int(1, 16), rng.randint(1, 12), log_int(2, 4000)
    while batch * beams * layers * heads * dim * length > 8 * 4 * 8 * 8 * 128 * 3001:
        batch, length = max(1, batch // 2), max(2, length // 2)
    return _reorder(batch, beams, layers, heads, dim, length, length + rng.randint(0, 100), rng.randint(0, beams - 1),
                    place=rng.random() < 0.7)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _hidden(gen, M, K, dtype):
    """Activations: channels of different size, a few outliers among them."""
    size = torch.exp2(torch.rand(K, generator=gen, device="cuda") * 4 - 3)
    size[torch.randint(0, K, (4,), generator=gen, device="cuda")] *= 20
    return (torch.randn((M, K), generator=gen, device="cuda") * size).to(dtype)


def _weight(gen, N, K):
    """Codes of normally distributed rows whose largest value lies near four deviations, and the rows' scales."""
    codes = torch.empty((N, K), dtype=torch.int8, device="cuda")
    rows = max(1, (1 << 28) // K)
    for n in range(0, N, rows):
        part = torch.randn((min(rows, N - n), K), generator=gen, device="cuda")
        codes[n:n + rows] = (part * 32).round_().clamp_(-127, 127).to(torch.int8)
    scales = torch.exp2(torch.rand(N, generator=gen, device="cuda") - 0.5) * (0.6 / math.sqrt(K) / 32)
    return codes, scales


def _parents(gen, case):
    """int32 [batch][beams]: `keep` beams of each entry stay, the others follow them in turn."""
    batch, beams, keep = case["batch"], case["beams"], case["keep"]
    order = torch.rand((batch, beams), generator=gen, device="cuda").argsort(dim=1)  # places, in random order
    if keep == 0:
        source = torch.roll(order, 1, dims=1)
    else:
        source = order[:, torch.arange(beams, device="cuda") % keep]
    return torch.empty_like(order).scatter_(1, order, source).to(torch.int32)


def prepare(case, seed):
    gen = _gen(seed)
    s = dict(case=case)
    op = case["op"]
    if own:
        from paper_2608_02703_gb300 import archead

        s["archead"] = archead
    if op in ("linear", "matmul"):
        M, N, K = case["M"], case["N"], case["K"]
        codes, scales = _weight(gen, N, K)
        x = _hidden(gen, M, K, _DTYPES[case["x"]])
        s["y"] = torch.empty((M, N), dtype=_DTYPES[case["out"]], device="cuda")
        if op == "linear":
            s["x"] = x
        else:
            s["codes"], s["scales"] = _plain_quantize(x)
        if own:
            s["weight"] = s["archead"].archead_int8_weight_create(codes, scales)
        else:
            s["w_codes"], s["w_scales"] = codes, scales
    elif op == "quantize":
        s["x"] = _hidden(gen, case["M"], case["K"], _DTYPES[case["x"]])
        s["codes"] = torch.empty((case["M"], case["K"]), dtype=torch.int8, device="cuda")
        s["scales"] = torch.empty(case["M"], dtype=torch.float32, device="cuda")
    elif op == "select":
        batch, beams, V, n = case["batch"], case["beams"], case["V"], case["n"]
        rows = batch * beams
        # A language model's logits: a wide floor and, in each row, a few tens of likely tokens.
        logits = 2 * torch.randn((rows, V), generator=gen, device="cuda")
        likely = torch.randint(0, V, (rows, 48), generator=gen, device="cuda")
        logits.scatter_add_(1, likely, 4 + 10 * torch.rand((rows, 48), generator=gen, device="cuda"))
        if case["banned"]:
            logits[:, torch.randint(0, V, (case["banned"],), generator=gen, device="cuda")] = -math.inf
        s["logits"] = logits.to(_DTYPES[case["x"]])
        s["scores"] = -20 * torch.rand((batch, beams), generator=gen, device="cuda")
        first = torch.rand((batch, beams), generator=gen, device="cuda").argsort(dim=1)
        s["ended"] = (first < case["ended"]).to(torch.uint8)
        s["end"] = min(2, V - 1)
        s["out_scores"] = torch.empty((batch, n), dtype=torch.float32, device="cuda")
        s["out_parents"] = torch.empty((batch, n), dtype=torch.int32, device="cuda")
        s["out_tokens"] = torch.empty((batch, n), dtype=torch.int32, device="cuda")
        if own:
            s["beam"] = s["archead"].archead_beam_create(rows, V, n)
    else:
        rows, room = case["batch"] * case["beams"], case["room"]
        shape = (rows, case["heads"], room, case["dim"])
        s["caches"] = [torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
                       for _ in range(2 * case["layers"])]
        s["history"] = torch.randint(0, 151936, (rows, room), generator=gen, device="cuda", dtype=torch.int32)
        s["parents"] = _parents(gen, case)
        if not case["place"]:
            s["new_caches"] = [torch.zeros_like(c) for c in s["caches"]]
            s["new_history"] = torch.zeros_like(s["history"])
        if own:
            new_caches = s.get("new_caches", [None] * len(s["caches"]))
            states = [s["archead"].archead_beam_state(old, length_dim=2, out=new)
                      for new, old in zip(new_caches, s["caches"])]
            states.append(s["archead"].archead_beam_state(s["history"], length_dim=1, out=s.get("new_history")))
            s["states"] = s["archead"].archead_beam_states(states)
    return s


def _plain_quantize(x):
    x = x.float()
    top = x.abs().amax(dim=1)
    scales = top / torch.full_like(top, 127)  # (by a Python number: a product with its rounded reciprocal on the GPU)
    usable = (scales > 0) & torch.isfinite(scales)
    q = torch.round(x / torch.where(usable, scales, 1)[:, None]).clamp(-127, 127)
    return torch.where(usable[:, None], q, 0).to(torch.int8), scales


def _plain_product(codes, scales, w_codes, w_scales, dtype):
    return ((codes.float() @ w_codes.float().t()) * scales[:, None] * w_scales[None, :]).to(dtype)


def _plain_select(logits, scores, ended, end, n):
    batch, beams = scores.shape
    V = logits.shape[1]
    x = logits.float() + 0.0  # (one zero)
    top = x.amax(dim=1)
    has = torch.isfinite(top)
    lse = top + torch.log(torch.exp(x - top[:, None]).sum(dim=1))
    # Order of the logits, then of the tokens, as one integer.
    bits = x.view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)
    key = (order << 20) + ((1 << 20) - 1 - torch.arange(V, device=x.device))
    m = min(n, V)
    key = torch.topk(key, m, dim=1).values
    tokens = (1 << 20) - 1 - (key & ((1 << 20) - 1))
    values = (scores.reshape(-1) - lse)[:, None] + x.gather(1, tokens)
    values = torch.where(has[:, None] & torch.isfinite(values), values, -math.inf)
    # An ended beam has one candidate.
    done = ended.reshape(-1, 1).bool()
    one = torch.full_like(values, -math.inf)
    one[:, 0] = torch.where(torch.isfinite(scores.reshape(-1)), scores.reshape(-1), -math.inf)
    values = torch.where(done, one, values).reshape(batch, beams * m)
    tokens = torch.where(done, end, tokens).reshape(batch, beams * m)
    values, at = torch.sort(values, dim=1, descending=True, stable=True)
    if beams * m < n:
        values = torch.nn.functional.pad(values, (0, n - beams * m), value=-math.inf)
        at = torch.nn.functional.pad(at, (0, n - at.shape[1]))
    values, at = values[:, :n], at[:, :n]
    none = values == -math.inf
    return (values, torch.where(none, -1, at // m).to(torch.int32),
            torch.where(none, -1, tokens.gather(1, at)).to(torch.int32))


def run(state):
    case = state["case"]
    return _own(state, case) if own else _plain(state, case)


def _plain(s, case):
    op = case["op"]
    if op in ("linear", "matmul"):
        codes, scales = _plain_quantize(s["x"]) if op == "linear" else (s["codes"], s["scales"])
        return _plain_product(codes, scales, s["w_codes"], s["w_scales"], _DTYPES[case["out"]])
    if op == "quantize":
        codes, scales = _plain_quantize(s["x"])
        return {"codes": codes, "scales": scales}
    if op == "select":
        scores, parents, tokens = _plain_select(s["logits"], s["scores"], s["ended"], s["end"], case["n"])
        return {"scores": scores, "parents": parents, "tokens": tokens}
    batch, beams, length = case["batch"], case["beams"], case["length"]
    source = (torch.arange(batch, device="cuda")[:, None] * beams + s["parents"]).reshape(-1)
    caches = s["caches"] if case["place"] else s["new_caches"]
    history = s["history"] if case["place"] else s["new_history"]
    for new, old in zip(caches, s["caches"]):
        new[:, :, :length] = old[source, :, :length]
    history[:, :length] = s["history"][source, :length]
    return {"caches": caches, "history": history}


def _own(s, case):
    op, lib = case["op"], s["archead"]
    if op == "linear":
        lib.archead_int8_linear(s["weight"], s["x"], case["M"], s["y"])
        return s["y"]
    if op == "matmul":
        lib.archead_int8_matmul(s["weight"], s["codes"], s["scales"], case["M"], s["y"])
        return s["y"]
    if op == "quantize":
        lib.archead_int8_quantize_tokens(s["x"], s["codes"], s["scales"])
        return {"codes": s["codes"], "scales": s["scales"]}
    if op == "select":
        lib.archead_beam_select(s["beam"], s["logits"], s["scores"], s["out_scores"], s["out_parents"],
                                s["out_tokens"], ended=s["ended"], end_token=s["end"])
        return {"scores": s["out_scores"], "parents": s["out_parents"], "tokens": s["out_tokens"]}
    lib.archead_beam_reorder(s["states"], s["parents"], case["length"])
    if case["place"]:
        return {"caches": s["caches"], "history": s["history"]}
    return {"caches": s["new_caches"], "history": s["new_history"]}


def work(case):
    op = case["op"]
    if op in ("linear", "matmul"):
        M, N, K = case["M"], case["N"], case["K"]
        inputs = M * K * _BYTES[case["x"]] if op == "linear" else M * K + 4 * M
        return {"bytes": N * K + 4 * N + inputs + M * N * _BYTES[case["out"]], "flops": 2 * M * N * K}
    if op == "quantize":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (_BYTES[case["x"]] + 1) + 4 * M, "flops": 3 * M * K}
    if op == "select":
        live = case["batch"] * (case["beams"] - case["ended"])
        small = case["batch"] * (5 * case["beams"] + 12 * case["n"])
        return {"bytes": live * case["V"] * _BYTES[case["x"]] + small, "flops": 4 * live * case["V"]}
    # Rows that stay are neither read nor written in place; a row that several beams take is read once.
    beams, keep = case["beams"], case["keep"]
    moved = beams - keep if case["place"] else beams
    read = beams if keep == 0 else min(keep, moved)
    row = case["length"] * (2 * case["layers"] * case["heads"] * case["dim"] * 2 + 4)
    return {"bytes": case["batch"] * ((moved + read) * row + 4 * beams), "flops": 0}


def exact(case, seed):
    """run()'s answer from the definitions in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("linear", "matmul"):
        if op == "linear":
            x = s["x"].double()
            scales = (x.abs().max(dim=1).values / 127).float().double()
            codes = torch.round(x / scales.clamp_min(1e-300)[:, None]).clamp_(-127, 127)
        else:
            codes, scales = s["codes"].double(), s["scales"].double()
        y = torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
        for n in range(0, case["N"], 16384):
            part = slice(n, n + 16384)
            y[:, part] = codes @ s["w_codes"][part].double().t()
            y[:, part] *= s["w_scales"][part].double()
        return y * scales[:, None]
    if op == "quantize":
        return {"codes": None, "scales": s["x"].double().abs().max(dim=1).values / 127}
    if op == "select":
        batch, beams = case["batch"], case["beams"]
        best = []
        for b in range(batch):
            values = []
            for k in range(beams):
                score = s["scores"][b, k].double()
                if s["ended"][b, k]:
                    values.append(score[None])
                else:
                    row = s["logits"][b * beams + k].double()
                    values.append(torch.topk(score + torch.log_softmax(row, dim=0), min(case["n"], case["V"])).values)
            values = torch.cat(values).sort(descending=True).values[:case["n"]]
            best.append(torch.nn.functional.pad(values, (0, case["n"] - values.numel()), value=-math.inf))
        return {"scores": torch.stack(best), "parents": None, "tokens": None}
    # Copies: the rows themselves, one at a time.
    def rows(old, new, used):
        new = old.clone() if new is None else new.clone()
        for b in range(case["batch"]):
            for k in range(case["beams"]):
                source = b * case["beams"] + int(s["parents"][b, k])
                used(new[b * case["beams"] + k]).copy_(used(old[source]))
        return new

    length = case["length"]
    new_caches = [None] * len(s["caches"]) if case["place"] else s["new_caches"]
    return {"caches": [rows(old, new, lambda t: t[:, :length]) for old, new in zip(s["caches"], new_caches)],
            "history": rows(s["history"], None if case["place"] else s["new_history"], lambda t: t[:length])}
