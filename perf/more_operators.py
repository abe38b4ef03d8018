"""The end of a decoder around the head, as measurable cases: the final norm,
the loss of a dense head, and their gradients.

In front of a head the residual stream takes its last addition and is
normalised; an INT8 head wants the result as 8-bit codes with a scale for each
token, the others as rows.  A head that is to be packed is trained first, and the
packed head's perplexity is held against the dense one's: that takes the cross
entropy over the whole vocabulary without its logits, the gradients of the hidden
states and of the weight, and the way back through the norm.

  norm       sum = x + residual, y = norm(sum) * weight, and / or y in 8-bit codes with scales
  norm_grad  gradients of the norm: of its input and of its weight
  loss       cross entropy of x W^T for each token, and the log-sum-exp that its gradient takes
  step       the same and its gradients: of x and of W
"""

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_EPS = 1e-6
_IGNORED = -100


def _norm(M, d, x="bf16", residual=True, y=None, codes=True):
    """y: the type of the rows that are wanted beside the codes, or None."""
    return dict(op="norm", M=M, d=d, x=x, residual=residual, y=y, codes=codes)


def _norm_grad(M, d, x="bf16", stream=True):
    """stream: the residual stream brings a gradient of its own."""
    return dict(op="norm_grad", M=M, d=d, x=x, stream=stream)


def _loss(op, M, V, d, x="bf16", ignored=0):
    """ignored: tokens of the M that have no target (prompts, padding)."""
    return dict(op=op, M=M, V=V, d=d, x=x, ignored=ignored)


def listed():
    named = [
        # One token on the package's tiny head: launches and latency only.
        ("norm, 1 token, tiny head", _norm(1, 512)),
        # One user's eight beams in front of the Row-INT8 form of the Qwen3-8B-shaped head.
        ("norm, 8 beams", _norm(8, 4096)),
        # A prompt from an fp32 residual stream at the Gemma-shaped width: codes, and rows for a bf16 head.
        ("norm, 4096 tokens, fp32 stream", _norm(4096, 2560, x="fp32", y="bf16")),
        # Rows of a width that divides by nothing, without a residual and without codes.
        ("norm, 1000 tokens, odd width", _norm(1000, 2501, x="fp16", residual=False, y="fp16", codes=False)),
        # A short sequence of a small model in training.
        ("norm gradient, 100 tokens", _norm_grad(100, 512, x="fp32", stream=False)),
        # A training batch at the Qwen3-8B width.
        ("norm gradient, 4096 tokens", _norm_grad(4096, 4096)),
        # One token's loss on the package's tiny head: launches and latency only.
        ("loss, 1 token, tiny head", _loss("loss", 1, 4096, 512)),
        # Scoring a window of text on the dense Qwen3-8B-shaped head.
        ("loss, 2048 tokens, wide head", _loss("loss", 2048, 151936, 4096)),
        # A few tokens of the package's tiny head in training.
        ("step, 4 tokens, tiny head", _loss("step", 4, 4096, 512)),
        # Fine-tuning on answers: the prompts' tokens have no target; sizes that divide by little, in fp16.
        ("step, 700 tokens, 300 ignored", _loss("step", 700, 10007, 1000, x="fp16", ignored=300)),
        # A small batch on the Gemma-shaped dense head: the weight is read, and its gradient written.
        ("step, 64 tokens, wide head", _loss("step", 64, 262144, 2560)),
        # A training batch on the Qwen3-8B-shaped dense head (the largest).
        ("step, 4096 tokens, wide head", _loss("step", 4096, 151936, 4096)),
    ]
    return [dict(c, name=n) for n, c in named]


def draw(rng):
    """One more case: sizes spread over the ranges that the listed cases stand for."""

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm", "norm", "norm_grad", "loss", "step", "step"])
    if op in ("norm", "norm_grad"):
        M, d, x = log_int(1, 8192), log_int(20, 16384), rng.choice(["bf16", "bf16", "fp16", "fp32"])
        if rng.random() < 0.5:  # widths of models are mostly multiples of 64
            d = max(64, d // 64 * 64)
        while M * d > 4096 * 4096:
            M = max(1, M // 2)
        if op == "norm_grad":
            return _norm_grad(M, d, x=x, stream=rng.random() < 0.5)
        y, codes = rng.choice([(None, True), ("bf16", True), (x, False), ("fp32", False)])
        return _norm(M, d, x=x, residual=rng.random() < 0.7, y=y, codes=codes)
    M, V, d = log_int(1, 4096), log_int(200, 262144), log_int(64, 8192) // 8 * 8
    if rng.random() < 0.7:
        d = max(64, d // 64 * 64)
    while M > 1 and M * V * d > 4096 * 151936 * 4096:
        M //= 2
    while V * d > 262144 * 4096:
        V //= 2
    ignored = int(M * rng.choice([0, 0, 0.3, 0.6]))
    return _loss(op, M, V, d, x=rng.choice(["bf16", "bf16", "fp16"]), ignored=ignored)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _hidden(gen, M, d):
    """A residual stream: channels of different size, a few outliers among them."""
    size = torch.exp2(torch.rand(d, generator=gen, device="cuda") * 4 - 3)
    size[torch.randint(0, d, (4,), generator=gen, device="cuda")] *= 20
    return torch.randn((M, d), generator=gen, device="cuda") * size


def prepare(case, seed):
    gen = _gen(seed)
    s = dict(case=case)
    op, M, d, dtype = case["op"], case["M"], case["d"], _DTYPES[case["x"]]
    if own:
        from paper_2608_02703_gb300 import archead

        s["archead"] = archead
    if op in ("norm", "norm_grad"):
        s["weight"] = 1 + 0.3 * torch.randn(d, generator=gen, device="cuda")
        if case["x"] != "fp32":
            s["weight"] = s["weight"].to(dtype)
        if op == "norm":
            s["x"] = _hidden(gen, M, d).to(dtype)
            s["residual"] = _hidden(gen, M, d).to(dtype) if case["residual"] else None
            s["sum"] = torch.empty((M, d), dtype=dtype, device="cuda") if case["residual"] else None
            s["y"] = torch.empty((M, d), dtype=_DTYPES[case["y"]], device="cuda") if case["y"] else None
            s["codes"] = torch.empty((M, d), dtype=torch.int8, device="cuda") if case["codes"] else None
            s["scales"] = torch.empty(M, dtype=torch.float32, device="cuda") if case["codes"] else None
        else:
            s["h"] = _hidden(gen, M, d).to(dtype)
            s["dy"] = (torch.randn((M, d), generator=gen, device="cuda") / d).to(dtype)
            s["dsum"] = (torch.randn((M, d), generator=gen, device="cuda") / d).to(dtype) if case["stream"] else None
            s["rstd"] = (s["h"].double().square().mean(dim=1) + _EPS).rsqrt().float()
            s["dx"] = torch.empty((M, d), dtype=dtype, device="cuda")
            s["dweight"] = torch.empty(d, dtype=torch.float32, device="cuda")
            if own:
                s["norm"] = s["archead"].archead_norm_create(d)
        return s
    # Hidden states after the final norm and a weight whose logits spread by some 2.5; of the tokens with targets about
    # two thirds have one that the model finds likely.
    V = case["V"]
    x = _hidden(gen, M, d)
    x = x * (x.square().mean(dim=1, keepdim=True) + _EPS).rsqrt()
    w = torch.empty((V, d), dtype=dtype, device="cuda")
    rows = max(1, (1 << 28) // d)
    for n in range(0, V, rows):
        w[n:n + rows] = torch.randn((min(rows, V - n), d), generator=gen, device="cuda") * (2.5 / math.sqrt(d))
    targets = torch.randint(0, V, (M,), generator=gen, device="cuda")
    of_target = w[targets].float()
    gain = 15 * torch.rand((M, 1), generator=gen, device="cuda") - 5
    x = x + gain.clamp_min(0) * of_target / of_target.square().sum(dim=1, keepdim=True).clamp_min(1e-3)
    order = torch.rand(M, generator=gen, device="cuda").argsort()
    s["targets"] = torch.where(order < case["ignored"], _IGNORED, targets).to(torch.int32)
    s["x"], s["w"] = x.to(dtype), w
    s["ce"] = torch.empty(M, dtype=torch.float32, device="cuda")
    s["lse"] = torch.empty(M, dtype=torch.float32, device="cuda")
    if op == "step":
        # The mean over the tokens with targets, weighted by how much each counts.
        part = 0.5 + torch.rand(M, generator=gen, device="cuda")
        s["grad"] = part / max(1, M - case["ignored"])
        s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(w)
    if own:
        s["loss"] = s["archead"].archead_loss_create(M, V, d, gradient=op == "step")
    return s


def run(state):
    case = state["case"]
    return _own(state, case) if own else _plain(state, case)


def _plain_norm(s, case):
    out = {}
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
        s["sum"].copy_(h)
        out["sum"] = s["sum"]
    # The codes stand next to borders: the factor in 64 bits, rounded once.
    rstd = (h.double().square().mean(dim=1, keepdim=True) + _EPS).rsqrt().float()
    y = (h.float() * rstd) * s["weight"].float()
    if s["y"] is not None:
        s["y"].copy_(y)
        out["y"] = s["y"]
    if s["codes"] is not None:
        top = y.abs().amax(dim=1)
        scales = top / torch.full_like(top, 127)  # (by a Python number: a product with its rounded reciprocal on the GPU)
        usable = (scales > 0) & torch.isfinite(scales)
        q = torch.round(y / torch.where(usable, scales, 1)[:, None]).clamp(-127, 127)
        s["codes"].copy_(torch.where(usable[:, None], q, 0))
        s["scales"].copy_(scales)
        out["values"] = s["codes"].float() * s["scales"][:, None]
        out["scales"] = s["scales"]
    return out


def _plain_norm_grad(s):
    n = s["h"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["weight"].float()
    dx = s["rstd"][:, None] * (g - n * (g * n).mean(dim=1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["dx"].dtype), "dweight": (dy * n).sum(dim=0)}


def _plain_logits(s):
    """The logits of the tokens that have targets, and what is known of each."""
    counts = s["targets"] != _IGNORED
    x, targets = s["x"][counts].float(), s["targets"][counts].long()
    logits = x @ s["w"].float().t()
    top = logits.amax(dim=1)
    lse = top + torch.log(torch.exp(logits - top[:, None]).sum(dim=1))
    ce, every = torch.zeros_like(s["ce"]), torch.zeros_like(s["lse"])
    ce[counts] = lse - logits.gather(1, targets[:, None])[:, 0]
    every[counts] = lse
    return counts, x, targets, logits, lse, {"ce": ce, "lse": every}


def _plain(s, case):
    if case["op"] == "norm":
        return _plain_norm(s, case)
    if case["op"] == "norm_grad":
        return _plain_norm_grad(s)
    counts, x, targets, logits, lse, out = _plain_logits(s)
    if case["op"] == "loss":
        return out
    p = torch.exp_(logits.sub_(lse[:, None]))
    p.scatter_add_(1, targets[:, None], torch.full_like(lse, -1)[:, None])
    p.mul_(s["grad"][counts][:, None])
    dx = torch.zeros_like(s["x"])
    dx[counts] = (p @ s["w"].float()).to(dx.dtype)
    return dict(out, dx=dx, dw=(p.t() @ x).to(s["w"].dtype))


def _own(s, case):
    op, lib = case["op"], s["archead"]
    if op == "norm":
        lib.archead_rms_norm(s["x"], s["weight"], _EPS, y=s["y"], residual=s["residual"], sum=s["sum"],
                             codes=s["codes"], scales=s["scales"])
        out = {k: s[k] for k in ("sum", "y", "scales") if s[k] is not None}
        if s["codes"] is not None:
            out["values"] = s["codes"].float() * s["scales"][:, None]
        return out
    if op == "norm_grad":
        lib.archead_rms_norm_backward(s["norm"], s["dy"], s["h"], s["weight"], s["rstd"], s["dx"],
                                      dweight=s["dweight"], dsum=s["dsum"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    lib.archead_linear_ce(s["loss"], s["x"], s["w"], s["targets"], s["ce"], lse=s["lse"], ignore_index=_IGNORED)
    if op == "loss":
        return {"ce": s["ce"], "lse": s["lse"]}
    lib.archead_linear_ce_backward(s["loss"], s["x"], s["w"], s["targets"], s["lse"], s["grad"], dx=s["dx"],
                                   dw=s["dw"], ignore_index=_IGNORED)
    return {"ce": s["ce"], "lse": s["lse"], "dx": s["dx"], "dw": s["dw"]}


def work(case):
    op, M, d = case["op"], case["M"], case["d"]
    b = _BYTES[case["x"]]
    if op == "norm":
        row = d * (b + (2 * b if case["residual"] else 0) + (_BYTES[case["y"]] if case["y"] else 0))
        row += d + 4 if case["codes"] else 0
        return {"bytes": M * row + d * b, "flops": 4 * M * d}
    if op == "norm_grad":
        return {"bytes": M * (d * b * (4 if case["stream"] else 3) + 4) + d * (b + 4), "flops": 10 * M * d}
    V, live = case["V"], case["M"] - case["ignored"]
    products = 1 if op == "loss" else 4
    flops = products * 2 * live * V * d
    bytes_ = V * d * b + live * d * b + 12 * M
    if op == "step":
        # The gradients, and the weight once more: no product of the gradient can begin before the last sum has ended.
        bytes_ += 2 * V * d * b + M * d * b + 4 * M
    return {"bytes": bytes_, "flops": flops}


def exact(case, seed):
    """run()'s answer from the definitions in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h = s["x"].double()
        out = {}
        if s["residual"] is not None:
            h = h + s["residual"].double()
            out["sum"] = h
            h = h.to(s["x"].dtype).double()
        y = h / torch.sqrt(h.pow(2).sum(dim=1, keepdim=True) / case["d"] + _EPS) * s["weight"].double()
        if s["y"] is not None:
            out["y"] = y
        if s["codes"] is not None:
            out["values"], out["scales"] = None, y.abs().max(dim=1).values / 127
        return out
    if op == "norm_grad":
        h, w, dy = s["h"].double(), s["weight"].double(), s["dy"].double()
        r = s["rstd"].double()[:, None]
        inner = (dy * w * h).sum(dim=1, keepdim=True)
        dx = r * dy * w - h * r.pow(3) * inner / case["d"]
        if s["dsum"] is not None:
            dx += s["dsum"].double()
        return {"dx": dx, "dweight": torch.einsum("mk,mk,m->k", dy, h, r[:, 0])}
    live = case["M"] - case["ignored"]
    if live * case["V"] * case["d"] * (1 if op == "loss" else 3) > 3e12:
        return None  # (64-bit products of this size take too long)
    w = s["w"].double()
    ce = torch.zeros(case["M"], dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(ce)
    dx = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda") if op == "step" else None
    dw = torch.zeros_like(w) if op == "step" else None
    at = torch.nonzero(s["targets"] != _IGNORED)[:, 0]
    for part in at.split(256):
        x, t = s["x"][part].double(), s["targets"][part].long()
        logits = x @ w.t()
        logp = torch.log_softmax(logits, dim=1)
        ce[part] = -logp[torch.arange(len(part), device="cuda"), t]
        lse[part] = torch.logsumexp(logits, dim=1)
        if op == "step":
            p = logp.exp()
            p[torch.arange(len(part), device="cuda"), t] -= 1
            p *= s["grad"][part].double()[:, None]
            dx[part] = p @ w
            dw += p.t() @ x
    return {"ce": ce, "lse": lse} if op == "loss" else {"ce": ce, "lse": lse, "dx": dx, "dw": dw}
