"""Timing and accuracy cases of the training operators that stand around the gradient compression.

The compressor takes a stack of weight gradients.  These operators are where such gradients come from in a decoder-style
language model whose activations are kept in 8 bits between the forward and the backward pass:

  loss    linear_cross_entropy         the last layer and its softmax cross entropy, loss only (held-out text)
  step    linear_cross_entropy_grad    the same with the gradients of the hidden states and of the vocabulary matrix
  linear  pack_activation + weight_gradient   a linear layer's input kept in 8 bits, and its weight gradient from them
  gated   swiglu_forward + swiglu_backward    the gated unit of the feed-forward block, its two inputs kept in 8 bits

A case is a dict of plain values.  `prepare` makes the inputs, `run` makes one pass: with `own` the calls of this package,
without it the same operators in elementary torch operations in 32 bits.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

IGNORE = -100
GROUP = 32                  # values of a row that share one power-of-two scale in an 8-bit checkpoint
DEVICE = "cuda"

_LOSS_CAP = 16384 * 32000 * 2048      # tokens x vocabulary x width of the largest drawn call, loss only
_STEP_CAP = 8192 * 131072 * 2048      # ... with gradients
_LINEAR_CAP = 16384 * 5504 * 2048
_GATED_CAP = 16384 * 5504


def listed():
    return [
        # one token scored against the whole vocabulary: latency, the vocabulary matrix is read once for one row
        {"name": "loss-one-token", "op": "loss", "tokens": 1, "width": 768, "vocab": 32000, "ignored": 0.0, "weighted": False, "spread": 0.6},
        # a ragged piece of held-out text with padding, vocabulary size without a factor of two
        {"name": "loss-ragged", "op": "loss", "tokens": 777, "width": 768, "vocab": 50257, "ignored": 0.3, "weighted": False, "spread": 1.0},
        # perplexity over a large batch, hidden size of the 24-layer stack
        {"name": "loss-eval", "op": "loss", "tokens": 16384, "width": 2048, "vocab": 32000, "ignored": 0.0, "weighted": False, "spread": 1.0},
        # a training micro-batch of the 12-layer stack (hidden 768)
        {"name": "step-768", "op": "step", "tokens": 4096, "width": 768, "vocab": 32000, "ignored": 0.05, "weighted": False, "spread": 0.6},
        # packed sequences with a weight per token, odd number of tokens, odd vocabulary
        {"name": "step-ragged", "op": "step", "tokens": 1023, "width": 2048, "vocab": 50257, "ignored": 0.1, "weighted": True, "spread": 1.0},
        # the largest: hidden 2048, vocabulary of 131072, whose logits would take 4 GB in 32 bits
        {"name": "step-large", "op": "step", "tokens": 8192, "width": 2048, "vocab": 131072, "ignored": 0.0, "weighted": False, "spread": 1.0},
        # the gate projection of the 12-layer stack, gradient in the compressor's 16-bit input type
        {"name": "linear-768", "op": "linear", "tokens": 4096, "inputs": 768, "outputs": 2048, "grad": "bfloat16"},
        # odd sizes everywhere, gradient in the compressor's 32-bit input type
        {"name": "linear-ragged", "op": "linear", "tokens": 1537, "inputs": 771, "outputs": 1001, "grad": "float32"},
        # the gate projection of the 24-layer stack over a large batch
        {"name": "linear-2048", "op": "linear", "tokens": 16384, "inputs": 2048, "outputs": 5504, "grad": "float32"},
        # a few tokens: launches and latency
        {"name": "gated-small", "op": "gated", "tokens": 33, "inputs": 2048},
        # the 12-layer stack's feed-forward width
        {"name": "gated-2048", "op": "gated", "tokens": 4096, "inputs": 2048},
        # the 24-layer stack's over a large batch
        {"name": "gated-5504", "op": "gated", "tokens": 16384, "inputs": 5504},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["loss", "step", "linear", "gated"])
    while True:
        if op in ("loss", "step"):
            case = {"op": op, "tokens": _log(rng, 1, 16384 if op == "loss" else 8192), "width": 8 * _log(rng, 32, 512),
                    "vocab": _log(rng, 1000, 131072), "ignored": rng.choice([0.0, 0.05, 0.3]), "weighted": rng.random() < 0.3,
                    "spread": round(rng.uniform(0.5, 1.5), 2)}
            if case["tokens"] * case["width"] * case["vocab"] <= (_LOSS_CAP if op == "loss" else _STEP_CAP):
                return case
        elif op == "linear":
            case = {"op": op, "tokens": _log(rng, 1, 16384), "inputs": _log(rng, 128, 5504), "outputs": _log(rng, 128, 5504),
                    "grad": rng.choice(["bfloat16", "float32"])}
            if rng.random() < 0.7:      # most layers have widths that are multiples of 64
                case["inputs"], case["outputs"] = (max(64, v // 64 * 64) for v in (case["inputs"], case["outputs"]))
            if case["tokens"] * case["inputs"] * case["outputs"] <= _LINEAR_CAP:
                return case
        else:
            case = {"op": op, "tokens": _log(rng, 1, 16384), "inputs": _log(rng, 128, 5504)}
            if rng.random() < 0.7:
                case["inputs"] = max(64, case["inputs"] // 64 * 64)
            if case["tokens"] * case["inputs"] <= _GATED_CAP:
                return case


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 7919 + 13)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    state = {"op": case["op"]}
    T = case["tokens"]
    if case["op"] in ("loss", "step"):
        V, D = case["vocab"], case["width"]
        # hidden states behind a norm have entries of size one; `spread` is the standard deviation of the logits
        state["hidden"] = normal(T, D).to(torch.bfloat16)
        state["weight"] = (normal(V, D) * (case["spread"] / math.sqrt(D))).to(torch.bfloat16)
        labels = torch.randint(V, (T,), generator=g, device=DEVICE)
        labels[torch.rand((T,), generator=g, device=DEVICE) < case["ignored"]] = IGNORE
        state["labels"] = labels
        state["token_weight"] = torch.rand((T,), generator=g, device=DEVICE) if case["weighted"] else None
        return state
    F = case["inputs"]
    # activations of a trained model: channels of different size, a few of them large
    channel = torch.exp(0.5 * normal(F))
    if case["op"] == "linear":
        state["x"] = (normal(T, F) * channel).to(torch.bfloat16)
        state["dy"] = (normal(T, case["outputs"]) * 1e-3).to(torch.bfloat16)
        state["grad"] = getattr(torch, case["grad"])
        return state
    state["gate"] = (normal(T, F) * channel).to(torch.bfloat16)
    state["up"] = (normal(T, F) * channel.flip(0)).to(torch.bfloat16)
    state["dh"] = (normal(T, F) * 1e-3).to(torch.bfloat16)
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- the package's calls ------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2509_11254_b200 as psgd

    if s["op"] == "loss":
        r = psgd.linear_cross_entropy(s["hidden"], s["weight"], s["labels"], token_weight=s["token_weight"], ignore_index=IGNORE)
        return {"loss": r.loss, "token_loss": r.token_loss, "lse": r.lse}
    if s["op"] == "step":
        r = psgd.linear_cross_entropy_grad(s["hidden"], s["weight"], s["labels"], token_weight=s["token_weight"], ignore_index=IGNORE)
        return {"loss": r.loss, "token_loss": r.token_loss, "lse": r.lse, "d_hidden": r.d_hidden, "d_weight": r.d_weight}
    if s["op"] == "linear":
        kept = psgd.pack_activation(s["x"])                                          # forward
        return {"d_weight": psgd.weight_gradient(s["dy"], kept, dtype=s["grad"])}    # backward
    h, gate, up = psgd.swiglu_forward(s["gate"], s["up"])                            # forward
    d_gate, d_up, h_again = psgd.swiglu_backward(s["dh"], gate, up, recompute=True)  # backward
    return {"h": h, "d_gate": d_gate, "d_up": d_up, "h_again": h_again}


# ---- elementary torch operations, 32 bits -------------------------------------------------------------------------
def _kept(x):
    """The values that an 8-bit checkpoint of x stands for: per row and group of 32 values one scale 2^e, e the smallest
    integer with max|x| <= 127 * 2^e (within -126..121), and whole numbers rint(x / 2^e) within -127..127.  A group that
    holds an infinity or a NaN stands for NaN throughout."""
    T, F = x.shape
    G = -(-F // GROUP)
    groups = x.new_zeros((T, G * GROUP), dtype=torch.float32)
    groups[:, :F] = x
    groups = groups.view(T, G, GROUP)
    top = groups.abs().amax(2, keepdim=True)
    fine = torch.isfinite(groups).all(2, keepdim=True)
    mantissa, exponent = torch.frexp(torch.where(fine, top, 0.0))
    e = (exponent - 7 + (mantissa > 127 / 128)).clamp(-126, 121)
    q = torch.round(torch.ldexp(groups, -e)).clamp(-127, 127)
    return torch.where(fine, torch.ldexp(q, e), math.nan).view(T, G * GROUP)[:, :F]


def _run_plain(s):
    if s["op"] == "linear":
        return {"d_weight": (s["dy"].float().T @ _kept(s["x"])).to(s["grad"])}
    if s["op"] == "gated":
        gate, up = s["gate"].float(), s["up"].float()
        h = gate / (1 + torch.exp(-gate)) * up
        gate, up, dh = _kept(s["gate"]), _kept(s["up"]), s["dh"].float()
        sig = 1 / (1 + torch.exp(-gate))
        return {"h": h.bfloat16(), "d_gate": (dh * up * sig * (1 + gate * (1 - sig))).bfloat16(), "d_up": (dh * gate * sig).bfloat16(),
                "h_again": (gate * sig * up).bfloat16()}
    hidden, weight, labels = s["hidden"].float(), s["weight"].float(), s["labels"]
    logits = hidden @ weight.T
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    valid = labels != IGNORE
    at = torch.where(valid, labels, 0)[:, None]
    token_loss = torch.where(valid, lse - logits.gather(1, at)[:, 0], 0.0)
    w = valid.float() if s["token_weight"] is None else torch.where(valid, s["token_weight"], 0.0)
    norm = w.sum()
    w = torch.where(norm != 0, w / norm, 0.0)
    out = {"loss": (w * token_loss).sum(), "token_loss": token_loss, "lse": lse}
    if s["op"] == "step":
        e /= total
        e.scatter_add_(1, at, torch.full_like(total, -1.0))
        e *= w[:, None]
        out["d_hidden"] = (e @ weight).bfloat16()
        out["d_weight"] = (e.T @ hidden).bfloat16()
    return out


# ---- what the path cannot do without ------------------------------------------------------------------------------
def work(case):
    T = case["tokens"]
    if case["op"] in ("loss", "step"):
        V, D = case["vocab"], case["width"]
        rows = T * (8 + 4 + 4 + (4 if case["weighted"] else 0)) + 4
        once = 2 * D * (T + V)
        if case["op"] == "loss":
            return {"bytes": once + rows, "flops": 2 * T * V * D}
        return {"bytes": 2 * once + rows, "flops": 6 * T * V * D}
    F = case["inputs"]
    kept = T * F + T * -(-F // GROUP)          # written in the forward, read in the backward pass
    if case["op"] == "linear":
        O = case["outputs"]
        return {"bytes": 2 * T * F + 2 * kept + 2 * T * O + O * F * (4 if case["grad"] == "float32" else 2), "flops": 2 * T * O * F}
    return {"bytes": (2 * 2 + 2) * T * F + 4 * kept + (2 + 3 * 2) * T * F, "flops": 30 * T * F}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _stands_for(x):
    """An 8-bit checkpoint's values, group by group of columns, in 64 bits; inputs are finite here."""
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], GROUP):
        block = x[:, c:c + GROUP]
        top = block.abs().max(dim=1, keepdim=True).values
        e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -130) / 127))
        e = torch.where(127 * torch.exp2(e) < top, e + 1, e)             # log2 was rounded
        e = torch.where(127 * torch.exp2(e - 1) >= top, e - 1, e)
        s = torch.exp2(torch.clamp(e, -126, 121))
        out[:, c:c + GROUP] = torch.clamp(torch.round(block / s), -127, 127) * s
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return {"d_weight": torch.einsum("to,tf->of", s["dy"].double(), _stands_for(s["x"]))}
    if case["op"] == "gated":
        def silu(v):
            return v * torch.sigmoid(v)

        h = silu(s["gate"].double()) * s["up"].double()
        gate, up, dh = _stands_for(s["gate"]), _stands_for(s["up"]), s["dh"].double()
        eps_free = torch.sigmoid(gate)
        slope = eps_free + gate * eps_free * torch.sigmoid(-gate)
        return {"h": h, "d_gate": dh * up * slope, "d_up": dh * silu(gate), "h_again": silu(gate) * up}
    T, V = case["tokens"], case["vocab"]
    W = s["weight"].double()
    valid = s["labels"] >= 0
    w = valid.double() if s["token_weight"] is None else s["token_weight"].double() * valid
    norm = float(w.sum())
    w = w / norm if norm else torch.zeros_like(w)
    lse = torch.empty(T, dtype=torch.float64, device=DEVICE)
    token_loss = torch.zeros_like(lse)
    d_hidden, d_weight = torch.empty((T, case["width"]), dtype=torch.float64, device=DEVICE), torch.zeros_like(W)
    piece = max(1, (1 << 27) // V)
    for a in range(0, T, piece):
        b = min(T, a + piece)
        h = s["hidden"][a:b].double()
        z = h @ W.T
        lse[a:b] = torch.logsumexp(z, 1)
        rows = torch.arange(b - a, device=DEVICE)[valid[a:b]]
        cols = s["labels"][a:b][valid[a:b]]
        token_loss[a:b][valid[a:b]] = lse[a:b][valid[a:b]] - z[rows, cols]
        if case["op"] == "step":
            p = torch.softmax(z, 1)
            p[rows, cols] -= 1
            p *= w[a:b, None]
            d_hidden[a:b] = p @ W
            d_weight += p.T @ h
    out = {"loss": (w * token_loss).sum(), "token_loss": token_loss, "lse": lse}
    if case["op"] == "step":
        out.update(d_hidden=d_hidden, d_weight=d_weight)
    return out
