"""Timing and accuracy cases of the operators between the matrix products of a decoder-style language model's training step.

  norm     layer_norm_forward + layer_norm_backward   layer norm (or without centring) of a residual sum, its result kept in 8 bits on
                                                      request, and its gradients, the reduction of the weight's among them
  rotary   rotary_forward + rotary_backward           rotary positions of queries and keys, and of their gradients
  teach    linear_distillation                        the last layer's distance from a teacher's top logits, loss only
  learn    linear_distillation_grad                   the same with the gradients of the hidden states and of the vocabulary matrix

A case is a dict of plain values.  `prepare` makes the inputs, `run` makes one pass: with `own` the calls of this package,
without it the same operators in elementary torch operations in 32 bits (angles in 64).  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

GROUP = 32                  # values of a row that share one power-of-two scale in an 8-bit checkpoint
EPS = 1e-5
DEVICE = "cuda"

_NORM_CAP = 16384 * 2048              # tokens x width of the largest drawn call
_ROTARY_CAP = 16384 * 32 * 128        # tokens x heads x width of a head
_TEACH_CAP = 16384 * 32000 * 2048     # tokens x vocabulary x width, loss only
_LEARN_CAP = 8192 * 131072 * 2048     # ... with gradients


def listed():
    return [
        # one token behind a prompt: launches and latency
        {"name": "norm-one-token", "op": "norm", "tokens": 1, "width": 768, "dtype": "bfloat16", "center": True, "residual": True, "keep": False},
        # the norm in front of a projection of the 12-layer stack: no centring, residual sum, the result kept for weight gradients
        {"name": "norm-768", "op": "norm", "tokens": 4096, "width": 768, "dtype": "bfloat16", "center": False, "residual": True, "keep": True},
        # a float32 residual stream with an odd number of tokens and an odd width
        {"name": "norm-ragged", "op": "norm", "tokens": 1537, "width": 771, "dtype": "float32", "center": True, "residual": False, "keep": False},
        # hidden size of the 24-layer stack over a large batch
        {"name": "norm-2048", "op": "norm", "tokens": 16384, "width": 2048, "dtype": "bfloat16", "center": True, "residual": True, "keep": False},
        # one token at a far position: twelve heads of 64
        {"name": "rotary-one-token", "op": "rotary", "tokens": 1, "heads": 12, "key_heads": 12, "head": 64, "rotated": 64, "layout": "half", "dtype": "bfloat16",
         "reach": 1 << 20, "factor": 8.0},
        # a ragged piece, a part of each head rotated, neighbouring pairs, float32
        {"name": "rotary-ragged", "op": "rotary", "tokens": 1023, "heads": 9, "key_heads": 3, "head": 80, "rotated": 20, "layout": "interleaved", "dtype": "float32",
         "reach": 4096, "factor": 1.0},
        # hidden size of the 24-layer stack: 16 heads of 128 over a large batch, long contexts
        {"name": "rotary-2048", "op": "rotary", "tokens": 16384, "heads": 16, "key_heads": 16, "head": 128, "rotated": 128, "layout": "half", "dtype": "bfloat16",
         "reach": 1 << 17, "factor": 16.0},
        # one token scored against a teacher's few logits: the vocabulary matrix is read once for one row
        {"name": "teach-one-token", "op": "teach", "tokens": 1, "width": 768, "vocab": 32000, "top": 8, "temperature": 1.0, "empty": 0.0, "weighted": False,
         "spread": 0.6, "dtype": "float32"},
        # held-out text with padding, a soft target, vocabulary size without a factor of two
        {"name": "teach-ragged", "op": "teach", "tokens": 777, "width": 768, "vocab": 50257, "top": 50, "temperature": 2.0, "empty": 0.3, "weighted": False,
         "spread": 1.0, "dtype": "bfloat16"},
        # a training micro-batch of the 12-layer stack (hidden 768)
        {"name": "learn-768", "op": "learn", "tokens": 4096, "width": 768, "vocab": 32000, "top": 64, "temperature": 1.0, "empty": 0.05, "weighted": False,
         "spread": 0.6, "dtype": "bfloat16"},
        # packed sequences with a weight per token, odd number of tokens, odd vocabulary
        {"name": "learn-ragged", "op": "learn", "tokens": 1023, "width": 2048, "vocab": 50257, "top": 100, "temperature": 2.0, "empty": 0.1, "weighted": True,
         "spread": 1.0, "dtype": "float32"},
        # the largest: hidden 2048, vocabulary of 131072, whose logits would take 4 GB in 32 bits
        {"name": "learn-large", "op": "learn", "tokens": 8192, "width": 2048, "vocab": 131072, "top": 32, "temperature": 1.0, "empty": 0.0, "weighted": False,
         "spread": 1.0, "dtype": "bfloat16"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "rotary", "rotary", "teach", "learn"])
    while True:
        if op == "norm":
            case = {"op": op, "tokens": _log(rng, 1, 16384), "width": _log(rng, 64, 8192), "dtype": rng.choice(["bfloat16", "bfloat16", "float32"]),
                    "center": rng.random() < 0.5, "residual": rng.random() < 0.5, "keep": rng.random() < 0.5}
            if rng.random() < 0.7:      # most layers have widths that are multiples of 64
                case["width"] = max(64, case["width"] // 64 * 64)
            if case["tokens"] * case["width"] <= _NORM_CAP:
                return case
        elif op == "rotary":
            head = rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256, 2 * rng.randint(8, 128)])
            keys = rng.randint(1, 16)
            case = {"op": op, "tokens": _log(rng, 1, 16384), "heads": keys * rng.choice([1, 2, 4]), "key_heads": keys, "head": head,
                    "rotated": head if rng.random() < 0.6 else 2 * rng.randint(1, head // 2), "layout": rng.choice(["half", "interleaved"]),
                    "dtype": rng.choice(["bfloat16", "bfloat16", "float32"]), "reach": _log(rng, 128, 1 << 20), "factor": rng.choice([1.0, 4.0, 32.0])}
            if case["tokens"] * (case["heads"] + keys) * head <= _ROTARY_CAP:
                return case
        else:
            case = {"op": op, "tokens": _log(rng, 1, 16384 if op == "teach" else 8192), "width": 8 * _log(rng, 32, 512), "vocab": _log(rng, 1000, 131072),
                    "top": _log(rng, 1, 256), "temperature": rng.choice([1.0, 1.0, 2.0, 0.7]), "empty": rng.choice([0.0, 0.05, 0.3]),
                    "weighted": rng.random() < 0.3, "spread": round(rng.uniform(0.5, 1.5), 2), "dtype": rng.choice(["bfloat16", "float32"])}
            if case["tokens"] * case["width"] * case["vocab"] <= (_TEACH_CAP if op == "teach" else _LEARN_CAP):
                return case


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 7919 + 17)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEVICE)

    T, dtype = case["tokens"], getattr(torch, case["dtype"])
    state = {"op": case["op"]}
    if case["op"] == "norm":
        F = case["width"]
        channel = torch.exp(0.5 * normal(F))             # channels of different size and offset, a few of them large
        state["x"] = (normal(T, F) * channel + 0.3 * normal(F)).to(dtype)
        state["residual"] = (normal(T, F) * channel.flip(0)).to(dtype) if case["residual"] else None
        state["weight"] = 1 + 0.2 * normal(F)
        state["bias"] = 0.1 * normal(F) if case["center"] else None
        state["dy"] = (normal(T, F) * 1e-3).to(dtype)
        state["d_x"] = (normal(T, F) * 1e-3).to(dtype) if case["residual"] else None       # what reaches the sum from the layers behind it
        state["center"], state["keep"] = case["center"], case["keep"]
        return state
    if case["op"] == "rotary":
        H, K, D, R = case["heads"], case["key_heads"], case["head"], case["rotated"]
        packed = normal(T, H + 2 * K, D).to(dtype)       # queries, keys and values side by side, as one projection leaves them
        state["q"], state["k"] = packed[:, :H], packed[:, H:H + K]
        state["dq"], state["dk"] = (normal(T, H, D) * 1e-3).to(dtype), (normal(T, K, D) * 1e-3).to(dtype)
        start = torch.randint(case["reach"], (1,), generator=g, device=DEVICE)
        state["positions"] = (start + torch.arange(T, device=DEVICE)) % case["reach"]      # a piece of a long context
        f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=DEVICE) / R)
        turns = f * (8192 / (2 * math.pi))               # within the length that the model was trained on
        share = ((turns - 1) / 3).clamp(0, 1)            # slow pairs are stretched by the factor, fast ones left alone
        state["frequencies"] = f * (share + (1 - share) / case["factor"])
        state["scale"] = 1 + 0.1 * math.log(case["factor"])
        state["layout"] = case["layout"]
        return state
    V, D, K = case["vocab"], case["width"], case["top"]
    # hidden states behind a norm have entries of size one; `spread` is the standard deviation of the logits
    state["hidden"] = normal(T, D).to(torch.bfloat16)
    state["weight"] = (normal(V, D) * (case["spread"] / math.sqrt(D))).to(torch.bfloat16)
    state["logits"] = torch.sort(2 * normal(T, K), dim=1, descending=True).values.to(dtype)
    gap = torch.randint(1, V // K + 1, (T, K), generator=g, device=DEVICE)                 # distinct columns in an order of their own
    column = gap.cumsum(1) - 1
    turn = torch.argsort(uniform(T, K), dim=1)
    index = column.gather(1, turn)
    index[uniform(T, K) < 0.02] = -1                     # a teacher's list that is shorter than the others
    index[uniform(T) < case["empty"]] = -1               # padding
    state["index"] = index
    state["token_weight"] = uniform(T) if case["weighted"] else None
    state["temperature"] = case["temperature"]
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- the package's calls ------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2509_11254_b200 as psgd

    if s["op"] == "norm":
        r = psgd.layer_norm_forward(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS, center=s["center"], keep=s["keep"])
        d = psgd.layer_norm_backward(s["dy"], r.x, s["weight"], r.mean, r.rstd, d_x=s["d_x"], bias=s["bias"] is not None)
        out = {"y": r.y, "rstd": r.rstd, "d_x": d.d_x, "d_weight": d.d_weight}
        if s["residual"] is not None:
            out["x"] = r.x
        if s["center"]:
            out.update(mean=r.mean, d_bias=d.d_bias)
        if s["keep"]:
            out["kept"] = r.kept.unpack()                      # exact in bfloat16
        return out
    if s["op"] == "rotary":
        q, k = psgd.rotary_forward(s["q"], s["k"], s["positions"], s["frequencies"], layout=s["layout"], scale=s["scale"])
        dq, dk = psgd.rotary_backward(s["dq"], s["dk"], s["positions"], s["frequencies"], layout=s["layout"], scale=s["scale"])
        return {"q": q, "k": k, "dq": dq, "dk": dk}
    call = psgd.linear_distillation if s["op"] == "teach" else psgd.linear_distillation_grad
    r = call(s["hidden"], s["weight"], s["logits"], s["index"], temperature=s["temperature"], token_weight=s["token_weight"])
    return r._asdict()


# ---- elementary torch operations, 32 bits -------------------------------------------------------------------------
def _kept(x):
    """The values that an 8-bit checkpoint of x stands for: per row and group of 32 values one scale 2^e, e the smallest
    integer with max|x| <= 127 * 2^e (within -126..121), and whole numbers rint(x / 2^e) within -127..127."""
    T, F = x.shape
    G = -(-F // GROUP)
    groups = x.new_zeros((T, G * GROUP), dtype=torch.float32)
    groups[:, :F] = x
    groups = groups.view(T, G, GROUP)
    mantissa, exponent = torch.frexp(groups.abs().amax(2, keepdim=True))
    e = (exponent - 7 + (mantissa > 127 / 128)).clamp(-126, 121)
    q = torch.round(torch.ldexp(groups, -e)).clamp(-127, 127)
    return torch.ldexp(q, e).view(T, G * GROUP)[:, :F]


def _norm_plain(s):
    dtype = s["x"].dtype
    x = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dtype)
    v = x.float()
    mean = v.mean(1) if s["center"] else torch.zeros_like(v[:, 0])
    v = v - mean[:, None]
    rstd = 1 / torch.sqrt(v.square().mean(1) + EPS)
    v = v * rstd[:, None]
    y = v * s["weight"]
    if s["bias"] is not None:
        y = y + s["bias"]
    y = y.to(dtype)
    dy = s["dy"].float()
    g = dy * s["weight"]
    d = g - v * (g * v).mean(1, keepdim=True)
    if s["center"]:
        d = d - g.mean(1, keepdim=True)
    d = d * rstd[:, None]
    if s["d_x"] is not None:
        d = d + s["d_x"].float()
    out = {"y": y, "rstd": rstd, "d_x": d.to(dtype), "d_weight": (dy * v).sum(0)}
    if s["residual"] is not None:
        out["x"] = x
    if s["center"]:
        out.update(mean=mean, d_bias=dy.sum(0))
    if s["keep"]:
        out["kept"] = _kept(y).bfloat16()
    return out


def _turned(x, cos, sin, layout):
    """x [T, heads, D] with the pairs of its first 2 * cos.shape[1] values turned by angles whose cosines and sines [T, pairs] are given."""
    n = cos.shape[1]
    v = x.float()
    cos, sin = cos[:, None], sin[:, None]
    out = v.clone()
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    out[..., first] = v[..., first] * cos - v[..., second] * sin
    out[..., second] = v[..., first] * sin + v[..., second] * cos
    return out.to(x.dtype)


def _rotary_plain(s):
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = (torch.cos(angle) * s["scale"]).float(), (torch.sin(angle) * s["scale"]).float()
    return {"q": _turned(s["q"], cos, sin, s["layout"]), "k": _turned(s["k"], cos, sin, s["layout"]),
            "dq": _turned(s["dq"], cos, -sin, s["layout"]), "dk": _turned(s["dk"], cos, -sin, s["layout"])}


def _run_plain(s):
    if s["op"] == "norm":
        return _norm_plain(s)
    if s["op"] == "rotary":
        return _rotary_plain(s)
    tau = s["temperature"]
    hidden, weight, index = s["hidden"].float(), s["weight"].float(), s["index"]
    there = index >= 0
    z = torch.where(there, s["logits"].float() / tau, -math.inf)
    counts = there.any(1)
    z = z - torch.where(counts, z.amax(1), 0.0)[:, None]
    q = torch.exp(z)
    total = q.sum(1, keepdim=True)
    total = torch.where(counts[:, None], total, 1.0)
    q = q / total
    logits = hidden @ weight.T
    logits /= tau
    top = logits.amax(1, keepdim=True)
    logits -= top
    at = torch.where(there, index, 0)
    mine = logits.gather(1, at)
    logits.exp_()
    sums = logits.sum(1, keepdim=True)
    log_sum = torch.log(sums)
    gap = torch.where(there, (z - torch.log(total)) - (mine - log_sum), 0.0)
    token_loss = tau * tau * (q * gap).sum(1)
    w = counts.float() if s["token_weight"] is None else torch.where(counts, s["token_weight"], 0.0)
    norm = w.sum()
    w = torch.where(norm != 0, w / norm, 0.0)
    out = {"loss": (w * token_loss).sum(), "token_loss": token_loss, "lse": (top + log_sum)[:, 0]}
    if s["op"] == "learn":
        logits /= sums
        logits.scatter_add_(1, at, -q)                   # q is 0 where there is no entry
        logits *= w[:, None] * tau
        out["d_hidden"] = (logits @ weight).bfloat16()
        out["d_weight"] = (logits.T @ hidden).bfloat16()
    return out


# ---- what the path cannot do without ------------------------------------------------------------------------------
def work(case):
    T, size = case["tokens"], 4 if case["dtype"] == "float32" else 2
    if case["op"] == "norm":
        F = case["width"]
        forward = (2 + 2 * case["residual"]) * T * F * size      # x (and what is added to it) read, y (and the sum) written
        if case["keep"]:
            # the result in 8 bits written; read, and its values written in bfloat16
            forward += 2 * (T * F + T * -(-F // GROUP)) + 2 * T * F
        backward = (3 + case["residual"]) * T * F * size         # dy, x (and the residual path's gradient) read, d_x written
        return {"bytes": forward + backward + 16 * T + 16 * F, "flops": 20 * T * F}
    if case["op"] == "rotary":
        values = T * (case["heads"] + case["key_heads"]) * case["head"]
        return {"bytes": 4 * values * size + 16 * T, "flops": 6 * values}
    V, D, K = case["vocab"], case["width"], case["top"]
    rows = T * (4 + 4 + (4 if case["weighted"] else 0)) + T * K * (8 + size) + 4
    once = 2 * D * (T + V)
    if case["op"] == "teach":
        return {"bytes": once + rows, "flops": 2 * T * V * D}
    return {"bytes": 2 * once + rows, "flops": 6 * T * V * D}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _stands_for(y):
    """An 8-bit checkpoint's values, group by group of columns, in 64 bits; inputs are finite here."""
    out = torch.empty_like(y)
    for c in range(0, y.shape[1], GROUP):
        block = y[:, c:c + GROUP]
        top = block.abs().max(dim=1, keepdim=True).values
        e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -130) / 127))
        e = torch.where(127 * torch.exp2(e) < top, e + 1, e)             # log2 was rounded
        e = torch.where(127 * torch.exp2(e - 1) >= top, e - 1, e)
        s = torch.exp2(torch.clamp(e, -126, 121))
        out[:, c:c + GROUP] = torch.clamp(torch.round(block / s), -127, 127) * s
    return out


def _exact_norm(s):
    dtype = s["x"].dtype
    x = s["x"].double()
    if s["residual"] is not None:
        x = (x + s["residual"].double()).to(dtype).double()              # the sum is held in the inputs' type
    F = x.shape[1]
    mean = x.sum(1, keepdim=True) / F if s["center"] else 0.0 * x[:, :1]
    var = ((x - mean) ** 2).sum(1, keepdim=True) / F
    rstd = (var + EPS) ** -0.5
    xh = (x - mean) * rstd
    w = s["weight"].double()
    y = xh * w + (0.0 if s["bias"] is None else s["bias"].double())
    dy = s["dy"].double()
    # through the projection that takes the row's own direction (and its mean) out of the gradient
    g = dy * w
    along = torch.einsum("tf,tf->t", g, xh)[:, None] / F
    d = rstd * (g - xh * along - (g.sum(1, keepdim=True) / F if s["center"] else 0.0))
    if s["d_x"] is not None:
        d = d + s["d_x"].double()
    out = {"y": y, "rstd": rstd[:, 0], "d_x": d, "d_weight": torch.einsum("tf,tf->f", dy, xh)}
    if s["residual"] is not None:
        out["x"] = x
    if s["center"]:
        out.update(mean=mean[:, 0], d_bias=dy.sum(0))
    if s["keep"]:
        out["kept"] = _stands_for(y.to(dtype).double())                  # of the result in its own type
    return out


def _exact_rotary(s):
    def rotated(x, way):
        n = s["frequencies"].numel()
        turn = torch.polar(torch.full_like(angle, s["scale"]), way * angle)[:, None]
        v = x.double()
        head = v[..., :2 * n]
        pairs = head.unflatten(2, (2, n)).transpose(2, 3) if s["layout"] == "half" else head.unflatten(2, (n, 2))
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        head = pairs.transpose(2, 3).flatten(2) if s["layout"] == "half" else pairs.flatten(2)
        return torch.cat([head, v[..., 2 * n:]], 2)

    angle = s["positions"].double()[:, None] * s["frequencies"]
    return {"q": rotated(s["q"], 1), "k": rotated(s["k"], 1), "dq": rotated(s["dq"], -1), "dk": rotated(s["dk"], -1)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "rotary":
        return _exact_rotary(s)
    T, V, tau = case["tokens"], case["vocab"], case["temperature"]
    W = s["weight"].double()
    there = s["index"] >= 0
    counts = there.any(1)
    w = counts.double() if s["token_weight"] is None else s["token_weight"].double() * counts
    norm = float(w.sum())
    w = w / norm if norm else torch.zeros_like(w)
    lse = torch.empty(T, dtype=torch.float64, device=DEVICE)
    token_loss = torch.zeros_like(lse)
    d_hidden, d_weight = torch.empty((T, case["width"]), dtype=torch.float64, device=DEVICE), torch.zeros_like(W)
    piece = max(1, (1 << 27) // V)
    for a in range(0, T, piece):
        b = min(T, a + piece)
        h = s["hidden"][a:b].double()
        log_p = torch.log_softmax(h @ W.T / tau, 1)
        lse[a:b] = torch.logsumexp(h @ W.T / tau, 1)
        z = s["logits"][a:b].double() / tau
        z = torch.where(there[a:b], z, -torch.inf)
        z[~counts[a:b]] = 0.0
        log_q = torch.log_softmax(z, 1)
        q = torch.exp(log_q) * there[a:b]
        at = s["index"][a:b].clamp(min=0)
        token_loss[a:b] = tau ** 2 * torch.where(q > 0, q * (log_q - log_p.gather(1, at)), 0.0).sum(1)
        if case["op"] == "learn":
            d = torch.exp(log_p)
            d.scatter_add_(1, at, -q)
            d *= tau * w[a:b, None]
            d_hidden[a:b] = d @ W
            d_weight += d.T @ h
    out = {"loss": (w * token_loss).sum(), "token_loss": token_loss, "lse": lse}
    if case["op"] == "learn":
        out.update(d_hidden=d_hidden, d_weight=d_weight)
    return out
