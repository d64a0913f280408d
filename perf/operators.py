"""What the performance of the token operators is measured on: the operators that follow the per-frame
network, one token per stream and frame, called through the public Python entry points.

  log_probs   scores of classes (or of a vocabulary) -> log probability of given labels, entropy, alternatives
  attention   linear attention with a decay for each head: state per stream, single tokens or whole prompts
  product     few tokens times a matrix of 4-bit weights with a scale for each group along its rows
  norm        norm behind a block, its gate and residual scale, and the norm in front of the next block

Every case names its operator in "op".  `run` computes it in plain operations, in 32 bits and rounded once,
or, where `own` is true, by the library's operator.
"""
from __future__ import annotations

import math

import torch

own = False

# The values of a 4-bit code: sign, two bits of exponent, one of mantissa.
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


# ---- cases ------------------------------------------------------------------------------------
def _log_probs(name, layout, n, classes, h=1, w=1, dtype="f32", top=0, labels=True, masked=0.0):
    """layout "map": scores [n][classes][h][w]; "rows": [n][classes].  masked: share of classes at -inf."""
    c = {"op": "log_probs", "layout": layout, "n": n, "classes": classes, "h": h, "w": w, "dtype": dtype, "top": top,
         "labels": labels, "masked": masked}
    return dict(c, name=name) if name else c


def _attention(name, streams, heads, kv_heads, tokens, dk, dv, dtype="bf16", ragged=False):
    c = {"op": "attention", "streams": streams, "heads": heads, "kv_heads": kv_heads, "tokens": tokens, "dk": dk, "dv": dv,
         "dtype": dtype, "ragged": ragged}
    return dict(c, name=name) if name else c


def _product(name, m, n, k, group, dtype="bf16", bias=False):
    c = {"op": "product", "m": m, "n": n, "k": k, "group": group, "dtype": dtype, "bias": bias}
    return dict(c, name=name) if name else c


def _norm(name, rows, d, group=0, gate="", residual="", next_norm=False, channel_scale=False, post=True, dtype="bf16"):
    c = {"op": "norm", "rows": rows, "d": d, "group": group, "gate": gate, "residual": residual, "next_norm": next_norm,
         "channel_scale": channel_scale, "post": post, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the 8 class maps that the 320x240 network answers a frame with: the confidence of one camera, every frame
        _log_probs("scores_80x60", "map", 1, 8, 60, 80, top=3),
        # one answer for each of 64 streams, from a vocabulary of odd size, an eighth of it ruled out
        _log_probs("answers_64", "rows", 64, 100003, dtype="bf16", top=5, masked=0.125),
        # a long text scored token by token, the largest
        _log_probs("text_2047", "rows", 2047, 131071, dtype="bf16", top=8),
        # the smallest step: one stream, one token, four small heads
        _attention("step_1", 1, 4, 4, 1, 64, 64),
        # one frame of 64 streams: every state is read and written once
        _attention("step_64", 64, 16, 16, 1, 128, 128),
        # a long prompt of one stream
        _attention("prompt_8192", 1, 16, 16, 8192, 128, 128),
        # clips of 12 streams caught up on, each of its own length (none at all among them), keys and values shared by heads
        _attention("clips_12", 12, 6, 2, 1023, 64, 96, dtype="f32", ragged=True),
        # a square projection of a single token
        _product("token_4096", 1, 4096, 4096, 64),
        # the maps of 64 streams of 320x240 embedded: 8 x 60 x 80 values each, as the network hands them over
        _product("embed_64", 64, 256, 38400, 128, dtype="f32", bias=True),
        # 16 streams' tokens against a vocabulary of odd size, small groups
        _product("vocabulary_16", 16, 100003, 2048, 32),
        # behind the attention of 64 streams' tokens: norm for each head and gate
        _norm("heads_64", 64, 2048, group=128, gate="silu"),
        # between two blocks of a long prompt: norm, gate, scale for each channel, float32 residual, next norm
        _norm("blocks_8192", 8192, 4096, gate="sigmoid", residual="f32", next_norm=True, channel_scale=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["log_probs", "attention", "product", "norm"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "log_probs":
        top, labels, masked = rng.choice([0, 1, 3, 5, 8]), rng.random() < 0.8, rng.choice([0.0, 0.0, 0.125, 0.5])
        most = 2047 * 131071 // (2 if dtype == "f32" else 1)
        if rng.random() < 0.5:
            classes, h, w = _log(rng, 8, 256), _log(rng, 8, 180), _log(rng, 8, 320)
            return _log_probs("", "map", max(1, min(_log(rng, 1, 64), most // (classes * h * w))), classes, h, w, dtype, top, labels, masked)
        classes = _log(rng, 50, 131071)
        return _log_probs("", "rows", min(_log(rng, 1, 4096), most // classes), classes, 1, 1, dtype, top, labels, masked)
    if op == "attention":
        dk, dv = rng.choice([32, 48, 64, 64, 96, 128, 128]), rng.choice([32, 64, 64, 80, 96, 128, 128])
        kv = rng.choice([1, 2, 3, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        heads = min(heads, 16) // kv * kv
        if rng.random() < 0.5:
            return _attention("", _log(rng, 1, 64), heads, kv, rng.choice([1, 1, 1, 2, 4, 7]), dk, dv, dtype)
        tokens = _log(rng, 16, 8192)
        most = 16 * 8192 * 8192 // (4 if dtype == "f32" else 1)
        streams = max(1, min(_log(rng, 1, 16), most // (heads * tokens * tokens)))
        if heads * tokens * tokens > most:
            tokens = 4096
        return _attention("", streams, heads, kv, tokens, dk, dv, dtype, streams > 1 and rng.random() < 0.5)
    if op == "product":
        n, m = _log(rng, 64, 100003), _log(rng, 1, 64)
        k = min(_log(rng, 64, 38400), 100003 * 2048 // n)
        most = 16 * 100003 * 2048 // (4 if dtype == "f32" else 1)
        return _product("", max(1, min(m, most // (n * k))), n, k, rng.choice([32, 64, 128]), dtype, rng.random() < 0.3)
    group = rng.choice([0, 0, 64, 96, 128])
    d = group * rng.choice([1, 2, 4, 5, 8, 11, 16, 20, 31]) if group else _log(rng, 128, 8192)
    residual = rng.choice(["", "", dtype, "f32"])
    rows = min(_log(rng, 1, 8192), 8192 * 4096 // (d * (2 if dtype == "f32" else 1)))
    post, gate = rng.random() < 0.8 or bool(group), rng.choice(["", "silu", "sigmoid"])
    return _norm("", rows, d, group, gate, residual, bool(residual) or rng.random() < 0.3, bool(residual) and rng.random() < 0.3, post, dtype)


# ---- inputs -----------------------------------------------------------------------------------
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _quantise(weight, group):
    """Codes [n][k] and scales [n][groups] of a float matrix: the largest value of a group becomes the largest code's."""
    n, k = weight.shape
    groups = -(-k // group)
    w = torch.nn.functional.pad(weight, (0, groups * group - k)).view(n, groups, group)
    scales = (w.abs().amax(-1) / 6).to(torch.bfloat16)
    v = w / scales.float().clamp_min(1e-30)[..., None]
    steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    codes = torch.bucketize(v.abs(), steps).to(torch.uint8) + 8 * (v < 0).to(torch.uint8)
    return codes.view(n, -1)[:, :k].contiguous(), scales


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 29)
    t = _TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=t):
        return (scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)

    s = {"op": case["op"]}
    if case["op"] == "log_probs":
        shape = (case["n"], case["classes"]) + ((case["h"], case["w"]) if case["layout"] == "map" else ())
        s["scores"] = normal(*shape, scale=2.5)
        if case["masked"]:
            out = torch.rand(case["classes"], generator=g, device="cuda") < case["masked"]
            out[0] = False
            s["scores"][:, out] = float("-inf")
        s["top"] = min(case["top"], case["classes"])
        s["labels"] = None
        if case["labels"]:
            s["labels"] = torch.randint(0, case["classes"], shape[:1] + shape[2:], generator=g, device="cuda")
            if case["masked"]:
                s["labels"] = torch.where(out[s["labels"]], 0, s["labels"])
    elif case["op"] == "attention":
        B, H, K, T, dk, dv = (case[x] for x in ("streams", "heads", "kv_heads", "tokens", "dk", "dv"))
        s["q"], s["k"], s["v"] = normal(B, T, H, dk), normal(B, T, K, dk), normal(B, T, K, dv)
        # memories from some tens to some thousands of tokens, head by head
        s["decay"] = [float(torch.tensor(1.0 - 2.0 ** (-5.0 - 5.0 * h / max(1, H - 1)), dtype=torch.float32)) for h in range(H)]
        s["gamma"] = torch.tensor(s["decay"], dtype=torch.float32, device="cuda")
        s["state"] = normal(B, H, dk, dv, dtype=torch.float32)
        s["scale"] = 1.0 / math.sqrt(dk)
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["lengths"][0], s["lengths"][-1] = T, 0
    elif case["op"] == "product":
        n, k = case["n"], case["k"]
        s["codes"], s["scales"] = _quantise(normal(n, k, scale=1.0 / math.sqrt(k), dtype=torch.float32), case["group"])
        s["group"] = case["group"]
        s["bias"] = normal(n, scale=0.1, dtype=torch.float32) if case["bias"] else None
        s["x"] = normal(case["m"], k)
    else:
        rows, d = case["rows"], case["d"]
        s["x"] = normal(rows, d)
        s["weight"] = 1.0 + normal(d, scale=0.1, dtype=torch.float32) if case["post"] else None
        s["group"], s["activation"] = case["group"], case["gate"] or None
        s["gate"] = normal(rows, d) if case["gate"] else None
        s["residual"] = normal(rows, d, scale=4.0, dtype=_TYPES[case["residual"]]) if case["residual"] else None
        s["scale"] = normal(d, scale=0.5, dtype=torch.float32) if case["channel_scale"] else 0.5 if case["residual"] else 1.0
        s["next_weight"] = 1.0 + normal(d, scale=0.1, dtype=torch.float32) if case["next_norm"] else None
    return s


def prepare(case, seed):
    """Inputs on the GPU, and what a program keeps: the layer with its packed weights, the attention with its states."""
    s = _inputs(case, seed)
    if own:
        import paper_1704_04313_amd as cb
        s["cb"] = cb
        if case["op"] == "attention":
            s["attention"] = cb.LinearAttention(s["decay"], case["dk"], case["dv"], n_streams=case["streams"],
                                                kv_heads=case["kv_heads"], scale=s["scale"])
            s["attention"].state.copy_(s["state"])
        elif case["op"] == "product":
            s["layer"] = cb.QuantisedLinear(s["codes"], s["scales"], s["bias"], group=case["group"])
    return s


# ---- one pass ---------------------------------------------------------------------------------
def _plain_log_probs(s):
    x = s["scores"].float().movedim(1, -1)
    C = x.shape[-1]
    d = x - x.amax(-1, keepdim=True)
    e = d.exp()
    total = e.sum(-1)
    log_total = total.log()
    entropy = log_total - (e * d.clamp_min(-200.0)).sum(-1) / total
    label = None
    if s["labels"] is not None:
        label = d.gather(-1, s["labels"][..., None])[..., 0] - log_total
    top = index = None
    if s["top"]:
        # values in order as whole numbers, and behind them the class, so that ties go to the lowest
        bits = (x + 0.0).contiguous().view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        order = order * (1 << 20) + torch.arange((1 << 20) - 1, (1 << 20) - 1 - C, -1, device=x.device)
        index = ((1 << 20) - 1) - (order.topk(s["top"], dim=-1).values & ((1 << 20) - 1))
        top = (d.gather(-1, index) - log_total[..., None]).movedim(-1, 1).contiguous()
        index = index.int().movedim(-1, 1).contiguous()
    return label, entropy, top, index


def _plain_attention(s):
    q, k, v = s["q"].float().transpose(1, 2), s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2)
    share = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)
    T, gamma = q.shape[2], s["gamma"]
    at = torch.arange(T, device=q.device, dtype=torch.float32)
    away = at[:, None] - at[None, :]
    decays = torch.where(away >= 0, gamma[:, None, None] ** away.clamp_min(0), 0.0)
    lengths = s["lengths"].float() if s["lengths"] is not None else torch.full((q.shape[0],), float(T), device=q.device)
    there = (at < lengths[:, None])[:, None, :, None]
    out = (q @ k.transpose(2, 3)).mul_(decays) @ v
    out += (gamma[:, None] ** (at + 1))[None, :, :, None] * (q @ s["state"])
    out = torch.where(there, out * s["scale"], 0.0)
    left = (lengths[:, None] - 1 - at)[:, None, :, None].clamp_min(0)
    faded = torch.where(there, k * gamma[None, :, None, None] ** left, 0.0)
    s["state"].copy_((gamma[None, :] ** lengths[:, None])[..., None, None] * s["state"] + faded.transpose(2, 3) @ v)
    return out.transpose(1, 2).to(s["q"].dtype), s["state"]


def _plain_product(s):
    values = torch.tensor(_E2M1, dtype=torch.float32, device=s["x"].device)
    n, k = s["codes"].shape
    scales = s["scales"].float().repeat_interleave(s["group"], 1)[:, :k]
    y = s["x"].float() @ (values[s["codes"].int()] * scales).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["x"].dtype)


def _plain_norm(s, eps=1e-6):
    x = s["x"].float()
    u = x
    if s["weight"] is not None:
        groups = x.view(x.shape[0], -1, s["group"] or x.shape[1])
        u = (groups * (groups.square().mean(-1, keepdim=True) + eps).rsqrt()).view_as(x) * s["weight"]
    if s["gate"] is not None:
        gate = s["gate"].float()
        open_ = 1.0 / (1.0 + (-gate).exp())
        u = u * (gate * open_ if s["activation"] == "silu" else open_)
    h = s["scale"] * u
    kind = s["x"].dtype
    if s["residual"] is not None:
        h = s["residual"].float() + h
        kind = s["residual"].dtype
    y = None
    if s["next_weight"] is not None:
        y = (h * (h.square().mean(-1, keepdim=True) + eps).rsqrt() * s["next_weight"]).to(s["x"].dtype)
    return h.to(kind), y


def run(state):
    s = state
    if own:
        if s["op"] == "log_probs":
            return s["cb"].log_probs(s["scores"], s["labels"], dim=1, top=s["top"])
        if s["op"] == "attention":
            return s["attention"].process(s["q"], s["k"], s["v"], s["lengths"]), s["attention"].state
        if s["op"] == "product":
            return s["layer"](s["x"])
        return s["cb"].gated_norm(s["x"], s["weight"], group=s["group"], gate=s["gate"], activation=s["activation"],
                                  residual=s["residual"], scale=s["scale"], next_weight=s["next_weight"])
    if s["op"] == "log_probs":
        return _plain_log_probs(s)
    if s["op"] == "attention":
        return _plain_attention(s)
    if s["op"] == "product":
        return _plain_product(s)
    return _plain_norm(s)


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "log_probs":
        positions = case["n"] * case["h"] * case["w"]
        back = 4 + (12 if case["labels"] else 0) + 8 * min(case["top"], case["classes"])
        return {"bytes": positions * (case["classes"] * e + back), "flops": 5.0 * positions * case["classes"]}
    if case["op"] == "attention":
        B, H, K, T, dk, dv = (case[x] for x in ("streams", "heads", "kv_heads", "tokens", "dk", "dv"))
        tokens = B * T if not case["ragged"] else T + (B - 2) * T / 2  # lengths are even over 0 .. T, the first T, the last 0
        return {"bytes": tokens * e * (H * dk + K * (dk + dv)) + B * T * H * dv * e + 8.0 * B * H * dk * dv,
                "flops": 4.0 * tokens * H * dk * dv}
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": n * k / 2 + 2.0 * n * -(-k // case["group"]) + m * (n + k) * e + (4 * n if case["bias"] else 0),
                "flops": 2.0 * m * n * k}
    n, r = case["rows"] * case["d"], 4 if case["residual"] == "f32" else e
    moved = e + (e if case["gate"] else 0) + (2 * r if case["residual"] else e) + (e if case["next_norm"] else 0)
    return {"bytes": n * moved + 4.0 * case["d"] * (case["post"] + case["next_norm"] + case["channel_scale"]), "flops": 12.0 * n}


# ---- the same in 64 bits ----------------------------------------------------------------------
def _exact_log_probs(s):
    scores = s["scores"]
    labels, entropies, tops, indices = [], [], [], []
    for r in range(scores.shape[0]):  # position by position of the first axis: [classes][positions]
        x = scores[r].double().reshape(scores.shape[1], -1)
        every = x - torch.logsumexp(x, 0, keepdim=True)
        p = every.exp()
        entropies.append(-torch.where(p > 0, p * every, torch.zeros_like(p)).sum(0))
        if s["labels"] is not None:
            labels.append(every.gather(0, s["labels"][r].reshape(1, -1))[0])
        if s["top"]:
            found = torch.sort(x, dim=0, descending=True, stable=True).indices[:s["top"]]
            tops.append(every.gather(0, found))
            indices.append(found)
    rest = scores.shape[2:]
    stack = lambda a, *more: torch.stack(a).view(scores.shape[0], *more, *rest)  # noqa: E731
    return (stack(labels) if labels else None, stack(entropies), stack(tops, s["top"]) if tops else None,
            stack(indices, s["top"]) if indices else None)


def _exact_attention(s):
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    B, T, H, _ = q.shape
    of = torch.arange(H, device=q.device) // (H // k.shape[2])
    S = s["state"].double()
    g = s["gamma"].double()[None, :, None, None]
    lengths = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    end = torch.tensor(lengths, device=q.device)
    out = torch.zeros(B, T, H, v.shape[3], dtype=torch.float64, device=q.device)
    for t in range(max(lengths)):  # token after token
        new = g * S + k[:, t, of, :, None] * v[:, t, of, None, :]
        alive = (t < end)[:, None, None, None]
        S = torch.where(alive, new, S)
        out[:, t] = torch.where(alive[..., 0], s["scale"] * (q[:, t, :, :, None] * S).sum(-2), 0.0)
    return out, S


def _exact_product(s):
    n, k = s["codes"].shape
    values = torch.tensor(_E2M1, dtype=torch.float64, device=s["x"].device)
    x, parts = s["x"].double(), []
    for a in range(0, n, 8192):
        w = values[s["codes"][a:a + 8192].long()]
        of = torch.arange(k, device=w.device) // s["group"]
        parts.append(x @ (w * s["scales"][a:a + 8192].double()[:, of]).t())
    y = torch.cat(parts, 1)
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_norm(s, eps=1e-6):
    x = s["x"].double()
    rows, d = x.shape
    u = x.clone()
    if s["weight"] is not None:
        size = s["group"] or d
        for a in range(0, d, size):
            part = x[:, a:a + size]
            u[:, a:a + size] = part / torch.sqrt((part ** 2).sum(1, keepdim=True) / size + eps)
        u = u * s["weight"].double()
    if s["gate"] is not None:
        g = s["gate"].double()
        u = u * torch.sigmoid(g) * (g if s["activation"] == "silu" else 1.0)
    u = u * (s["scale"].double() if isinstance(s["scale"], torch.Tensor) else s["scale"])
    if s["residual"] is not None:
        u = u + s["residual"].double()
    y = None
    if s["next_weight"] is not None:
        y = u / torch.sqrt((u ** 2).sum(1, keepdim=True) / d + eps) * s["next_weight"].double()
    return u, y


def exact(case, seed):
    s = _inputs(case, seed)
    return {"log_probs": _exact_log_probs, "attention": _exact_attention, "product": _exact_product, "norm": _exact_norm}[case["op"]](s)
