"""The token operators in 64 bits on the CPU, written out from their formulas, and how far float32 sums may be
from them."""
import torch

U = 2.0 ** -24  # one rounding to float32, relative
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64)


def assert_within(got, want, allowed, what):
    """float32: |got - want| <= allowed.  bfloat16: got is the rounding of some value that near; rounding is monotonic, so
    it lies between the roundings of the two ends."""
    low, high = want - allowed, want + allowed
    if got.dtype == torch.bfloat16:
        low, high = low.to(torch.bfloat16).double(), high.to(torch.bfloat16).double()
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~same & ~((got >= low) & (got <= high))
    if bad.any():
        i = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError("%s: %d of %d values off; first at %d: got %r, want %r, allowed %r" % (
            what, int(bad.sum()), bad.numel(), i, float(got.reshape(-1)[i]), float(want.reshape(-1)[i]),
            float(torch.as_tensor(allowed).expand(want.shape).reshape(-1)[i])))


def log_probs64(scores, labels, dim, top):
    x = scores.detach().cpu().double().movedim(dim, -1)
    flat = x.reshape(-1, x.shape[-1])
    rows = []
    for r, row in enumerate(flat):
        broken = bool((row.isnan() | (row == float("inf"))).any())
        key = row + 0.0
        order = sorted(range(len(row)), key=lambda c: (0 if row[c].isnan() else 1, -float(key[c]) if not row[c].isnan() else 0.0, c))[:top]
        if broken:
            every, entropy = torch.full_like(row, float("nan")), float("nan")
        elif bool((row == float("-inf")).all()):
            every, entropy = row, 0.0
        else:
            every = row - row.max()
            every = every - every.exp().sum().log()
            p = every.exp()
            entropy = -float(torch.where(p > 0, p * every, torch.zeros_like(p)).sum())
        label = None
        if labels is not None:
            l = int(labels.reshape(-1)[r])
            label = 0.0 if l < 0 else float("nan") if l >= len(row) else float(every[l])
        rows.append((label, entropy, [float(every[c]) for c in order], order))
    rest = x.shape[:-1]
    label = None if labels is None else torch.tensor([r[0] for r in rows], dtype=torch.float64).reshape(rest)
    entropy = torch.tensor([r[1] for r in rows], dtype=torch.float64).reshape(rest)
    at = dim % scores.dim()
    values = torch.tensor([r[2] for r in rows], dtype=torch.float64).reshape(rest + (top,)).movedim(-1, at)
    index = torch.tensor([r[3] for r in rows], dtype=torch.int64).reshape(rest + (top,)).movedim(-1, at)
    return label, entropy, values, index


def check_log_probs(got, scores, labels, dim, top, what=""):
    """A sum of C positive terms in float32 is off by 4 sqrt(C) roundings at the very most (each is at most one rounding of
    the sum, of random sign), each term by its exponential (32 with the argument's rounding); the logarithm keeps this as an
    absolute error, to which the roundings of the value itself come.  The entropy weighs the same errors by itself."""
    label, entropy, values, index = log_probs64(scores, labels, dim, top)
    C = scores.shape[dim]
    base = (32 + 4 * C ** 0.5) * U
    if labels is not None:
        assert_within(got.label, label, base + 4 * U * label.abs().nan_to_num(0, 0, 0), what + " label")
    else:
        assert got.label is None
    assert_within(got.entropy, entropy, base * (2 + entropy.nan_to_num(0)), what + " entropy")
    if top:
        assert torch.equal(got.index.cpu().long(), index), what + " index"
        assert_within(got.top, values, base + 4 * U * values.abs().nan_to_num(0, 0, 0), what + " top")
    else:
        assert got.top is None and got.index is None


def attention64(q, k, v, state, decay, scale, lengths):
    """Output and state, and the same sums over magnitudes, which bound what roundings can do."""
    q, k, v, S = (t.detach().cpu().double() for t in (q, k, v, state))
    B, T, H, dk = q.shape
    share = H // k.shape[2]
    out, out_m = torch.zeros(B, T, H, v.shape[3], dtype=torch.float64), torch.zeros(B, T, H, v.shape[3], dtype=torch.float64)
    S, M = S.clone(), S.abs()
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for h in range(H):
            g = float(torch.tensor(decay[h], dtype=torch.float32))
            for t in range(n):
                kv = torch.outer(k[b, t, h // share], v[b, t, h // share])
                S[b, h] = g * S[b, h] + kv
                M[b, h] = g * M[b, h] + kv.abs()
                out[b, t, h] = scale * (q[b, t, h] @ S[b, h])
                out_m[b, t, h] = abs(scale) * (q[b, t, h].abs() @ M[b, h])
    return out, S, out_m, M


def check_attention(out, state, ref, tokens, dk, dtype, what=""):
    """Sums of products in any order: one rounding a term at most, tokens + key size of them and some for decays and
    scale, of the sum over magnitudes.  bfloat16: operands formed on the way (scores, states) keep 16 bits at least."""
    want, S, out_m, M = ref
    c = (tokens + dk + 32) * U
    assert_within(state, S, c * M, what + " state")
    more = 2.0 ** -15 * out_m if dtype == torch.bfloat16 else 0.0
    assert_within(out, want, c * out_m + more, what + " output")


def weights64(codes, scales, group):
    codes, scales = codes.cpu(), scales.cpu().double()
    cols = codes.shape[1]
    return VALUES[(codes & 15).long()] * scales.repeat_interleave(group, 1)[:, :cols]


def norm64(x, weight, group, gate, activation, residual, scale, next_weight, eps):
    """h, y and the magnitudes that h was added up from."""
    x = x.detach().cpu().double()
    u = x
    if weight is not None:
        parts = x.reshape(*x.shape[:-1], -1, group or x.shape[-1])
        u = (parts / (parts.square().mean(-1, keepdim=True) + eps).sqrt()).reshape(x.shape) * weight.cpu().double()
    if gate is not None:
        g = gate.detach().cpu().double()
        u = u * (1 / (1 + (-g).exp())) * (g if activation == "silu" else 1.0)
    u = u * (scale.cpu().double() if isinstance(scale, torch.Tensor) else float(torch.tensor(scale, dtype=torch.float32)))
    r = torch.zeros_like(u) if residual is None else residual.detach().cpu().double()
    h = r + u
    y = None
    factor = None
    if next_weight is not None:
        factor = next_weight.cpu().double().abs() / (h.square().mean(-1, keepdim=True) + eps).sqrt()
        y = h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * next_weight.cpu().double()
    return h, y, r.abs() + u.abs(), factor
