"""Norms around a block with its gate and residual scale against 64 bits: every part left out or there, groups, sizes,
strides, types, results in place of inputs."""
import itertools

import pytest
import torch

import paper_1704_04313_amd as cb
from token_util import assert_within, norm64

pytestmark = pytest.mark.gpu
KINDS = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)]
EPS = 1e-6


def _check(h, y, x, what, weight=None, group=0, gate=None, activation=None, residual=None, scale=1.0, next_weight=None, eps=EPS):
    """Norms and gates: a sum over at most 16384 squares, an exponential, a quotient and some products, each a few roundings to
    float32: 2^-20 of every value in all.  y carries what h is off by, twice for the mean, and its own."""
    want_h, want_y, most, factor = norm64(x, weight, group, gate, activation, residual, scale, next_weight, eps)
    off = 2.0 ** -20 * most
    assert_within(h, want_h, off, what + " h")
    if next_weight is None:
        assert y is None
    else:
        assert_within(y, want_y, 2 * factor * off + 2.0 ** -20 * want_y.abs(), what + " y")


def _all(rows, d, kind, sum_kind, seed=0):
    g = torch.Generator().manual_seed(seed + d)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    return {"x": r(rows, d).to(kind).cuda(), "weight": (1 + 0.1 * r(d)).cuda(), "gate": r(rows, d).to(kind).cuda(),
            "residual": (3 * r(rows, d)).to(sum_kind).cuda(), "channel": (0.5 * r(d)).cuda(), "next": (1 + 0.1 * r(d)).cuda()}


@pytest.mark.parametrize("kind,sum_kind", KINDS)
@pytest.mark.parametrize("d", [96, 130])
def test_every_set_of_parts(d, kind, sum_kind):
    t = _all(5, d, kind, sum_kind)
    for post, act, res, chan, nxt in itertools.product((0, 1), (None, "silu", "sigmoid"), (0, 1), (0, 1), (0, 1)):
        kw = dict(weight=t["weight"] if post else None, gate=t["gate"] if act else None, activation=act,
                  residual=t["residual"] if res else None, scale=t["channel"] if chan else 0.75, next_weight=t["next"] if nxt else None)
        _check(*cb.gated_norm(t["x"], **kw), t["x"], "%s" % ((post, act, res, chan, nxt),), **kw)


@pytest.mark.parametrize("kind,sum_kind", KINDS)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (2, 7), (1, 64), (4, 127), (7, 256), (1, 1000), (64, 1024), (3, 2047), (2, 4096),
                                    (5, 4104), (1, 8192), (2, 10001), (1, 16384), (300, 72)])
def test_sizes(rows, d, kind, sum_kind):
    t = _all(rows, d, kind, sum_kind)
    kw = dict(weight=t["weight"], gate=t["gate"], activation="silu", residual=t["residual"], scale=t["channel"], next_weight=t["next"])
    _check(*cb.gated_norm(t["x"], **kw), t["x"], "%dx%d" % (rows, d), **kw)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group,heads", [(64, 16), (128, 16), (96, 5), (1, 40), (7, 9), (33, 31), (256, 3), (512, 2), (1000, 4), (40, 50),
                                         (8, 100), (128, 1), (80, 64), (4096, 4)])
def test_groups(group, heads, kind):
    t = _all(6, group * heads, kind, kind)
    kw = dict(weight=t["weight"], group=group, gate=t["gate"], activation="silu")
    _check(*cb.gated_norm(t["x"], **kw), t["x"], "%d x %d" % (heads, group), **kw)
    kw = dict(weight=t["weight"], group=group, residual=t["residual"], scale=0.5, next_weight=t["next"])
    _check(*cb.gated_norm(t["x"], **kw), t["x"], "%d x %d" % (heads, group), **kw)


@pytest.mark.parametrize("kind,sum_kind", KINDS)
def test_strides(kind, sum_kind):
    for d, at in ((128, 0), (128, 8), (128, 3), (99, 1), (1024, 8), (1024, 2)):
        big = _all(8, 3 * d + 64, kind, sum_kind)
        t = _all(8, d, kind, sum_kind)
        x, gate = big["x"][:, at:at + d], big["x"][:, d + at:2 * d + at]
        kw = dict(weight=t["weight"], gate=gate, activation="sigmoid", residual=big["residual"][:, at:at + d], scale=2.0, next_weight=t["next"])
        _check(*cb.gated_norm(x, **kw), x, "strides", **kw)
        x3, kw3 = x.unflatten(0, (2, 4)), dict(kw, gate=gate.unflatten(0, (2, 4)), residual=kw["residual"].unflatten(0, (2, 4)))
        h, y = cb.gated_norm(x3, **kw3)
        _check(h, y, x3, "three axes", **kw3)


@pytest.mark.parametrize("kind,sum_kind", KINDS)
@pytest.mark.parametrize("d", [512, 515, 9000])
def test_residual_updated_in_place(d, kind, sum_kind):
    t = _all(9, d, kind, sum_kind)
    before = t["residual"].clone()
    kw = dict(weight=t["weight"], gate=t["gate"], activation="silu", scale=0.5, next_weight=t["next"])
    h, y = cb.gated_norm(t["x"], residual=t["residual"], sum_out=t["residual"], **kw)
    assert h is t["residual"]
    _check(h, y, t["x"], "in place", residual=before, **kw)


def test_rows_of_zeros_large_and_small_values():
    t = _all(6, 256, torch.float32, torch.float32)
    x = t["x"]
    x[0] = 0.0
    x[1] *= 1e-12
    x[2] *= 1e15
    kw = dict(weight=t["weight"], next_weight=t["next"])
    _check(*cb.gated_norm(x, **kw), x, "scales", **kw)
    h, y = cb.gated_norm(x[:1], t["weight"], next_weight=t["next"], eps=0.0)
    assert h.isnan().all() and y.isnan().all()  # 0 / 0, as the formula has it


def test_not_finite_stays_in_its_row():
    t = _all(4, 300, torch.bfloat16, torch.float32)
    kw = dict(weight=t["weight"], gate=t["gate"], activation="silu", residual=t["residual"], next_weight=t["next"])
    clean = cb.gated_norm(t["x"], **kw)
    t["x"][1, 7], t["gate"][2, 9] = float("nan"), float("inf")
    got = cb.gated_norm(t["x"], **kw)
    for a, b in zip(got, clean):
        assert torch.equal(a[0], b[0]) and torch.equal(a[3], b[3]) and a[1].isnan().all()
    g = torch.tensor([-200.0, -3e38, 200.0, 3e38, 0.0], device="cuda")
    h, _ = cb.gated_norm(torch.ones(1, 5, device="cuda"), gate=g[None], activation="silu")
    assert torch.equal(h[0, 2:].cpu(), g[2:].cpu()) and bool((h[0, :2].abs() <= 1e-30).all())


def test_nothing_to_do_and_other_streams():
    x = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    h, y = cb.gated_norm(x, torch.ones(64, device="cuda"))
    assert h.shape == (0, 64) and y is None
    t = _all(50, 2048, torch.bfloat16, torch.float32)
    want = cb.gated_norm(t["x"], t["weight"], group=128, residual=t["residual"], next_weight=t["next"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cb.gated_norm(t["x"], t["weight"], group=128, residual=t["residual"], next_weight=t["next"])
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind,sum_kind", KINDS)
@pytest.mark.parametrize("rows,d", [(9, 5), (3000, 513), (5, 519), (2100, 1023), (3, 1025), (2, 2049), (3, 4095), (2, 4097), (2, 8191), (1, 16383)])
def test_rows_that_end_inside_eight(rows, d, kind, sum_kind):
    t = _all(rows, d, kind, sum_kind)
    kw = dict(weight=t["weight"], gate=t["gate"], activation="sigmoid", residual=t["residual"], scale=t["channel"], next_weight=t["next"])
    _check(*cb.gated_norm(t["x"], **kw), t["x"], "%dx%d" % (rows, d), **kw)


@pytest.mark.parametrize("kind,sum_kind", KINDS)
def test_no_rows(kind, sum_kind):
    x, w = torch.empty(0, 24, dtype=kind, device="cuda"), torch.ones(24, device="cuda")
    h, y = cb.gated_norm(x, w, group=8, residual=torch.empty(0, 24, dtype=sum_kind, device="cuda"), next_weight=w)
    assert h.shape == y.shape == (0, 24) and h.dtype == sum_kind and y.dtype == kind


@pytest.mark.parametrize("activation", ["silu", "sigmoid"])
@pytest.mark.parametrize("d", [1000, 1023, 99])
def test_gates_of_any_size(d, activation):
    """The bound of _check holds for every gate: the exponential of a large argument is as exact as that of a small one."""
    t = _all(4, d, torch.float32, torch.float32)
    gate = torch.linspace(-87.0, 87.0, 4 * d).view(4, d).cuda()
    for group in (0, 11) if d == 99 else (0,):
        kw = dict(weight=t["weight"], group=group, gate=gate, activation=activation)
        h, _ = cb.gated_norm(t["x"], **kw)
        want, _, most, _ = norm64(t["x"], residual=None, scale=1.0, next_weight=None, eps=EPS, **kw)
        # some are below the normal numbers: h is the rounding to float32 of a value within the bound
        low, high = (want - 2.0 ** -20 * most).float(), (want + 2.0 ** -20 * most).float()
        assert bool(((h.cpu() >= low) & (h.cpu() <= high)).all())


@pytest.mark.parametrize("activation", ["silu", "sigmoid"])
def test_gates_whose_exponential_is_no_normal_number(activation):
    """From -87.4 on e^g is below the normal numbers: results are off by a step of what float32 has there (2^-149) for each of three
    roundings, times the gate where it multiplies."""
    gate = torch.linspace(-110.0, -87.4, 128).view(2, 64).cuda()
    h, _ = cb.gated_norm(torch.ones(2, 64, device="cuda"), gate=gate, activation=activation)
    g = gate.cpu().double()
    want = 1 / (1 + (-g).exp()) * (g if activation == "silu" else 1.0)
    off = (h.cpu().double() - want).abs()
    assert bool((off <= 2.0 ** -20 * want.abs() + 3 * 2.0 ** -149 * (g.abs() if activation == "silu" else 1.0)).all()), float(off.max())


@pytest.mark.parametrize("activation", ["silu", "sigmoid"])
def test_bfloat16_gates_of_any_size(activation):
    """The same bound with gates of 8 bits and a result of 24."""
    d = 1024
    t = _all(4, d, torch.bfloat16, torch.float32)
    gate = torch.linspace(-86.0, 86.0, 4 * d).view(4, d).to(torch.bfloat16).cuda()
    x, zero = torch.ones(4, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, d, device="cuda")
    kw = dict(weight=t["weight"], gate=gate, activation=activation, residual=zero)
    _check(*cb.gated_norm(x, **kw), x, "gates", **kw)
    for bad, want in ((float("inf"), float("inf") if activation == "silu" else 1.0), (float("nan"), float("nan")),
                      (float("-inf"), float("nan") if activation == "silu" else 0.0)):
        for kind in (torch.bfloat16, torch.float32):
            h, _ = cb.gated_norm(x.to(kind), gate=torch.full_like(x, bad, dtype=kind), activation=activation)
            assert bool((h.float() == want).all() if want == want else h.isnan().all()), (bad, kind)
