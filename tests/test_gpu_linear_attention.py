"""Linear attention with a decay for each head against the recurrence in 64 bits: sizes of heads, lengths from none to
several hundred, shared heads, strides, decays from 0 to 1."""
import pytest
import torch

import paper_1704_04313_amd as cb
from token_util import attention64, check_attention

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


def _run(B, T, H, K, dk, dv, dtype, *, lengths=None, decay=None, seed=0, scale=0.3, what="", change=None, fused=False):
    g = torch.Generator().manual_seed(seed + T + 31 * dk + dv)
    decay = decay or [1.0 - 2.0 ** -(1.5 + 6.0 * h / max(1, H - 1)) for h in range(H)]
    if fused:  # parts of one wider tensor, as a projection hands them over
        wide = torch.randn(B, T + 1, H * dk + K * (dk + dv) + 3, generator=g).to(dtype).cuda()[:, 1:, 1:]
        q, k, v = wide[..., :H * dk], wide[..., H * dk:(H + K) * dk], wide[..., (H + K) * dk:(H + K) * dk + K * dv]
        q, k, v = q.unflatten(2, (H, dk)), k.unflatten(2, (K, dk)), v.unflatten(2, (K, dv))
    else:
        q, k, v = (torch.randn(B, T, n, d, generator=g).to(dtype).cuda() for n, d in ((H, dk), (K, dk), (K, dv)))
    if change:
        change(q, k, v)
    att = cb.LinearAttention(decay, dk, dv, n_streams=B, kv_heads=K, scale=scale)
    start = torch.randn(B, H, dk, dv, generator=g)
    att.state.copy_(start)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    out = att.process(q, k, v, n)
    check_attention(out, att.state, attention64(q, k, v, start, decay, scale, lengths), T, dk, dtype, what)
    return att, out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (1, 1), (3, 5), (16, 256), (256, 16), (48, 80), (33, 96), (128, 100), (200, 36), (256, 256)])
def test_single_tokens(dk, dv, dtype):
    for B, H, K in ((1, 1, 1), (3, 4, 2)):
        _run(B, 1, H, K, dk, dv, dtype, what="step %d %d" % (dk, dv))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [2, 3, 7, 15, 16, 17, 31, 33, 63, 64, 65, 100, 128, 129, 200])
def test_lengths(T, dtype):
    _run(1, T, 2, 1, 64, 64, dtype, what="T %d" % T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dk,dv", [(128, 128), (32, 32), (48, 80), (96, 64), (33, 31), (8, 200), (256, 64), (130, 256), (64, 1), (1, 64)])
def test_prompts_of_any_head_size(dk, dv, dtype):
    _run(2, 150, 2, 2, dk, dv, dtype, what="%d %d" % (dk, dv))


@pytest.mark.parametrize("dtype", TYPES)
def test_long_prompts(dtype):
    _run(1, 700, 2, 1, 64, 64, dtype, what="long")
    _run(1, 1023, 1, 1, 128, 96, dtype, what="long")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [5, 130, 400])
def test_ragged(T, dtype):
    lengths = [T, 0, 1, T // 2, T + 9, -3, T - 1]
    _run(7, T, 3, 1, 64, 48, dtype, lengths=lengths, what="ragged")


@pytest.mark.parametrize("T", [4, 150])
@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_beyond_a_length_is_read(T, dtype):
    def spoil(q, k, v):
        q[1, 2:], k[1, 2:], v[1, 2:] = float("nan"), float("inf"), float("nan")
    _, out = _run(3, T, 2, 2, 64, 64, dtype, lengths=[T, 2, T], change=spoil)
    assert not out[1, 2:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [4, 150])
def test_no_token_sees_a_later_one(T, dtype):
    """What is not finite in a later token leaves earlier outputs alone."""
    for at, bad in ((T - 1, float("nan")), (T - 2, float("inf"))):
        def spoil(q, k, v):
            v[0, at, 0, 3] = bad
            k[0, at, 0, 5] = bad
        g = torch.Generator().manual_seed(1)
        q, k, v = (torch.randn(1, T, 1, 32, generator=g).to(dtype).cuda() for _ in range(3))
        clean = cb.LinearAttention([0.9], 32, 32).process(q, k, v)
        spoil(q, k, v)
        got = cb.LinearAttention([0.9], 32, 32).process(q, k, v)
        torch.testing.assert_close(got[:, :at], clean[:, :at], rtol=2.0 ** -7 if dtype == torch.bfloat16 else 1e-5, atol=1e-3)
        assert not got[0, at].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 3, 100, 300])
def test_decays_at_both_ends(T, dtype):
    _run(1, T, 4, 2, 32, 32, dtype, decay=[0.0, 1.0, 1e-30, 0.5], what="decays")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 6, 140])
def test_strided_inputs(T, dtype):
    _run(2, T, 4, 2, 40, 24, dtype, fused=True, what="fused")
    _run(2, T, 2, 1, 64, 64, dtype, fused=True, what="fused")


@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_and_steps_agree(dtype):
    """A prompt in one call, in pieces, and token by token: one recurrence."""
    g = torch.Generator().manual_seed(4)
    T, d = 150, 64
    q, k, v = (torch.randn(2, T, 3, d, generator=g).to(dtype).cuda() for _ in range(3))
    decay = [0.99, 0.9, 0.5]
    ref = attention64(q, k, v, torch.zeros(2, 3, d, d), decay, 0.125, None)
    for cuts in ([0, T], [0, 64, T], [0, 1, 90, 91, T], list(range(T + 1))):
        att = cb.LinearAttention(decay, d, d, n_streams=2, scale=0.125)
        out = torch.cat([att.process(q[:, a:b], k[:, a:b], v[:, a:b]) for a, b in zip(cuts, cuts[1:])], 1)
        check_attention(out, att.state, ref, T, d, dtype, "cuts %s" % len(cuts))
    att.reset()
    assert not att.state.any()


def test_same_bits_every_time_and_on_another_stream():
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(1, 900, 4, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    runs = []
    side = torch.cuda.Stream()
    for s in (torch.cuda.current_stream(), side, side):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            att = cb.LinearAttention([0.999, 0.99, 0.9, 1.0], 128, 128)
            runs.append((att.process(q, k, v), att.state))
        torch.cuda.synchronize()
    for o, s in runs[1:]:
        assert torch.equal(o, runs[0][0]) and torch.equal(s, runs[0][1])


def test_output_given_and_no_tokens():
    att = cb.LinearAttention([0.9] * 2, 32, 32, n_streams=2)
    att.state.fill_(3.0)
    q = torch.randn(2, 0, 2, 32, device="cuda")
    assert att.process(q, q, q).shape == (2, 0, 2, 32) and bool((att.state == 3.0).all())
    wide = torch.full((2, 80, 2, 40), 7.0, device="cuda")
    q = torch.randn(2, 80, 2, 32, device="cuda")
    out = att.process(q, q, q, out=wide[..., :32])
    assert out.data_ptr() == wide.data_ptr() and bool((wide[..., 32:] == 7.0).all())
    att.reset()
    torch.testing.assert_close(att.process(q, q, q), cb.LinearAttention([0.9] * 2, 32, 32, n_streams=2).process(q, q, q), rtol=0, atol=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dk,dv", [(129, 33), (192, 64), (256, 128), (200, 130)])
def test_prompts_with_long_keys(dk, dv, dtype):
    _run(1, 400, 3, 1, dk, dv, dtype, what="long keys")
    _run(4, 300, 2, 2, dk, dv, dtype, lengths=[300, 0, 64, 131], what="long keys, ragged")


@pytest.mark.parametrize("dtype", TYPES)
def test_more_parts_than_an_output_joins(dtype):
    _run(1, 1500, 1, 1, 64, 48, dtype, what="many parts")
    _run(2, 1300, 1, 1, 160, 32, dtype, lengths=[1300, 700], what="many parts, ragged")
    _run(3, 1100, 1, 1, 32, 32, dtype, lengths=[64, 65, 1088], what="a chunk, and one token more")


def _integers(T, d, seed, wide):
    """Whole numbers whose sums of products stay below 2^24, so that they are exact in float32 in any order, although they cancel: what is
    added up has far more bits than the result.  `wide` "scores": queries and keys of 8 bits, keys of neighbours opposite but for one
    place, values +-1.  "state": entries of 18 bits, neighbours opposite but for their last bits."""
    g = torch.Generator().manual_seed(seed)
    whole = lambda m, *s: torch.randint(-m, m + 1, s, generator=g).float()  # noqa: E731
    state = torch.zeros(1, 1, d, d)
    if wide == "scores":
        q, k, v = whole(255, 1, T, 1, d), whole(127, 1, T, 1, d), 2 * torch.randint(0, 2, (1, T, 1, d), generator=g).float() - 1
        k[:, 1::2] = -k[:, :T // 2 * 2:2]
        k[:, 1::2, :, 3] += 1
        v[:, 1::2] = v[:, :T // 2 * 2:2]
    else:
        q, k, v = whole(1, 1, T, 1, d), torch.zeros(1, T, 1, d), torch.zeros(1, T, 1, d)
        q[..., 1::2] = q[..., ::2]
        state[:, :, ::2] = whole(2 ** 18 - 8, 1, 1, d // 2, d)
        state[:, :, 1::2] = whole(3, 1, 1, d // 2, d) - state[:, :, ::2]
    return q, k, v, state


@pytest.mark.parametrize("wide", ["scores", "state"])
@pytest.mark.parametrize("T,d", [(1, 64), (5, 64), (15, 128), (64, 32), (150, 64), (150, 128), (90, 256)])
def test_scores_and_states_keep_24_bits(T, d, wide):
    q, k, v, state = _integers(T, d, T + d, wide)
    att = cb.LinearAttention([1.0], d, d)
    att.state.copy_(state)
    want, S, _, _ = attention64(q, k, v, state, [1.0], 1.0, None)
    out = att.process(*(t.bfloat16().cuda() for t in (q, k, v)))
    assert torch.equal(att.state.cpu().double(), S)
    assert torch.equal(out.cpu(), want.to(torch.bfloat16))


def _some_heads(out, state, q, k, v, start, decay, scale, lengths, dtype, what, until=None):
    """A sample of a larger call's streams and heads against 64 bits; until: outputs alone, of the tokens in front."""
    B, T, H, dk = q.shape
    share = H // k.shape[2]
    for b, h in ((0, 0), (B - 1, H - 1), (B // 2, 1), (1, H // 2)):
        s, g = slice(b, b + 1), slice(h, h + 1)
        kv = slice(h // share, h // share + 1)
        n = None if lengths is None else [lengths[b]]
        ref = attention64(q[s, :until, g], k[s, :until, kv], v[s, :until, kv], start[s, g], decay[g], scale, n)
        if until is None:
            check_attention(out[s, :, g], state[s, g], ref, T, dk, dtype, "%s, stream %d, head %d" % (what, b, h))
        else:
            check_attention(out[s, :until, g], ref[1], ref, T, dk, dtype, "%s, stream %d, head %d" % (what, b, h))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dk,dv", [(64, 96), (64, 100), (128, 128), (128, 100), (40, 128)])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("aligned", [True, False])
def test_enough_heads_to_fill_the_chip(aligned, ragged, dk, dv, dtype):
    """Streams and heads enough for workgroups of 128 columns."""
    B, T, H, K = 8, 300, 8, 4
    g = torch.Generator().manual_seed(dk + dv)
    r = lambda n, d: torch.randn(B, T, n, d + 3, generator=g).to(dtype).cuda()  # noqa: E731
    q, k, v = (t[..., :-3].contiguous() if aligned else t[..., 1:-2] for t in (r(H, dk), r(K, dk), r(K, dv)))
    decay = [1.0 - 2.0 ** -(1.0 + h) for h in range(H)]
    start = torch.randn(B, H, dk, dv, generator=g)
    lengths = [300, 0, 1, 64, 65, 299, 128, 257] if ragged else None
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    att = cb.LinearAttention(decay, dk, dv, n_streams=B, kv_heads=K, scale=0.3)
    att.state.copy_(start)
    out = att.process(q, k, v, n)
    _some_heads(out, att.state, q, k, v, start, decay, 0.3, lengths, dtype, "filled")
    if ragged:
        for b, length in enumerate(lengths):
            assert not out[b, length:].any()
        assert torch.equal(att.state[1].cpu(), start[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dk,dv", [(64, 96), (128, 128), (128, 100)])
def test_not_finite_among_heads_that_fill_the_chip(dk, dv, dtype):
    """A later token that is not finite, in every stream: the outputs in front of it, in its own 64 tokens too, are as they were."""
    B, T, H, at = 8, 300, 8, 290
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(B, T, H, d, generator=g).to(dtype).cuda() for d in (dk, dk, dv))
    v[:, at, :, 5], v[:, at, :, dv - 1] = float("nan"), float("inf")
    decay = [0.9] * H
    att = cb.LinearAttention(decay, dk, dv, n_streams=B, scale=0.3)
    out = att.process(q, k, v)
    _some_heads(out, None, q, k, v, torch.zeros(B, H, dk, dv), decay, 0.3, None, dtype, "in front", until=at)
    assert not out[:, at:, :, 5].isfinite().any() and not out[:, at:, :, dv - 1].isfinite().any()
    rest = [c for c in range(dv) if c not in (5, dv - 1)]
    assert out[..., rest].isfinite().all() and att.state[..., rest].isfinite().all()


@pytest.mark.parametrize("wide", ["scores", "state"])
def test_24_bits_with_heads_that_fill_the_chip(wide):
    T, d = 300, 128
    q, k, v, state = _integers(T, d, 11, wide)
    att = cb.LinearAttention([1.0] * 8, d, d, n_streams=8)
    att.state.copy_(state)
    want, S, _, _ = attention64(q, k, v, state, [1.0], 1.0, None)
    out = att.process(*(t.bfloat16().cuda().expand(8, T, 8, d).contiguous() for t in (q, k, v)))
    assert bool((att.state.cpu().double() == S).all())
    assert bool((out.cpu() == want.to(torch.bfloat16)).all())
