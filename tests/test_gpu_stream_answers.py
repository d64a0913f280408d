"""The token operators run together as examples/stream_answers.py uses them: against the same block in 64 bits, and frame by
frame against whole clips."""
import importlib.util
import os

import pytest
import torch

import paper_1704_04313_amd as cb
from token_util import attention64, norm64, weights64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("stream_answers", os.path.join(ROOT, "examples", "stream_answers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _block64(w, x, heads, size):
    """Log probabilities of every word: the formulas one after the other, with the quantised weights."""
    def product(v, name, group):
        return v @ weights64(*cb.quantise_weights(w[name], group), group).t()
    x = product(x.cpu().double(), "embed", 128)
    _, y, _, _ = norm64(x, None, 0, None, None, None, 1.0, w["norm_in"], 1e-6)
    q, k, v, gate = product(y, "qkvg", 64).split(heads * size, -1)
    q, k, v = (t.unflatten(-1, (heads, size)) for t in (q, k, v))
    B = x.shape[0]
    seen, _, _, _ = attention64(q, k, v, torch.zeros(B, heads, size, size), w["decay"], size ** -0.5, None)
    seen, _, _, _ = norm64(seen.flatten(2), w["norm_heads"], size, gate, "silu", None, 1.0, None, 1e-6)
    _, y, _, _ = norm64(product(seen, "out", 64), None, 0, None, None, x, w["block_scale"], w["norm_out"], 1e-6)
    return torch.log_softmax(product(y, "vocabulary", 32), -1)


@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_block_against_64_bits(tokens):
    ex = _example()
    heads, size, words, features, B = 3, 32, 333, 700, 2
    w = ex.make_weights(features, heads, size, words, seed=3)
    x = torch.randn(B, tokens, features, generator=torch.Generator().manual_seed(1)).cuda()
    labels = torch.randint(0, words, (B, tokens), generator=torch.Generator().manual_seed(2)).cuda()
    got = ex.RecurrentHead(w, B, heads, size)(x, labels, top=4)
    want = _block64(w, x, heads, size)
    # nine operators in float32, each to a few millionths of its values, which the last product spreads over scores of some tens
    tol = dict(rtol=0, atol=2e-4)
    torch.testing.assert_close(got.label.cpu().double(), want.gather(-1, labels.cpu()[..., None])[..., 0], **tol)
    torch.testing.assert_close(got.top.cpu().double(), want.topk(4).values, **tol)
    torch.testing.assert_close(got.entropy.cpu().double(), -(want.exp() * want).sum(-1), **tol)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_frame_by_frame_and_clip_at_once(kind):
    ex = _example()
    heads, size, B, T = 4, 64, 3, 70
    w = ex.make_weights(500, heads, size, 200, seed=5)
    x = torch.randn(B, T, 500, generator=torch.Generator().manual_seed(4)).to(kind).cuda()
    head = ex.RecurrentHead(w, B, heads, size)
    clip = head(x)
    after = head.attention.state.clone()
    head.reset()
    for t in range(T):
        step = head(x[:, t:t + 1])
        torch.testing.assert_close(step.entropy[:, 0], clip.entropy[:, t], rtol=0, atol=2e-4 if kind == torch.float32 else 0.2)
    # bfloat16 rounds every operator's output: two ways of summing differ by some of its steps (2^-8)
    torch.testing.assert_close(head.attention.state, after, rtol=0, atol=1e-3 if kind == torch.float32 else 0.5)


def test_example_runs():
    said = []
    answers = _example().run(n_streams=2, n_frames=4, height=48, width=64, say=said.append)
    assert len(said) == 2 and len(answers) == 4
    for places, answer in answers:
        assert places.top.shape == (2, 2, 12, 16) and answer.index.shape == (2, 1, 5)
        assert bool((answer.top <= 0).all()) and bool((places.entropy >= 0).all())


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_frame_by_frame_and_a_short_clip(kind):
    """Up to 16 tokens a call the block's products give a token the same bits alone and in a clip, so queries, keys and values are the same,
    and the states differ by the roundings of their sums alone."""
    ex = _example()
    heads, size, B, T = 4, 64, 3, 5
    w = ex.make_weights(500, heads, size, 200, seed=5)
    x = torch.randn(B, T, 500, generator=torch.Generator().manual_seed(4)).to(kind).cuda()
    head = ex.RecurrentHead(w, B, heads, size)
    seen, process = [], head.attention.process
    head.attention.process = lambda q, k, v: (seen.append((q, k, v)), process(q, k, v))[1]
    head(x)
    after = head.attention.state.clone()
    head.reset()
    for t in range(T):
        head(x[:, t:t + 1])
        for a, b in zip(seen[0], seen[-1]):
            assert torch.equal(a[:, t:t + 1], b)
    _, S, _, M = attention64(*seen[0], torch.zeros(B, heads, size, size), w["decay"], size ** -0.5, None)
    for state in (after, head.attention.state):
        assert bool(((state.cpu().double() - S).abs() <= (T + size + 32) * 2.0 ** -24 * M).all())
