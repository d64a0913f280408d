"""Answers about camera streams: the change-based network looks at every frame, and a recurrent block with one token per
stream and frame, built from the token operators, remembers and names what is going on.

    frame -> CBInfer -> class maps -> log_probs per position          (what is where, and how sure)
                     -> 4-bit embedding -> token
    token -> norm -> 4-bit q, k, v, gate -> linear attention with decay, state per stream -> norm per head, gate
          -> 4-bit projection, residual, norm -> 4-bit vocabulary -> log_probs   (what is going on)

Weights are random: the example shows the calls, not a trained model.

    python examples/stream_answers.py --streams 4 --frames 20
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1704_04313_amd as cb  # noqa: E402
from workloads import get_config  # noqa: E402


class RecurrentHead:
    """One recurrent block on tokens of `features` values, and a vocabulary behind it.  `weights`: see make_weights."""

    def __init__(self, weights, n_streams: int, heads: int, size: int):
        self.heads, self.size = heads, size
        self.embed = cb.QuantisedLinear.from_weights(weights["embed"], group=128)
        self.qkvg = cb.QuantisedLinear.from_weights(weights["qkvg"], group=64)
        self.out = cb.QuantisedLinear.from_weights(weights["out"], group=64)
        self.vocabulary = cb.QuantisedLinear.from_weights(weights["vocabulary"], group=32)
        self.attention = cb.LinearAttention(weights["decay"], size, size, n_streams=n_streams, scale=size ** -0.5)
        self.norm_in, self.norm_heads, self.norm_out = (weights[n] for n in ("norm_in", "norm_heads", "norm_out"))
        self.block_scale = weights["block_scale"]

    def __call__(self, features, labels=None, top: int = 5) -> cb.LogProbs:
        """features [streams][tokens][features]: one token a stream as the frames come, or a clip at once -- the state is
        the same behind both."""
        x = self.embed(features)
        x, y = cb.gated_norm(x, next_weight=self.norm_in, sum_out=x)
        q, k, v, gate = self.qkvg(y).split(self.heads * self.size, -1)
        q, k, v = (t.unflatten(-1, (self.heads, self.size)) for t in (q, k, v))
        seen = self.attention.process(q, k, v).flatten(2)
        seen, _ = cb.gated_norm(seen, self.norm_heads, group=self.size, gate=gate, activation="silu")
        x, y = cb.gated_norm(self.out(seen), residual=x, scale=self.block_scale, next_weight=self.norm_out, sum_out=x)
        return cb.log_probs(self.vocabulary(y), labels, dim=-1, top=top)

    def reset(self):
        self.attention.reset()


def make_weights(features: int, heads: int, size: int, words: int, seed: int = 0):
    """Random weights of a RecurrentHead, on the GPU."""
    g = torch.Generator().manual_seed(seed)
    wide = heads * size
    matrix = lambda n, k: (torch.randn(n, k, generator=g) / k ** 0.5).cuda()  # noqa: E731
    vector = lambda n: (1 + 0.1 * torch.randn(n, generator=g)).cuda()  # noqa: E731
    return {"embed": matrix(wide, features), "qkvg": matrix(4 * wide, wide), "out": matrix(wide, wide), "vocabulary": 4 * matrix(words, wide),
            "norm_in": vector(wide), "norm_heads": vector(wide), "norm_out": vector(wide), "block_scale": 0.5 * vector(wide),
            "decay": [1.0 - 2.0 ** (-3.0 - h) for h in range(heads)]}


def run(n_streams: int = 4, n_frames: int = 20, height: int = 240, width: int = 320, heads: int = 4, size: int = 64, words: int = 1000, say=print):
    cfg = get_config(5, n_streams=n_streams, height=height, width=width)
    net = cb.CBInfer(cfg.layers, cfg.weights(), (cfg.channels, height, width), cfg.tau, n_streams=n_streams)
    videos = [cfg.video(s) for s in range(n_streams)]
    head = RecurrentHead(make_weights(int(np.prod(net.out_shape[1:])), heads, size, words), n_streams, heads, size)
    answers = []
    for t in range(n_frames):
        maps = net.process_frame(torch.from_numpy(np.stack([v.frame(t) for v in videos])).cuda())
        places = cb.log_probs(maps, dim=1, top=2)
        answer = head(maps.flatten(1)[:, None])
        answers.append((places, answer))
        if t == n_frames - 1:  # the only copy to the host
            for s in range(n_streams):
                say("stream %d, frame %d: words %s (log probabilities %s); mean entropy of the class maps %.3f" % (
                    s, t, answer.index[s, 0].tolist(), ["%.2f" % v for v in answer.top[s, 0].tolist()], float(places.entropy[s].mean())))
    net.destroy()
    return answers


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--streams", type=int, default=4)
    ap.add_argument("--frames", type=int, default=20)
    args = ap.parse_args()
    run(args.streams, args.frames)
