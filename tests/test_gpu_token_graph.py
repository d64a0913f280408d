"""A head's step recorded into a HIP graph: replays on new inputs give what the eager calls give, bit for bit, with other work on
the device in between."""
import pytest
import torch

import paper_1704_04313_amd as cb

pytestmark = pytest.mark.gpu


class Head:
    """Norm, a product with the queries, keys and values of a step, linear attention, a gated norm, scores and their best classes."""

    def __init__(self, streams, size=256, heads=4, classes=5000):
        g = torch.Generator().manual_seed(7)
        self.heads, self.each = heads, size // heads
        self.norm = (1.0 + 0.1 * torch.randn(size, generator=g)).cuda()
        self.inner = torch.ones(size, device="cuda")
        codes, scales = cb.quantise_weights((0.06 * torch.randn(4 * size, size, generator=g)).cuda(), group=64)
        self.project = cb.QuantisedLinear(codes, scales, None, group=64)
        codes, scales = cb.quantise_weights((0.06 * torch.randn(classes, size, generator=g)).cuda(), group=32)
        self.scores = cb.QuantisedLinear(codes, scales, torch.randn(classes, generator=g).cuda(), group=32)
        self.attention = cb.LinearAttention(torch.linspace(0.9, 0.999, heads).cuda(), self.each, self.each, n_streams=streams)

    def __call__(self, x, labels):
        h, _ = cb.gated_norm(x, self.norm)
        *qkv, gate = self.project(h).chunk(4, dim=-1)
        o = self.attention.process(*(t.unflatten(-1, (self.heads, self.each)) for t in qkv))
        y, _ = cb.gated_norm(o.flatten(-2), self.inner, group=self.each, gate=gate, activation="silu")
        return cb.log_probs(self.scores(y).flatten(0, 1), labels, dim=1, top=5)


@pytest.mark.parametrize("dtype,streams,tokens", [(torch.bfloat16, 3, 1), (torch.float32, 2, 1), (torch.bfloat16, 2, 300)])
def test_replays_give_the_eager_results(dtype, streams, tokens):
    eager, graphed = Head(streams), Head(streams)
    x = torch.zeros(streams, tokens, 256, dtype=dtype, device="cuda")
    labels = torch.zeros(streams * tokens, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed(x, labels)
    torch.cuda.current_stream().wait_stream(side)
    graphed.attention.reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = graphed(x, labels)
    graphed.attention.reset()

    g = torch.Generator().manual_seed(11)
    for turn in range(5):
        new = torch.randn(streams, tokens, 256, generator=g).to(dtype).cuda()
        wanted = torch.randint(0, 5000, (streams * tokens,), generator=g).cuda()
        x.copy_(new)
        labels.copy_(wanted)
        graph.replay()
        expect = eager(new, wanted)  # the program's own work between the replays
        if turn % 2:
            torch.cuda.synchronize()
        for a, b in zip(out, expect):
            assert torch.equal(a, b)
        assert torch.equal(graphed.attention.state, eager.attention.state)
