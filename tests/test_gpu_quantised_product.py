"""Products with 4-bit weights against 64 bits: every code, sizes that end inside a group, a block and a tile, strides,
values that are not finite."""
import threading

import pytest
import torch

import paper_1704_04313_amd as cb
from token_util import U, VALUES, assert_within, weights64

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


def _layer(n, k, group, seed, bias=True):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    scales = (0.02 + torch.rand(n, -(-k // group), generator=g)).to(torch.bfloat16)
    b = torch.randn(n, generator=g) if bias else None
    return codes, scales, b, cb.QuantisedLinear(codes.cuda(), scales.cuda(), None if b is None else b.cuda(), group=group)


def _check(y, x, codes, scales, bias, group, what):
    """A sum of k products in float32, in any order: 4 sqrt(k) roundings of the sum over magnitudes at the very most, some for
    scales and bias."""
    w, x64 = weights64(codes, scales, group), x.detach().cpu().double()
    want, most = x64 @ w.t(), x64.abs() @ w.abs().t()
    if bias is not None:
        want, most = want + bias.double(), most + bias.double().abs()
    assert_within(y, want, (32 + 4 * w.shape[1] ** 0.5) * U * most, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k,group", [(1, 1, 1, 32), (1, 16, 128, 32), (1, 17, 129, 64), (2, 100, 300, 128), (3, 64, 1000, 32),
                                         (5, 33, 31, 64), (7, 256, 4096, 64), (16, 48, 640, 128), (17, 80, 100, 32), (33, 500, 256, 64),
                                         (64, 96, 2000, 128), (65, 40, 160, 32), (100, 16, 5000, 64), (130, 200, 136, 128), (1, 2999, 512, 32),
                                         (64, 256, 9600, 128), (12, 20, 20000, 64)])
def test_sizes(m, n, k, group, dtype):
    codes, scales, bias, layer = _layer(n, k, group, m + n + k, bias=n % 2 == 0)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    _check(layer(x), x, codes, scales, bias, group, "%dx%dx%d" % (m, n, k))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_code_in_every_place(group, dtype):
    """One token at a time picks one column: the weights themselves come back, exactly."""
    n, k = 40, 300
    codes, scales, _, layer = _layer(n, k, group, 3, bias=False)
    y = layer(torch.eye(k, dtype=dtype, device="cuda"))
    w = weights64(codes, scales, group)
    assert torch.equal(y.cpu().double(), w.t().to(dtype).double())


@pytest.mark.parametrize("m", [1, 4, 20, 64])
def test_integers_exactly(m):
    n, k, group = 200, 2500, 64
    g = torch.Generator().manual_seed(8)
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    scales = torch.tensor([2.0, 4.0, 8.0])[torch.randint(0, 3, (n, -(-k // group)), generator=g)].to(torch.bfloat16)
    x = torch.randint(-6, 7, (m, k), generator=g).float()
    y = cb.QuantisedLinear(codes.cuda(), scales.cuda(), group=group)(x.cuda())
    assert torch.equal(y.cpu().double(), x.double() @ weights64(codes, scales, group).t())


def test_float32_values_keep_24_bits():
    """x of 24 bits times powers of two: nothing is lost when x is taken apart."""
    k = 64
    codes = torch.full((16, k), 2, dtype=torch.uint8)
    scales = torch.ones(16, 1, dtype=torch.bfloat16)
    layer = cb.QuantisedLinear(codes.cuda(), scales.cuda(), group=64)
    x = torch.zeros(6, k)
    x[:, 7] = torch.tensor([1 + 2.0 ** -23, 3.4028234e38, -1.1754944e-27, 16777215.0, 0.1, -1e30])
    assert torch.equal(layer(x.cuda()).cpu(), x[:, 7:8].expand(6, 16))


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite(dtype):
    codes, scales, _, layer = _layer(32, 200, 64, 5, bias=False)
    x = torch.randn(5, 200, generator=torch.Generator().manual_seed(2)).to(dtype)
    x[0, 3], x[1, 150], x[2, 199], x[3, 0] = float("inf"), float("nan"), float("-inf"), float("inf")
    x[3, 1] = float("-inf")
    want = x.double() @ weights64(codes, scales, 64).t()
    got = layer(x.cuda()).cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[got.isinf()], want[want.isinf()])
    assert torch.equal(got.isinf(), want.isinf()) and got[4].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_shapes(dtype):
    codes, scales, bias, layer = _layer(70, 260, 64, 6)
    wide = torch.randn(3, 5, 700, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    for at in (0, 1, 4, 8):
        x = wide[..., at:at + 260]
        _check(layer(x).view(15, 70), x.reshape(15, 260), codes, scales, bias, 64, "part from %d" % at)
    x = wide[0, 0, 3:263]
    assert layer(x).shape == (70,)
    _check(layer(x)[None], x[None], codes, scales, bias, 64, "vector")
    out = torch.empty(15, 70, dtype=dtype, device="cuda")
    assert layer(wide.view(15, 700)[:, :260], out=out) is out
    _check(out, wide.view(15, 700)[:, :260], codes, scales, bias, 64, "out")
    assert layer(wide[:0, :, :260]).shape == (0, 5, 70)


def test_same_bits_alone_and_among_others():
    """A token's result does not depend on the tokens beside it in its tile, nor on the stream."""
    _, _, _, layer = _layer(300, 1500, 32, 9)
    x = torch.randn(16, 1500, generator=torch.Generator().manual_seed(5)).cuda()
    y = layer(x)
    assert torch.equal(y, layer(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = layer(x)
    side.synchronize()
    assert torch.equal(y, z)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantising(group, dtype):
    g = torch.Generator().manual_seed(10)
    w = torch.randn(37, 333, generator=g).to(dtype)
    w[3] = 0.0
    w[4, :40] *= 1e-3
    codes, scales = (t.cpu() for t in cb.quantise_weights(w.cuda(), group))
    w64 = w.double()
    for n in range(37):
        for a in range(0, 333, group):
            part, s = w64[n, a:a + group], float(scales[n, a // group])
            assert s == float((part.abs().max().float() / 6).to(torch.bfloat16))
            c = codes[n, a:a + group].long()
            if s == 0:
                assert not c.any()
                continue
            near = ((part / s)[:, None] - VALUES[None, :]).abs()
            # the quotient is rounded to float32 before it is compared: at most that far from the nearest
            assert bool((near.gather(1, c[:, None])[:, 0] <= near.min(1).values + 8 * U).all())
    layer = cb.QuantisedLinear.from_weights(w.cuda(), group=group)
    x = torch.randn(3, 333, generator=g).to(dtype).cuda()
    _check(layer(x), x, codes, scales, None, group, "from weights")


def test_ties_take_the_even_code():
    w = torch.zeros(1, 32)
    w[0, :16] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0])
    codes, scales = cb.quantise_weights(w.cuda(), 32)
    assert float(scales) == 1.0
    assert codes[0, :16].tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 0, 10, 10, 12, 12, 14, 14, 15]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k,group", [(20, 16400, 2100, 64), (40, 16401, 140, 32), (24, 1030, 2900, 128), (50, 1500, 900, 64)])
def test_many_rows(m, n, k, group, dtype):
    codes, scales, bias, layer = _layer(n, k, group, m + n)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    _check(layer(x), x, codes, scales, bias, group, "%dx%dx%d" % (m, n, k))


@pytest.mark.parametrize("dtype", TYPES)
def test_as_many_tokens_and_as_long_a_row_as_there_may_be(dtype):
    codes, scales, bias, layer = _layer(3, 2, 32, 5)
    x = torch.randn(1 << 19, 2, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    _check(layer(x), x, codes, scales, bias, 32, "2^19 tokens")
    codes = torch.full((1, 1 << 25), 2, dtype=torch.uint8, device="cuda")  # ones
    layer = cb.QuantisedLinear(codes, torch.ones(1, 1 << 18, dtype=torch.bfloat16, device="cuda"), group=128)
    x = torch.zeros(1, 1 << 25, dtype=dtype, device="cuda")
    for at, value in ((0, 1.0), (1023, 2.0), (1024, 4.0), ((1 << 24) + 1, 8.0), ((1 << 25) - 1, 16.0)):
        x[0, at] = value
    assert layer(x).item() == 31.0


@pytest.mark.parametrize("m", [33, 48, 49, 64, 70])
@pytest.mark.parametrize("k,group", [(1300, 64), (2048, 32), (2500, 128)])
def test_many_rows_and_tokens(m, k, group):
    codes, scales, bias, layer = _layer(16390, k, group, m + k)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    _check(layer(x), x, codes, scales, bias, group, "%dx16390x%d" % (m, k))


@pytest.mark.parametrize("dtype", TYPES)
def test_no_tokens(dtype):
    layer = _layer(40, 70, 32, 1)[3]
    assert layer(torch.empty(0, 70, dtype=dtype, device="cuda")).shape == (0, 40)
    assert layer(torch.empty(2, 0, 3, 70, dtype=dtype, device="cuda")).shape == (2, 0, 3, 40)


def test_a_layer_used_by_two_threads():
    """Each with its own tokens, on its own stream, at the same time: what each gets alone."""
    layer = _layer(300, 9000, 64, 9)[3]
    work = [torch.randn(m, 9000, generator=torch.Generator().manual_seed(m)).to(t).cuda() for m, t in ((3, torch.float32), (70, torch.bfloat16))]
    alone = [layer(x) for x in work]
    torch.cuda.synchronize()
    got = [[], []]

    def call(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(200):
                got[i].append(layer(work[i]))
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=call, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in (0, 1):
        assert len(got[i]) == 200 and all(torch.equal(y, alone[i]) for y in got[i])


def test_every_nan_stays_a_nan():
    """float32 NaN whatever its bits: those that are told from infinity by their last bits too."""
    layer = _layer(32, 200, 64, 5, bias=False)[3]
    bits = torch.tensor([0x7f800001, 0x7f80ffff, 0x7fc00000, 0x7fffffff, 0x7f810000], dtype=torch.int64)
    bits = torch.cat([bits, bits | 0x80000000])
    x = torch.randn(20, 200, generator=torch.Generator().manual_seed(2))
    x.view(torch.int32)[torch.arange(10), 13 * torch.arange(10)] = bits.to(torch.int32)
    got = layer(x.cuda()).cpu()
    assert bool(got[:10].isnan().all()) and bool(got[10:].isfinite().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 16, 33, 64])
@pytest.mark.parametrize("n,k", [(40, 1200), (40, 600), (16400, 1200), (600, 4500)])
def test_infinite_scales(m, n, k, dtype):
    """A scale that is infinite makes its row's results infinite: no column that is not there turns them into NaN."""
    g = torch.Generator().manual_seed(m + n)
    codes = torch.randint(1, 8, (n, k), generator=g, dtype=torch.uint8)
    scales = (0.02 + torch.rand(n, -(-k // 64), generator=g)).to(torch.bfloat16)
    scales[3, -1], scales[5, 0] = float("inf"), float("inf")
    x = (0.1 + torch.rand(m, k, generator=g)).to(dtype)
    got = cb.QuantisedLinear(codes.cuda(), scales.cuda(), group=64)(x.cuda()).cpu()
    want = torch.zeros(n, dtype=torch.bool)
    want[3] = want[5] = True
    assert bool((got[:, want] == float("inf")).all()) and bool(got[:, ~want].isfinite().all())


@pytest.mark.parametrize("rows,cols", [(1 << 16, 1 << 16), (66000000, 65)])
def test_quantising_as_many_weights_as_there_may_be(rows, cols):
    """Groups of 32 that need more threads than a launch has: the first rows, the last, some in the middle."""
    few = torch.randn(512, cols, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    places = [0, rows // 3, 2 * rows // 3, rows - 512]
    w = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    for at in places:
        w[at:at + 512] = few
    want = cb.quantise_weights(few, 32)
    codes, scales = cb.quantise_weights(w, 32)
    for at in places:
        assert torch.equal(codes[at:at + 512], want[0]) and torch.equal(scales[at:at + 512], want[1]), at


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k", [(300, 1500), (500, 300), (70, 20000)])
@pytest.mark.parametrize("few,many", [(1, 16), (18, 32)])
def test_a_token_alone_and_among_others(few, many, n, k, dtype):
    """For 1 .. 16 tokens, and for 17 .. 32, a token's result has the same bits whatever tokens are beside it, and however many."""
    layer = _layer(n, k, 32, 9)[3]
    g = torch.Generator().manual_seed(5)
    x = torch.randn(many, k, generator=g).to(dtype).cuda()
    y = layer(x)
    assert torch.equal(layer(x[:few]), y[:few])
    z = x.clone()
    z[few:] = torch.randn(many - few, k, generator=g).to(dtype).cuda()
    z[few, 0], z[many - 1, k - 1] = float("nan"), float("inf")
    got = layer(z)
    assert torch.equal(got[:few], y[:few]) and got[few].isnan().all() and not got[many - 1].isfinite().any()
