"""Log probabilities, entropy and alternatives against 64 bits: layouts, sizes, strides, ties, scores that are not
finite, labels out of range."""
import pytest
import torch

import paper_1704_04313_amd as cb
from token_util import check_log_probs

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


def _scores(shape, dtype, seed, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=g)).to(dtype).cuda()


def _labels(shape, classes, seed, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed + 77)
    return torch.randint(0, classes, shape, generator=g).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes,top", [(1, 1, 1), (3, 2, 2), (5, 7, 0), (2, 63, 5), (4, 64, 64), (3, 65, 64), (9, 1000, 8),
                                              (2, 4099, 3), (1, 50021, 16), (70, 513, 1), (300, 129, 4), (3, 20011, 8)])
def test_rows(rows, classes, top, dtype):
    x, l = _scores((rows, classes), dtype, classes + rows), _labels((rows,), classes, rows, torch.int32 if rows % 2 else torch.int64)
    check_log_probs(cb.log_probs(x, l, top=top), x, l, 1, top, "%dx%d" % (rows, classes))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,classes,h,w,top", [(1, 8, 60, 80, 3), (2, 3, 5, 7, 3), (1, 1, 4, 4, 1), (3, 21, 17, 9, 8), (2, 150, 8, 8, 5),
                                               (1, 300, 3, 3, 17), (5, 8, 33, 31, 0), (1, 40, 1, 16, 20), (2, 64, 16, 17, 64), (1, 2000, 4, 5, 2)])
def test_maps(n, classes, h, w, top, dtype):
    x, l = _scores((n, classes, h, w), dtype, classes), _labels((n, h, w), classes, n)
    check_log_probs(cb.log_probs(x, l, dim=1, top=top), x, l, 1, top, "map")


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_axes(dtype):
    big = _scores((6, 40, 90), dtype, 1)
    for x, dim, top in ((big[1:5, :33, 5:85], 1, 4), (big.transpose(1, 2), 2, 3), (big[:, :, ::3], 1, 2), (big[:, ::2], 2, 5),
                        (big[2, 1:], 1, 3), (big[2, 1:].t(), 1, 3), (big[0, 0, 1:], 0, 5), (big, 0, 6), (big[:1, :, 3:4], 1, 2)):
        labels = _labels(tuple(x.shape[:dim]) + tuple(x.shape[dim + 1:]), x.shape[dim], 3)
        check_log_probs(cb.log_probs(x, labels, dim=dim, top=top), x, labels, dim, top, "%s %s" % (tuple(x.shape), x.stride()))
        check_log_probs(cb.log_probs(x, None, dim=dim - x.dim(), top=0), x, None, dim, 0, "no labels")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
def test_rows_at_any_address(offset, dtype):
    flat = _scores((offset + 5 * 1003,), dtype, 5)
    x = flat[offset:].view(5, 1003)
    l = _labels((5,), 1003, 2)
    check_log_probs(cb.log_probs(x, l, top=5), x, l, 1, 5)


@pytest.mark.parametrize("shape", [(4, 700), (2, 30, 4, 5), (2, 40000), (1, 300, 40, 20)])
def test_ties_go_to_the_lowest_class(shape):
    g = torch.Generator().manual_seed(9)
    x = torch.randint(-2, 3, shape, generator=g).float().cuda()
    x[0] = 0.0
    x[0, ::2] = -0.0
    check_log_probs(cb.log_probs(x, None, top=20), x, None, 1, 20, "ties")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(6, 900), (6, 12, 3, 5), (6, 30011), (6, 64, 24, 40)])
def test_masks(shape, dtype):
    """-inf scores: some, all but one, all; the type's lowest value as a mask, in all places and in some."""
    x = _scores(shape, dtype, 11)
    low = torch.finfo(dtype).min
    ninf = float("-inf")
    x[0, 1::2] = ninf
    x[1] = ninf
    x[1, 5] = 2.0
    x[2] = ninf
    x[3] = low
    x[4, 3:] = low
    x[5, :7] = ninf
    x[5, 8:] = low
    labels = torch.full(shape[:1] + shape[2:], 5).cuda()
    check_log_probs(cb.log_probs(x, labels, top=4), x, labels, 1, 4, "masks")


@pytest.mark.parametrize("shape", [(5, 500), (5, 20, 3, 4), (5, 30011), (5, 40, 64, 30)])
def test_not_finite(shape):
    x = _scores(shape, torch.float32, 13)
    x[0, 3] = float("nan")
    x[1, 4] = float("inf")
    x[2, 2], x[2, 4], x[2, 7] = float("inf"), float("nan"), float("nan")
    x[3] = float("nan")
    x[4] *= 1e37
    labels = torch.full(shape[:1] + shape[2:], 4).cuda()
    check_log_probs(cb.log_probs(x, labels, top=5), x, labels, 1, 5, "not finite")


def test_labels_out_of_range():
    for shape, rest in (((7, 33), (7,)), ((7, 9, 4, 6), (7, 4, 6))):
        x = _scores(shape, torch.float32, 17)
        for kind in (torch.int32, torch.int64):
            labels = _labels(rest, shape[1], 1, kind)
            labels[1], labels[2], labels[3], labels[4] = -1, shape[1], -100, 2 ** 31 - 1
            check_log_probs(cb.log_probs(x, labels, top=2), x, labels, 1, 2, "labels")
        labels = labels.long()
        labels[5] = 2 ** 40
        check_log_probs(cb.log_probs(x, labels, top=2), x, labels, 1, 2, "labels of 64 bits")


@pytest.mark.parametrize("value", [1e30, -1e30, 80.0, -3e38])
def test_large_scores(value):
    x = _scores((3, 400), torch.float32, 19) + value
    check_log_probs(cb.log_probs(x, None, top=3), x, None, 1, 3, "large")


def test_rising_and_falling_scores():
    """Every score a new maximum, or none behind the first: the running sums are rescaled always or never."""
    for n in (1000, 40000):
        x = torch.linspace(-30, 30, n).repeat(2, 1).cuda()
        x[1] = x[1].flip(0)
        check_log_probs(cb.log_probs(x, None, top=8), x, None, 1, 8, "slopes")


def test_offsets_beyond_32_bits():
    """Scores whose last row begins behind 2^32 bytes and 2^31 elements."""
    classes, rows = 1 << 20, 2050
    x = torch.zeros((rows, classes), dtype=torch.bfloat16, device="cuda")
    part = _scores((1, 3000), torch.bfloat16, 23)
    x[-1, -3000:] = part[0]
    x[-1, :-3000] = float("-inf")
    labels = torch.full((rows,), classes - 1).cuda()
    got = cb.log_probs(x, labels, top=3)
    want = cb.log_probs(part, labels[:1] * 0 + 2999, top=3)
    assert torch.equal(got.index[-1].cpu(), want.index[0].cpu() + classes - 3000)
    torch.testing.assert_close(got.top[-1], want.top[0], rtol=0, atol=1e-5)
    torch.testing.assert_close(got.label[-1], want.label[0], rtol=0, atol=1e-5)
    torch.testing.assert_close(got.entropy[-1], want.entropy[0], rtol=0, atol=1e-5)
    assert torch.equal(got.index[0].cpu(), torch.arange(3, dtype=torch.int32))


def test_nothing_to_do_and_other_streams():
    for shape in ((0, 10), (3, 10, 0, 4)):
        got = cb.log_probs(torch.empty(shape, device="cuda"), None, top=2)
        assert got.entropy.numel() == 0 and got.top.numel() == 0
    x, l = _scores((40, 30000), torch.bfloat16, 29), _labels((40,), 30000, 1)
    want = cb.log_probs(x, l, top=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cb.log_probs(x, l, top=4)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("outer_stride", [0, 7, 640, 1300])
def test_maps_that_overlap_or_repeat(outer_stride, dtype):
    x = _scores((6000,), dtype, 9).as_strided((5, 40, 16), (outer_stride, 16, 1))
    labels = _labels((5, 16), 40, 4)
    check_log_probs(cb.log_probs(x, labels, top=5), x, labels, 1, 5, "stride %d" % outer_stride)


@pytest.mark.parametrize("dtype,outer_stride", [(torch.float32, 1 << 26), (torch.bfloat16, 1 << 27)])
@pytest.mark.parametrize("inner", [16, 300])
def test_maps_far_apart(dtype, outer_stride, inner):
    """A workgroup's positions span more than 32 bits of offsets, were the maps as many as it has positions for."""
    memory = torch.empty(2 * outer_stride + 100 * inner, dtype=dtype, device="cuda")
    x = memory.as_strided((3, 37, inner), (outer_stride, inner, 1))
    x.copy_(_scores((3, 37, inner), dtype, inner))
    labels = _labels((3, inner), 37, 8)
    check_log_probs(cb.log_probs(x, labels, top=4), x, labels, 1, 4, "far apart")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,classes,h,w,top", [(1, 33, 20, 20, 3), (2, 35, 16, 31, 5), (3, 47, 40, 40, 1), (2, 9, 250, 260, 2), (5, 40, 230, 235, 3),
                                               (5, 40, 230, 235, 0)])
def test_larger_maps(n, classes, h, w, top, dtype):
    """A waves' share of the classes, or all of them a lane: some of the positions."""
    x, l = _scores((n, classes, h, w), dtype, classes), _labels((n, h, w), classes, n, torch.int32)
    got = cb.log_probs(x, l, top=top)
    some = torch.randint(0, n * h * w, (200,), generator=torch.Generator().manual_seed(top)).cuda()
    some[0], some[1] = 0, n * h * w - 1
    rows = lambda t: t.movedim(1, -1).flatten(0, 2)[some]  # noqa: E731
    got = type(got)(got.label.flatten()[some], got.entropy.flatten()[some], rows(got.top) if top else None, rows(got.index) if top else None)
    check_log_probs(got, rows(x), l.flatten()[some], 1, top, "map")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [32, 33, 36, 40, 47, 56, 61])
@pytest.mark.parametrize("top", [8, 10, 12, 16])
def test_maps_with_fewer_live_classes_than_alternatives(classes, top, dtype):
    """Positions with 0 .. top - 1 classes that are not ruled out, anywhere among the classes: those ruled out follow, each once, the
    lowest first, wherever a position's classes are divided among waves."""
    g = torch.Generator().manual_seed(classes + 100 * top)
    x = torch.randn(2, classes, 6, 16, generator=g)
    places = torch.rand(2, classes, 6, 16, generator=g).argsort(1).argsort(1)
    live = (torch.arange(2 * 6 * 16) % top).view(2, 1, 6, 16)
    x[places >= live] = float("-inf")
    x = x.to(dtype).cuda()
    labels = _labels((2, 6, 16), classes, top)
    check_log_probs(cb.log_probs(x, labels, top=top), x, labels, 1, top, "%d classes, %d best" % (classes, top))


@pytest.mark.parametrize("dtype,classes", [(torch.bfloat16, 2 ** 31 - 1), (torch.float32, 2 ** 31 - 1), (torch.bfloat16, 2 ** 31 - 64)])
def test_as_many_classes_as_there_may_be(dtype, classes):
    """One row of 2^31 - 1 scores: the last ones are the best, in front of the last whole 16 bytes and behind."""
    x = torch.full((1, classes), -30.0, dtype=dtype, device="cuda")
    best = {classes - 1: 2.0, 0: 1.0, classes - 9: 3.0, 2 ** 30 + 1: 0.5, classes - 2: 0.0}
    for at, value in best.items():
        x[0, at] = value
    got = cb.log_probs(x, torch.tensor([classes - 1], device="cuda"), top=5)
    order = sorted(best, key=lambda c: -best[c])
    every = torch.tensor([best[c] for c in order], dtype=torch.float64)
    # 2^31 terms of e^-30 are 2e-4: of their sum's roundings (4 sqrt(2^31) at most) nothing reaches the logarithm's last bits
    log_s = (every.exp().sum() + (classes - 5) * torch.tensor(-30.0, dtype=torch.float64).exp()).log()
    assert got.index[0].tolist() == order
    torch.testing.assert_close(got.top[0].cpu().double(), every - log_s, rtol=0, atol=1e-5)
    torch.testing.assert_close(got.label[0].cpu().double(), 2.0 - log_s, rtol=0, atol=1e-5)
