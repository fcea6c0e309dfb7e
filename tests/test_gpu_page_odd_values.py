"""Values that are not finite in the bf16 calls over pages: they reach the outputs of the tokens that see them, in their
head dim, whichever kernel a call goes to and however its keys are split over waves and workgroups, and no other."""
import pytest

from page_odd import INF, NAN, rescaled, value_case
from page_path import decode, suffix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_splits", [1, 3, 8])
@pytest.mark.parametrize("rope", [False, True])
def test_decode_values(d, n_splits, rope):
    # in the first tile and a last one, a wave's only key, the new token itself, opposite infinities in one sum
    ctx = [0, 32, 40, 700, 2000, 3001]
    bad = [(0, 0, 1, 5, INF), (1, 31, 0, 0, -INF), (1, 32, 0, 1, INF), (2, 7, 1, d - 1, NAN), (2, 40, 0, 9, -INF),
           (3, 0, 0, 3, INF), (3, 650, 0, 3, INF), (3, 11, 1, 20, INF), (3, 690, 1, 20, -INF), (4, 1999, 0, 33, INF),
           (4, 2000, 0, 34, NAN), (5, 1500, 1, 16, -INF), (5, 3001, 1, 16, -INF), (5, 2999, 0, 63, INF)]
    value_case(lambda x, **k: decode(x, n_splits=n_splits, **k), (16, 2, d, "bf16", 16, ctx, [1] * 6), bad, rope=rope)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_splits", [1, 2, 8])
def test_decode_values_of_small_probability(d, n_splits):
    """Scores so far apart that most probabilities, waves' and ranges' weights are 0 in 32 bits: an infinity is none
    the less in the average."""
    ctx = [100, 900, 6000, 6000]
    bad = [(b, s, g, 4 * i + b, INF if i % 2 else -INF) for b, n in enumerate(ctx) for g in range(2)
           for i, s in enumerate((0, 13, 33, n // 2, n - 1, n))]
    value_case(lambda x, **k: decode(x, n_splits=n_splits, **k), (16, 2, d, "bf16", 64, ctx, [1] * 4), bad, queries=200.0)


@pytest.mark.parametrize("hq,hkv,d,n", [(32, 8, 128, 1), (32, 8, 128, 4), (32, 8, 128, 8), (8, 4, 64, 5), (16, 2, 64, 4)])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("queries", [1.0, 200.0])
@pytest.mark.parametrize("batch", [16, 28])
def test_few_rows_values(hq, hkv, d, n, rope, queries, batch):
    """Cached values and new tokens' together; batches that the kernel of few rows takes, whole and in two ranges."""
    ctx = [1700 + 64 * i for i in range(batch)]
    ctx[:3] = [64, 1, 40]
    bad = [(0, 0, 0, 1, INF), (0, 63, 1, 2, -INF), (0, 64 + n - 1, 0, 1, INF), (1, 0, 1, 3, NAN), (2, 5, 0, 9, INF),
           (2, 40, 0, 9, -INF), (5, 1000, 1, 60, INF), (6, 3, 0, 0, -INF), (6, ctx[6] - 1, 0, 0, -INF),
           (7, ctx[7] - 1, 2 % hkv, 33, INF), (8, ctx[8] + n // 2, 1, 7, INF), (9, 800, 0, 12, NAN)]
    value_case(suffix, (hq, hkv, d, "bf16", 32, ctx, [n] * len(ctx)), bad, queries, rope)


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 8, 128, 128, [190] * 12), (32, 8, 128, 40, [9001, 20]), (8, 2, 64, 67, [4161, 30]),
                                            (32, 8, 128, 128, [6000] * 8)])
@pytest.mark.parametrize("rope", [False, True])
def test_prefill_values(hq, hkv, d, n, ctx, rope):
    """The prefill kernel, whole and split, with both kinds of shares."""
    bad = [(0, 0, 0, 1, INF), (0, ctx[0] - 1, 1, 2, -INF), (0, ctx[0] + n // 2, 0, 1, INF), (1, 3, 1, 40, NAN), (1, 7, 0, 9, -INF),
           (1, ctx[1] + n - 1, 1, 50, INF), (0, ctx[0] // 2, 1, 63, INF)]
    value_case(suffix, (hq, hkv, d, "bf16", 16, ctx, [n] * len(ctx)), bad, rope=rope, slack=rescaled)


@pytest.mark.parametrize("n,ctx", [(40, [9001, 20]), (128, [6000] * 8)])
def test_prefill_new_values_of_small_probability(n, ctx):
    """New tokens' infinities in a range whose weight is 0 in 32 bits when the ranges are joined."""
    bad = [(b, ctx[b] + i, g, 8 * g + j, v) for b in (0, 1) for g in (0, 3) for j, (i, v) in enumerate([(0, INF), (n // 2, -INF)])]
    value_case(suffix, (32, 8, 128, "bf16", 64, ctx, [n] * len(ctx)), bad, queries=200.0, slack=rescaled)
