"""Values and keys that are not finite in float32 pages: as in the bf16 calls (test_gpu_page_odd_values.py)."""
import pytest

from page_odd import INF, NAN, key_case, value_case
from page_path import decode, suffix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("queries", [1.0, 200.0])
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 64), (8, 2, 128)])
def test_decode_values(hq, hkv, d, queries):
    ctx = [0, 16, 40, 700, 2000]
    bad = [(0, 0, 1, 5, INF), (1, 15, 0, 0, -INF), (1, 16, 0, 1, INF), (2, 7, 1, d - 1, NAN), (2, 40, 0, 9, -INF),
           (3, 0, 0, 3, INF), (3, 650, 0, 3, INF), (3, 11, 1, 20, INF), (3, 690, 1, 20, -INF), (4, 1999, 0, 33, INF),
           (4, 2000, 0, 34, NAN), (4, 17, 1, 35, -INF)]
    value_case(decode, (hq, hkv, d, "f32", 16, ctx, [1] * 5), bad, queries, slack=reordered)


def reordered(x):
    """Float32 sums of the same terms in another order: of at most T terms no larger than the batch's values, 2^-24 T
    each, in numerator and denominator."""
    most, T = float(max(v[v.isfinite()].abs().max() for v in x.V)), max(k.shape[2] for k in x.K)
    return lambda want: 4 * T * 2.0 ** -24 * most + 0 * want


@pytest.mark.parametrize("queries", [1.0, 200.0])
@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(16, 4, 64, 21, [300, 64, 0]), (8, 2, 128, 5, [900, 3]), (32, 2, 64, 100, [200] * 20)])
def test_suffix_values(hq, hkv, d, n, ctx, queries):
    bad = [(0, 0, 0, 1, INF), (0, ctx[0] - 1, 1, 2, -INF), (0, ctx[0] + n // 2, 0, 1, INF), (1, 0, 1, 40, NAN),
           (1, ctx[1] + n - 1, 1, 50, INF), (0, ctx[0] // 2, 1, 63, INF), (1, ctx[1], 0, 17, -INF)]
    value_case(suffix, (hq, hkv, d, "f32", 16, ctx, [n] * len(ctx)), bad, queries, slack=reordered)


def test_keys_that_are_nan():
    bad = [(0, 0, 1), (1, 16, 0), (2, 128, 1), (4, 1999, 0)] + [(3, s, 0) for s in range(32)]
    key_case(decode, (16, 2, 64, "f32", 16, [0, 16, 128, 300, 2000], [1] * 5), bad)
    key_case(suffix, (16, 4, 64, "f32", 16, [256, 64], [21, 21]), [(0, 256, 1), (0, 260, 0), (1, 3, 2)])
