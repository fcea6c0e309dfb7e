"""Keys and queries that are not finite in the bf16 calls over pages: a NaN score makes its output NaN and a score of -inf
has no weight, whichever kernel a call goes to and however its keys are split over waves and workgroups."""
import math

import pytest
import torch

from page_odd import INF, NAN, key_case, rounded_anew, same_but
from page_path import DEV, decode, rows, setup, suffix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_splits", [1, 2, 8])
@pytest.mark.parametrize("rope", [False, True])
def test_decode_keys_that_are_nan(d, n_splits, rope):
    """A NaN in a visible key makes every output of its kv head NaN: the newest key where it is a wave's or a
    range's only one, whole tiles, ranges and one key in the middle."""
    ctx = [0, 32, 128, 300, 127, 640, 1024, 5000]
    bad = [(0, 0, 1), (1, 32, 0), (2, 128, 1), (4, 127, 0), (6, 500, 1), (7, 5000, 1)] + [(3, s, 0) for s in range(96)]
    bad += [(5, s, 1) for s in range(512, 641)]
    call = lambda z, **k: decode(z, n_splits=n_splits, **k)  # noqa: E731
    key_case(call, (16, 2, d, "bf16", 16, ctx, [1] * 8), bad, rope)


@pytest.mark.parametrize("hq,hkv,d,n", [(32, 8, 128, 1), (32, 8, 128, 4), (32, 8, 128, 8), (8, 4, 64, 5)])
@pytest.mark.parametrize("rope", [False, True])
def test_few_rows_keys_that_are_nan(hq, hkv, d, n, rope):
    ctx = [0, 32, 256, 300, 255, 2048] + [1700 + 64 * i for i in range(24)]
    bad = [(0, 0, 1), (1, 32, 0), (2, 256, 1), (4, 255 + n - 1, 0), (5, 2048 + n // 2, 1), (9, 700, 1)]
    bad += [(3, s, 0) for s in range(64)] + [(8, s, 2 % hkv) for s in range(256, 640)]
    key_case(suffix, (hq, hkv, d, "bf16", 32, ctx, [n] * len(ctx)), bad, rope)


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 8, 128, 40, [4096] * 2), (32, 8, 128, 40, [4096]), (8, 2, 64, 64, [4096] * 2),
                                            (8, 2, 128, 33, [4096] * 3), (32, 8, 128, 128, [6016] * 8), (8, 2, 128, 64, [130, 700])])
@pytest.mark.parametrize("rope", [False, True])
def test_prefill_keys_that_are_nan(hq, hkv, d, n, ctx, rope):
    """Among them a range of a split launch whose only key of a row is NaN: 4096 cached keys in 8 ranges of 8 tiles
    and a last one that begins with the new tokens."""
    bad = [(0, ctx[0], 0), (len(ctx) - 1, ctx[-1] + n // 2, 1), (len(ctx) - 1, 3, 0)]
    key_case(suffix, (hq, hkv, d, "bf16", 64, ctx, [n] * len(ctx)), bad, rope)


@pytest.mark.parametrize("kind", ["decode", "few"])
def test_queries_that_are_nan(kind):
    n = 1 if kind == "decode" else 4
    ctx = [100, 2600, 2600] + [2600] * 13
    x, y = (setup(32, 8, 128, "bf16", 64, ctx, [n] * 16) for _ in range(2))
    x.q[0, 1, n - 1, 5, 17] = NAN
    for z in (x, y):
        (decode if kind == "decode" else suffix)(z)
    want = y.out.clone()
    want[0, 1, n - 1, 5] = NAN
    same_but(x, want, rounded_anew(y))


@pytest.mark.parametrize("kind", ["decode", "decode whole", "few"])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_of_minus_infinity(kind, d):
    """Keys whose score is -inf have no weight, also where they are all that a wave or a range holds."""
    n = 1
    ctx = [3000, 200] + [2500] * 62 if kind == "few" else [3000, 200, 129, 5000]
    x = setup(4, 4, d, "bf16", 16, ctx, [n] * len(ctx))
    gone = {0: list(range(0, 1500)), 1: list(range(32, 200)), 2: list(range(128)) + [129], 3: list(range(640, ctx[3] + 1))}
    for b, slots in gone.items():
        for g in range(4):
            # -inf times the sign of this head's query in one head dim
            v = -INF if float(x.q[0, b, 0, g, 3]) > 0 else INF
            old = [s for s in slots if s < ctx[b]]
            at = torch.cat([rows(x, b, s, s + 1) for s in old])
            x.pk[0, g, at, 3] = v
            if ctx[b] in slots:
                x.k[0, b, 0, g, 3] = v
    suffix(x) if kind == "few" else decode(x, n_splits=1 if kind == "decode whole" else 0)
    for b, slots in gone.items():
        keep = torch.ones(ctx[b] + 1, dtype=torch.bool, device=DEV)
        keep[torch.tensor(slots, device=DEV)] = False
        for g in range(4):
            K, V = x.K[b][0, g].double()[keep], x.V[b][0, g].double()[keep]
            p = (K @ x.q[0, b, 0, g].double() / math.sqrt(d)).softmax(0)
            ref, mag = p @ V, p @ V.abs()
            # output 2^-8, probabilities in two bfloat16 terms 2^-16 in numerator and denominator, float32 sums
            tol = 2.0 ** -8 * ref.abs() + (2 * 2.0 ** -16 + 2.0 ** -14) * mag
            assert ((x.out[0, b, 0, g].double() - ref).abs() <= tol).all(), (b, g)
