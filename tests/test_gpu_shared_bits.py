"""Shared prefixes keep 16 bits of every probability wherever the calls that they take the place of do, and what a request
gets does not depend on the lengths, padding or inputs of the others in its group."""
import pytest

from page_path import check
from shared_path import batch, decode, starts, suffix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (8, 1, 64)])
@pytest.mark.parametrize("sizes", [[17], [40, 3], [9, 9, 30]])
def test_decode_of_many_rows(hq, hkv, d, sizes):
    """Groups of more than 64 query rows: two terms of a probability, 2^-16 of it."""
    shared = [640 + 200 * i for i in range(len(sizes))]
    ctx = [s + (11 * i) % 90 for n, s in zip(sizes, shared) for i in range(n)]
    x = batch(hq, hkv, d, 32, ctx, [1] * len(ctx), starts(sizes), shared)
    decode(x)
    check(x, decoded=True)


@pytest.mark.parametrize("hq,hkv,d,n", [(32, 8, 128, 2), (32, 8, 64, 8), (28, 4, 128, 4), (8, 1, 64, 4)])
def test_suffixes_of_up_to_32_rows(hq, hkv, d, n):
    ctx = [1300 + 7 * i for i in range(16)]
    x = batch(hq, hkv, d, 64, ctx, [1 + i % n for i in range(16)], [0, 10, 16], [1300, 1340], n=n)
    suffix(x)
    check(x, decoded=True)


def test_a_bound_far_above_the_groups():
    """max_group is a bound: groups of two under one of 64 keep their bits."""
    x = batch(32, 8, 128, 64, [700 + i for i in range(8)], [1] * 8, [0, 2, 4, 6, 8], [700, 702, 650, 706])
    x.shared.max_group = 64
    decode(x)
    check(x, decoded=True)
