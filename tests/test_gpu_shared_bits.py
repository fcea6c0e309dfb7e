"""Shared prefixes keep 16 bits of every probability wherever the calls that they take the place of do, and what a request
gets does not depend on the lengths, padding or inputs of the others in its group."""
import pytest
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, SENTINEL, check, rows, setup
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


def _group_of_copies(hq, hkv, d, ctx, shared, n):
    """One group whose requests hold the shared slots in pages of their own, so that any of them may be cut short."""
    x = setup(hq, hkv, d, "bf16", 32, ctx, [n] * len(ctx), n=n, slack=64)
    for b in range(1, x.B):
        x.K[b][:, :, :shared], x.V[b][:, :, :shared] = x.K[0][:, :, :shared], x.V[0][:, :, :shared]
        r = rows(x, b, 0, shared)
        x.pk[:, :, r], x.pv[:, :, r] = x.K[0][:, :, :shared], x.V[0][:, :, :shared]
    x.start = torch.tensor([0, x.B], dtype=torch.int32, device=DEV)
    x.shared_len = torch.tensor([shared], dtype=torch.int32, device=DEV)
    x.shared = pic.Shared.of(1, x.B, shared)
    return x


@pytest.mark.parametrize("hq,hkv,d,n", [(32, 8, 128, 1), (32, 4, 128, 9), (32, 8, 64, 9), (8, 1, 128, 3)])
def test_bits_do_not_depend_on_the_neighbours(hq, hkv, d, n):
    """Requests 0 and 5 stay as they are; the others grow shorter than the prefix, become padding, lose tokens, and what their
    queries hold (padding included) turns from small to huge to NaN: the same bits for 0 and 5."""
    keep, others = [0, 5], [1, 2, 3, 4, 6, 7]
    x = _group_of_copies(hq, hkv, d, [1700 + 3 * b for b in range(8)], 1690, n)
    run = decode if n == 1 else suffix
    want = run(x)[:, keep].clone()
    check(x, decoded=n * (hq // hkv) <= 32)
    assert (want != SENTINEL).any()
    base, valid = x.len.clone(), x.n_valid.clone()
    pages = x.pk.clone(), x.pv.clone()
    lengths = {"same": [base[b].item() for b in others], "short": [1600, 700, 64, 63, 0, 1], "padding": [-1] * 6,
               "mixed": [-1, 1500, -1, 128, -1, 9]}
    for name, lens in lengths.items():
        for fill in (0.01, 30.0, 3e4, float("nan")):
            for tokens in sorted({0, n // 2, n}):
                x.len, x.n_valid = base.clone(), valid.clone()
                x.len[others] = torch.tensor(lens, dtype=torch.int32, device=DEV)
                x.n_valid[others] = tokens
                x.pk.copy_(pages[0]), x.pv.copy_(pages[1])
                q = x.q.clone()
                x.q[:, others] = q[:, others] * fill if fill == fill else float("nan")
                got = run(x)[:, keep]
                assert (got == want).all(), (name, fill, tokens, int((got != want).sum()))
                x.q = q
