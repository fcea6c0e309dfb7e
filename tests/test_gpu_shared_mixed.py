"""Shared prefixes beside requests that share nothing or little: outside the groups, past max_group, in groups of one of their
own; their many key ranges against the definition in 64 bits."""
import pytest
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, check
from shared_path import batch, decode, suffix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (8, 2, 64)])
@pytest.mark.parametrize("where", ["before", "after", "both"])
def test_decode_beside_a_group(hq, hkv, d, where):
    lone = [5003, 17, 4800]
    group = [4700, 4690, 4750]
    ctx = {"before": lone + group, "after": group + lone, "both": lone[:2] + group + lone[2:]}[where]
    at = {"before": 3, "after": 0, "both": 2}[where]
    x = batch(hq, hkv, d, 64, ctx, [1] * 6, [0, at, at + 3, 6], [0, 4690, 0])
    x.start, x.shared_len = x.start[1:3].clone(), x.shared_len[1:2].clone()
    x.shared = pic.Shared.of(1, 3, 4690)
    decode(x, step=2)
    check(x, decoded=True)


def test_past_max_group():
    x = batch(32, 8, 128, 32, [3000 + 7 * b for b in range(7)], [1] * 7, [0, 7], [3000])
    x.shared = pic.Shared.of(1, 3, 3000)
    decode(x)
    check(x, decoded=True)


def test_suffix_beside_groups():
    x = batch(16, 4, 64, 16, [1200, 1210, 2500, 1300, 1290, 70], [3, 4, 4, 1, 4, 2], [0, 2, 3, 5, 6], [1200, 0, 1290, 0], n=4, L=2)
    x.start = torch.tensor([0, 2, 3, 5], dtype=torch.int32, device=DEV)
    x.shared_len = torch.tensor([1200, 0, 1290], dtype=torch.int32, device=DEV)
    x.shared = pic.Shared.of(2, 2, 1290)
    x.start, x.shared_len = x.start[:3].clone(), x.shared_len[:2].clone()   # (requests 3 to 5 in no group)
    suffix(x)
    check(x, decoded=True)


def test_a_group_of_its_own():
    """A long request beside a group, as a group of one that shares its whole length with nobody."""
    ctx = [2100, 2110, 2090, 6000, 333]
    x = batch(32, 8, 128, 64, ctx, [1] * 5, [0, 3, 4, 5], [2090, 6000, 333])
    decode(x)
    check(x, decoded=True)
