"""Page copies: exact in every layer and kv head of both buffers, everything else untouched."""
import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,hkv,d,P,n_pages,n_pairs", [
    (1, 1, 64, 16, 2, 1), (1, 2, 64, 16, 40, 20), (3, 8, 128, 64, 33, 5), (2, 4, 128, 16, 1400, 700),
    (1, 1, 64, 1024, 5, 2), (28, 4, 128, 128, 9, 4), (1, 3, 64, 32, 600, 256), (1, 3, 64, 32, 600, 257), (40, 1, 64, 16, 8, 3),
    (40000, 1, 64, 16, 3, 1)])
def test_copy(dtype, L, hkv, d, P, n_pages, n_pairs):
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    at = np.random.default_rng(n_pairs).permutation(n_pages)[: 2 * n_pairs].reshape(-1, 2)
    k, v = (torch.randn((L, hkv, n_pages, P, d), device=DEV, dtype=dt) for _ in range(2))
    k[0, 0, at[0, 0], 0, 0] = float("nan")   # bits are moved, not values
    want = []
    for x in (k, v):
        w = x.clone()
        w[:, :, torch.from_numpy(at[:, 1].copy()).to(DEV)] = x[:, :, torch.from_numpy(at[:, 0].copy()).to(DEV)]
        want.append(w)
    m = pic.Model.of(L, hkv, hkv, d, dtype, 1e4)
    pic.pic_page_copy(m, pic.Pages.of(n_pages, P, 0), k, v, at)
    i = torch.int32 if dtype == "f32" else torch.int16
    for x, w in zip((k, v), want):
        assert (x.view(i) == w.view(i)).all()


def test_copy_past_32_bits():
    n_pages, P = 1 << 19, 64   # a stream of 8.6 GB
    k = torch.zeros((1, 1, n_pages, P, 128), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    k[0, 0, n_pages - 1], v[0, 0, 3] = 2.0, 3.0
    pairs = [[n_pages - 1, 1], [3, n_pages - 2]]
    pic.pic_page_copy(pic.Model.of(1, 1, 1, 128, "bf16", 1e4), pic.Pages.of(n_pages, P, 0), k, v, pairs)
    assert (k[0, 0, 1] == 2).all() and (v[0, 0, n_pages - 2] == 3).all()
    assert (v[0, 0, 1] == 0).all() and (k[0, 0, n_pages - 2] == 0).all()
    assert int((k != 0).any(-1).any(-1).sum()) == 2 and int((v != 0).any(-1).any(-1).sum()) == 2


def test_refused_copies_write_nothing():
    k = torch.randn((1, 2, 4, 16, 64), device=DEV, dtype=torch.bfloat16)
    v, was = k.clone(), k.clone()
    m, g = pic.Model.of(1, 2, 2, 64, "bf16", 1e4), pic.Pages.of(4, 16, 0)
    for pairs in ([[0, 1], [1, 2]], [[0, 1], [2, 1]], [[0, 4]], [[2, 2]]):
        with pytest.raises(pic.PicError):
            pic.pic_page_copy(m, g, k, v, pairs)
    with pytest.raises(ValueError):
        pic.pic_page_copy(m, g, k, v, [0, 1])
    pic.pic_page_copy(m, g, k, v, np.zeros((0, 2), np.int32))
    torch.cuda.synchronize()
    assert (k == was).all() and (v == was).all()
