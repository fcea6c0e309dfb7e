"""What other tests of shared prefixes take for granted: that values that are not finite were put where rows see them, and which
rows of the pages a call with a partly wrong table may change."""
import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, SENTINEL, rows
from shared_path import batch, suffix
from test_gpu_shared import _odd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("kind", ["inf", "nan", "both"])
def test_odd_values_are_there(n, kind):
    x = batch(8, 1, 128, 64, [140, 150, 133], [n] * 3, [0, 3], [131], n=n)
    assert all(torch.isfinite(v).all() for v in x.V)
    _odd(x, kind)
    for b in range(3):
        bad = ~torch.isfinite(x.V[b])
        assert bad.sum() >= 4
        assert (bad[:, :, : x.ctx[b]] == ~torch.isfinite(x.pv[:, :, rows(x, b, 0, x.ctx[b])])).all()
        assert (bad[:, :, x.ctx[b]:] == ~torch.isfinite(x.v[:, b].transpose(1, 2))).all()


@pytest.mark.parametrize("n", [1, 3, 20])
def test_tables_that_are_wrong_in_part(n):
    """Entries that are pages, none, past the last page or far out of range, lengths and counts out of range: exactly the rows of new
    tokens whose entry is a page change, keys and values alike; padding keeps its output rows."""
    r = np.random.default_rng(n)
    stored = 0
    for it in range(8):
        B, P = 5, 16
        x = batch(8, 2, 64, P, [300, 350, 310, 333, 200], [n] * B, [0, 3, 5], [300, 200], n=n, L=2)
        N = x.pages.n_pages
        table = np.where(r.random(x.table_host.shape) < 0.5, r.choice([-1, N, N + 1, -2**31, 2**31 - 1, -N], x.table_host.shape), 0)
        own = np.argwhere(table == 0)
        own = own[r.permutation(len(own))][:N]      # (no page twice)
        table[table == 0] = -1
        table[own[:, 0], own[:, 1]] = r.permutation(N)[: len(own)]
        x.table_host = table.astype(np.int32)
        x.table = torch.from_numpy(x.table_host).to(DEV)
        lens = [int(v) for v in r.choice([300, 350, 17, 0, -1, -2**31, 2**31 - 1], B)]
        valid = [n] * B if n == 1 else [int(v) for v in r.choice([n, n - 1, 1, 0, -5, 2**31 - 1], B)]
        x.len, x.n_valid = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (lens, valid))
        x.start = torch.from_numpy(r.integers(-9, 9, 3).astype(np.int32)).to(DEV)
        x.shared_len = torch.from_numpy(r.integers(-2**31, 2**31, 2).astype(np.int32)).to(DEV)
        want = x.pk.clone(), x.pv.clone()
        live = torch.zeros((B, n), dtype=torch.bool)
        for b in range(B):
            if lens[b] < 0:
                continue
            for i in range(min(max(valid[b], 0), n)):
                live[b, i] = True
                slot = min(lens[b], x.max_ctx) + i
                page = int(x.table_host[b, slot // P])
                if 0 <= page < N:
                    stored += 1
                    at = page * P + slot % P
                    want[0][:, :, at], want[1][:, :, at] = x.k[:, b, i], x.v[:, b, i]
        if n == 1:
            pic.pic_page_shared_decode_attn(x.model, x.pages, x.shared, x.q, x.k, x.v, x.pk, x.pv, x.table, B, x.start, x.shared_len, x.len, 0,
                                            x.max_ctx, x.out, torch.empty(max(16, pic.pic_page_shared_workspace_bytes(
                                                x.model, x.shared, B, 1, x.max_ctx)), dtype=torch.uint8, device=DEV))
        else:
            suffix(x)
        torch.cuda.synchronize()
        for got, w in zip((x.pk, x.pv), want):
            assert (got.view(torch.int16) == w.view(torch.int16)).all(), it
        assert (x.out[:, ~live.to(DEV)] == SENTINEL).all(), it
    assert stored > 0   # (not for nothing)
