"""Shared set-up of the tests of batches that share prefixes: requests of page_path.setup made to share their first
slots' pages in groups."""
import numpy as np
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, rows, setup


def share(x, start, shared):
    """Requests [start[g], start[g + 1]) hold the first one's tokens in slots [0, shared[g]), whole pages of them the same
    pages; the rows that they held before are NaN."""
    for g, s in enumerate(shared):
        a = start[g]
        for b in range(a + 1, start[g + 1]):
            n = min(s, max(x.ctx[b], 0))
            whole = n // x.P * x.P
            x.K[b][:, :, :n], x.V[b][:, :, :n] = x.K[a][:, :, :n], x.V[a][:, :, :n]
            for p in (x.pk, x.pv):
                p[:, :, rows(x, b, 0, whole)] = float("nan")
            x.table_host[b, : whole // x.P] = x.table_host[a, : whole // x.P]
            r = rows(x, b, whole, n)
            x.pk[:, :, r], x.pv[:, :, r] = x.K[b][:, :, whole:n], x.V[b][:, :, whole:n]
    x.table = torch.from_numpy(x.table_host).to(DEV)
    x.start = torch.tensor(start, dtype=torch.int32, device=DEV)
    x.shared_len = torch.tensor(shared, dtype=torch.int32, device=DEV)
    sizes = [b - a for a, b in zip(start, start[1:])]
    x.shared = pic.Shared.of(len(shared), max(sizes), min(max(shared + [1]), x.pages.table_cap * x.P))
    return x


def batch(hq, hkv, d, P, ctx, new, start, shared, **kw):
    return share(setup(hq, hkv, d, kw.pop("dtype", "bf16"), P, ctx, new, **kw), start, shared)


def workspace(x, n, max_ctx):
    return torch.full((max(pic.pic_page_shared_workspace_bytes(x.model, x.shared, x.B, n, max_ctx), 16),), 0xFF, dtype=torch.uint8,
                      device=DEV)


def decode(x, step=0, ws="query", scale=0.0, start="given", **kw):
    base = torch.where(x.len >= 0, x.len - step, x.len)
    pic.pic_page_shared_decode_attn(x.model, x.pages, x.shared, x.q, x.k, x.v, x.pk, x.pv, x.table, x.B,
                                    x.start if isinstance(start, str) else start, x.shared_len, base, step, x.max_ctx - step, x.out,
                                    workspace(x, 1, x.max_ctx) if isinstance(ws, str) else ws, scale, **kw)
    return x.out


def suffix(x, ws="query", scale=0.0, n_valid="given", **kw):
    pic.pic_page_shared_suffix_attn(x.model, x.pages, x.shared, x.q, x.k, x.v, x.pk, x.pv, x.table, x.B, x.start, x.shared_len, x.len,
                                    x.max_ctx, x.n, x.out, workspace(x, x.n, x.max_ctx) if isinstance(ws, str) else ws,
                                    x.n_valid if isinstance(n_valid, str) else n_valid, scale, **kw)
    return x.out


def starts(sizes):
    return [0] + list(np.cumsum(sizes).tolist())
