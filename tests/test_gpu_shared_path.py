"""A batch of forked requests served as a loop would: page tables grown on the device, the copies that asks for, queries and
keys normalised and turned out of one projection, attention with the prefixes read once; first several tokens per
request, then single ones, captured and replayed.  Tables against the host's calls, numbers against 64 bits."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, SENTINEL, check, rows
from test_gpu_qk_norm import reference as turned, tolerance

pytestmark = pytest.mark.gpu


class Loop:
    """Request 0 holds a prefix and is padding of the batch, 1 to 5 are its forks; 6 has another, 7 is its fork; 8 starts from
    nothing, in no group."""

    def __init__(self, hq, hkv, d, P, pairing, seed=0):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.B, self.L, self.shared = 9, 2, [300, 150]
        held = [300, 300, 300, 300, 300, 300, 150, 150, 0]
        cap, n_pages = 512 // P, 100 if P == 16 else 40
        x = self.x = SimpleNamespace(L=self.L, B=self.B, n=1, hq=hq, hkv=hkv, d=d, P=P, dtype="bf16", dt=torch.bfloat16, pairing=pairing,
                                     max_ctx=440, ctx=[-1] + held[1:], new=[0] * self.B)
        x.model = pic.Model.of(self.L, hq, hkv, d, "bf16", 1e4, pairing)
        x.pages = pic.Pages.of(n_pages, P, cap)
        self.refs, x.table_host = np.zeros(n_pages, np.int32), np.full((self.B, cap), -1, np.int32)
        pic.pic_page_grow(x.pages, self.refs, x.table_host, [0] * self.B, [300, 0, 0, 0, 0, 0, 150, 0, 0])
        for src, dst in [(0, b) for b in range(1, 6)] + [(6, 7)]:
            pic.pic_page_fork(x.pages, self.B, self.refs, x.table_host, src, held[src], dst)
        x.pk = torch.full((self.L, hkv, n_pages * P, d), float("nan"), dtype=x.dt, device=DEV)
        x.pv = x.pk.clone()
        x.K, x.V = [None] * self.B, [None] * self.B
        for src, forks in ((0, range(6)), (6, (6, 7)), (8, (8,))):
            k, v = self.rand(self.L, hkv, held[src], d), self.rand(self.L, hkv, held[src], d)
            r = rows(x, src, 0, held[src])
            x.pk[:, :, r], x.pv[:, :, r] = k, v
            for b in forks:
                x.K[b], x.V[b] = k, v
        i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
        self.d_refs, x.table, self.len = i32(self.refs), i32(x.table_host), i32(x.ctx)
        self.groups = pic.Shared.of(2, 6, 300)
        self.start, self.shared_len = i32([0, 6, 8]), i32(self.shared)
        self.w = [1 + 0.3 * torch.randn(self.L, d, generator=self.g, device=DEV) for _ in "qk"]
        self.how = pic.QkNorm.of(*self.w, eps=1e-6)
        self.mad = 512
        self.rope = torch.empty(pic.pic_rope_table_bytes(x.model, self.mad) // 4, dtype=torch.float32, device=DEV)
        pic.pic_rope_table_init(x.model, self.mad, self.rope)
        self.pairs, self.ready, self.result = i32(np.zeros((self.B, 2))), i32(np.zeros(self.B)), i32([0, 0, 0])

    def rand(self, *s):
        return torch.randn(s, generator=self.g, device=DEV, dtype=torch.bfloat16)

    def inputs(self, n):
        """Buffers of calls with n tokens per request; the workspaces are those of the longest context."""
        x = self.x
        x.n = n
        self.qkv = self.rand(self.L, self.B, n, (x.hq + 2 * x.hkv) * x.d)
        x.q, x.k, x.v = (torch.zeros((self.L, self.B, n, h, x.d), dtype=x.dt, device=DEV) for h in (x.hq, x.hkv, x.hkv))
        x.out = torch.full((self.L, self.B, n, x.hq, x.d), SENTINEL, dtype=x.dt, device=DEV)
        self.n_valid = torch.full((self.B,), n, dtype=torch.int32, device=DEV)
        ws = pic.pic_page_shared_workspace_bytes(x.model, self.groups, self.B, n, x.max_ctx)
        self.ws = torch.full((ws,), 0xFF, dtype=torch.uint8, device=DEV)
        self.grow_ws = torch.empty(pic.pic_page_grow_workspace_bytes(x.pages, self.B, n), dtype=torch.uint8, device=DEV)

    def step(self, max_ctx):
        """All of it on the device: the new tokens in self.qkv to x.out and the pages, lengths moved on."""
        x = self.x
        heads = self.qkv.unflatten(-1, (x.hq + 2 * x.hkv, x.d))
        pic.pic_page_grow_async(x.pages, self.B, self.d_refs, x.table, self.len, x.n, self.pairs, self.ready, self.result, self.grow_ws,
                                self.n_valid)
        pic.pic_page_copy_async(x.model, x.pages, x.pk, x.pv, self.pairs, self.B)
        pic.pic_qk_norm_rope(x.model, self.how, heads[..., : x.hq, :], heads[..., x.hq: x.hq + x.hkv, :], heads[..., x.hq + x.hkv:, :],
                             self.B, x.n, self.rope, self.mad, x.q, x.k, x.v, base_len=self.ready, max_base_len=max_ctx,
                             n_valid=self.n_valid)
        head = (x.model, x.pages, self.groups, x.q, x.k, x.v, x.pk, x.pv, x.table, self.B, self.start, self.shared_len, self.ready)
        if x.n == 1:
            pic.pic_page_shared_decode_attn(*head, 0, max_ctx, x.out, self.ws)
        else:
            pic.pic_page_shared_suffix_attn(*head, max_ctx, x.n, x.out, self.ws, self.n_valid)
        self.len.add_(torch.where(self.ready >= 0, self.n_valid, 0).to(torch.int32))

    def right(self, n_valid):
        """After a step: the host's bookkeeping does the same, and every number is right."""
        x = self.x
        torch.cuda.synchronize()
        x.new = [0 if c < 0 else n for c, n in zip(x.ctx, n_valid)]
        frm = [max(c, 0) for c in x.ctx]
        pairs = pic.pic_page_grow(x.pages, self.refs, x.table_host, frm, [f + n for f, n in zip(frm, x.new)])
        assert self.result[:2].tolist() == [0, len(pairs)]
        assert (self.pairs[: len(pairs)].cpu().numpy() == pairs).all() and (self.pairs[len(pairs):] == -1).all()
        assert (self.d_refs.cpu().numpy() == self.refs).all() and (x.table.cpu().numpy() == x.table_host).all()
        assert self.ready.tolist() == x.ctx
        heads = self.qkv.unflatten(-1, (x.hq + 2 * x.hkv, x.d))
        freq = 1e4 ** (-2.0 * np.arange(x.d // 2) / x.d)
        for b, m in enumerate(x.new):
            pos = torch.arange(frm[b], frm[b] + m, device=DEV)
            for l in range(self.L):
                for got, at, w in ((x.q, 0, self.w[0]), (x.k, x.hq, self.w[1])):
                    raw = heads[l, b, :m, at: at + got.shape[3]]
                    want = turned(raw, w[l], 1e-6, pos, freq, 1.0, x.d, x.pairing, "keep")
                    size = turned(raw, w[l], 1e-6, pos, None, 1.0, x.d, "half" if x.pairing == "half" else "interleaved", "keep").abs()
                    if x.pairing == "half":
                        pair = size + size.roll(x.d // 2, -1)
                    else:
                        pair = (size[..., ::2] + size[..., 1::2]).repeat_interleave(2, -1)
                    assert ((got[l, b, :m].double() - want).abs() <= tolerance(want, pair, False)).all()
            assert (x.v[:, b, :m] == heads[:, b, :m, x.hq + x.hkv:]).all()
            x.K[b] = torch.cat([x.K[b], x.k[:, b, :m].transpose(1, 2)], 2)
            x.V[b] = torch.cat([x.V[b], x.v[:, b, :m].transpose(1, 2)], 2)
        check(x, decoded=self.groups.max_group * x.n * (x.hq // x.hkv) <= 64)
        x.ctx = [c if c < 0 else c + n for c, n in zip(x.ctx, x.new)]
        assert self.len.tolist() == x.ctx


@pytest.mark.parametrize("hq,hkv,d,P,pairing", [(8, 2, 128, 16, "half"), (6, 1, 64, 64, "interleaved"), (28, 4, 128, 16, "half")])
def test_served_together(hq, hkv, d, P, pairing):
    s = Loop(hq, hkv, d, P, pairing)
    x = s.x
    s.inputs(9)
    for n_valid in ([9, 9, 4, 0, 1, 9, 9, 2, 9], [0, 1, 9, 3, 0, 0, 1, 9, 6]):
        s.qkv.copy_(s.rand(*s.qkv.shape))
        x.out.fill_(SENTINEL)
        s.n_valid.copy_(torch.tensor(n_valid, dtype=torch.int32))
        s.step(x.max_ctx - 9)
        s.right(n_valid)
    s.inputs(1)
    ones = [1] * s.B
    for _ in range(2):   # eager, with a bound on the lengths that grows: the workspace of the longest serves
        s.qkv.copy_(s.rand(*s.qkv.shape))
        x.out.fill_(SENTINEL)
        s.step(max(x.ctx))
        s.right(ones)
    before = [t.clone() for t in (s.d_refs, x.table, s.len, x.pk, x.pv)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(x.max_ctx)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.step(x.max_ctx)
    for t, y in zip((s.d_refs, x.table, s.len, x.pk, x.pv), before):
        t.copy_(y)
    for it in range(20):
        s.qkv.copy_(s.rand(*s.qkv.shape))
        x.out.fill_(SENTINEL)
        if it % 7 == 6:   # an eager step in between, in the same workspaces
            s.step(x.max_ctx)
        else:
            g.replay()
        s.right(ones)
    # no page is left: nothing is stored, no length moves
    free = s.d_refs == 0
    s.d_refs[free] = 1
    while True:
        x.out.fill_(SENTINEL)
        before = [t.clone() for t in (s.d_refs, x.table, s.len, x.pk, x.pv)]
        g.replay()
        torch.cuda.synchronize()
        if s.result[0].item() != 0:
            break
    assert s.result[0].item() == -4 and s.ready.tolist() == [-1] * s.B and (x.out == SENTINEL).all()
    for t, y in zip((s.d_refs, x.table, s.len, x.pk, x.pv), before):
        assert (t.view(torch.int16) == y.view(torch.int16)).all()
