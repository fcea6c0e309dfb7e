"""The paged cache as a serving loop uses it: documents composed into pages, suffix prefill, sampling several
answers from one prompt (fork, copy on write, drafted tokens taken back), compaction; against the same
requests served from contiguous caches, in graphs, and on two streams at once."""
import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic
import synth
from synth import inputs as S

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Server:
    """Pages, bookkeeping and a contiguous twin of every request."""

    def __init__(self, shape, dtype, P, batch, n_pages, cap_tokens, L=2, seed=0):
        self.hq, self.hkv, self.d = shape
        self.L, self.B, self.P = L, batch, P
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.model = pic.Model.of(L, *shape, dtype, 5e5)
        self.pages = pic.Pages.of(n_pages, P, -(-cap_tokens // P))
        self.refs = np.zeros(n_pages, np.int32)
        self.table = np.full((batch, self.pages.table_cap), -1, np.int32)
        self.pk = torch.full((L, self.hkv, n_pages * P, self.d), float("nan"), dtype=self.dt, device=DEV)
        self.pv = self.pk.clone()
        self.cap = cap_tokens
        self.ck = torch.full((L, batch, self.hkv, cap_tokens, self.d), float("nan"), dtype=self.dt, device=DEV)
        self.cv = self.ck.clone()
        self.len = np.zeros(batch, np.int32)
        self.mad = cap_tokens
        self.rope = torch.empty(pic.pic_rope_table_bytes(self.model, self.mad) // 4, dtype=torch.float32, device=DEV)
        pic.pic_rope_table_init(self.model, self.mad, self.rope)

    def rand(self, *s):
        return torch.randn(s, generator=self.g, device=DEV, dtype=self.dt)

    def grow(self, new_len):
        pairs = pic.pic_page_grow(self.pages, self.refs, self.table, self.len, new_len)
        pic.pic_page_copy(self.model, self.pages, self.pk, self.pv, pairs)
        return len(pairs)

    def dev(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)

    def compose(self, requests, offs, lens, cpos, pool_k, pool_v):
        T = int(lens.sum())
        blocks, ctx = pic.pic_plan_layout(requests, offs, lens, cpos, T)
        self.grow(ctx)
        at = pic.pic_page_blocks(self.pages, self.table, blocks)
        srt, starts = pic.pic_plan_shared(at)
        put = lambda b: self.dev(b.view(np.int32))  # noqa: E731
        pic.pic_compose_shared(self.model, pool_k, pool_v, T, put(srt), len(srt), self.dev(starts), len(starts) - 1, self.rope,
                               self.mad, self.pk, self.pv, 1, self.pages.n_pages * self.P)
        pic.pic_compose(self.model, pool_k, pool_v, T, put(blocks), len(blocks), self.rope, self.mad, self.ck, self.cv, self.B,
                        self.cap)
        self.len = np.asarray(ctx, np.int32).copy()

    def suffix(self, n, valid=None):
        valid = np.full(self.B, n) if valid is None else np.asarray(valid)
        self.grow(self.len + valid)
        q, k, v = self.rand(self.L, self.B, n, self.hq, self.d), *(self.rand(self.L, self.B, n, self.hkv, self.d) for _ in range(2))
        out = torch.zeros_like(q)
        mx = int(self.len.max())
        ws = torch.empty(max(pic.pic_prefill_workspace_bytes(self.model, self.B, n, mx), 16), dtype=torch.uint8, device=DEV)
        pic.pic_page_suffix_attn(self.model, self.pages, q, k, v, self.pk, self.pv, self.dev(self.table), self.B,
                                 self.dev(self.len), mx, n, out, ws, self.dev(valid))
        # the twin, request by request
        want = torch.zeros_like(q)
        for b in range(self.B):
            m = int(valid[b])
            if m:
                self._twin(b, q[:, b, :m], k[:, b, :m], v[:, b, :m], want[:, b, :m])
        self.len = self.len + valid.astype(np.int32)
        return out, want

    def _twin(self, b, q, k, v, want):
        m, L = q.shape[1], self.L
        ws = torch.empty(max(pic.pic_prefill_workspace_bytes(self.model, 1, m, int(self.len[b])), 16), dtype=torch.uint8, device=DEV)
        o = torch.empty((L, 1, m, self.hq, self.d), dtype=self.dt, device=DEV)
        ck, cv = self.ck[:, b: b + 1].contiguous(), self.cv[:, b: b + 1].contiguous()
        pic.pic_suffix_prefill_attn(self.model, q[:, None].contiguous(), k[:, None].contiguous(), v[:, None].contiguous(), ck, cv, 1,
                                    self.cap, self.dev(self.len[b: b + 1]), int(self.len[b]), m, o, ws)
        self.ck[:, b: b + 1], self.cv[:, b: b + 1] = ck, cv
        want.copy_(o[:, 0])

    def decode(self, active=None):
        active = np.ones(self.B, bool) if active is None else np.asarray(active)
        self.grow(self.len + active)
        q, k, v = self.rand(self.L, self.B, self.hq, self.d), *(self.rand(self.L, self.B, self.hkv, self.d) for _ in range(2))
        out, want = torch.zeros_like(q), torch.zeros_like(q)
        mx = int(self.len.max())
        ws = torch.empty(max(pic.pic_decode_workspace_bytes(self.model, self.B, mx + 1), 16), dtype=torch.uint8, device=DEV)
        pic.pic_page_decode_attn(self.model, self.pages, q, k, v, self.pk, self.pv, self.dev(self.table), self.B,
                                 self.dev(np.where(active, self.len, -1)), 0, mx, out, ws)
        for b in np.nonzero(active)[0]:
            self._twin(b, q[:, b: b + 1], k[:, b: b + 1], v[:, b: b + 1], want[:, b: b + 1])
        self.len = self.len + active.astype(np.int32)
        return out, want

    def same_cache(self):
        i = torch.int32 if self.dt == torch.float32 else torch.int16
        for b in range(self.B):
            t = np.arange(self.len[b])
            row = torch.from_numpy(self.table[b, t // self.P].astype(np.int64) * self.P + t % self.P).to(DEV)
            for p, c in ((self.pk, self.ck), (self.pv, self.cv)):
                assert (p[:, :, row].view(i) == c[:, b, :, : self.len[b]].view(i)).all(), f"request {b}"


def close(got, want, dt):
    """Two results of the same inputs: float32 sums in another order; bf16 the roundings of either (three of
    2^-8 relative to the values averaged at most, an average of at most ~1 here)."""
    err = (got.double() - want.double()).abs()
    if dt == torch.float32:
        assert float(err.max()) < 1e-5
    else:
        assert float(err.norm() / want.double().norm()) < 2 * 2.0 ** -8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [16, 64])
def test_serving_with_pages(dtype, P):
    rng = np.random.default_rng(3)
    lens = np.array([100, 64, 37, 250, 8])
    offs = np.concatenate([[0], np.cumsum(lens)[:-1]])
    s = Server((8, 2, 64), dtype, P, batch=5, n_pages=6000 // P, cap_tokens=1024)
    T = int(lens.sum())
    pool_k, pool_v = s.rand(2, 2, T, 64), s.rand(2, 2, T, 64)
    # three requests over shared documents; two places of the batch stay empty for now
    s.compose([[4, 0, 2], [3, 1], [0, 1, 2, 3, 4], [], []], offs, lens, np.zeros(5), pool_k, pool_v)
    s.same_cache()
    close(*s.suffix(23, valid=[23, 7, 0, 0, 0]), s.dt)
    close(*s.suffix(70, valid=[0, 1, 70, 0, 0]), s.dt)
    s.same_cache()
    # one prompt sampled three times: forks share its pages, and copy the last one when they write
    for dst in (3, 4):
        pic.pic_page_fork(s.pages, s.B, s.refs, s.table, 0, int(s.len[0]), dst)
        s.len[dst] = s.len[0]
        s.ck[:, dst], s.cv[:, dst] = s.ck[:, 0], s.cv[:, 0]
    used = int((s.refs > 0).sum())
    for step in range(20):
        close(*s.decode(active=[True, step % 2 == 0, True, True, step < 11]), s.dt)
    s.same_cache()
    assert int((s.refs > 0).sum()) <= used + 2 + 5 * (20 // P + 1)   # the prompt's whole pages are held once
    # drafted tokens: six at once, of which two are kept
    close(*s.suffix(6, valid=[6, 0, 6, 6, 0]), s.dt)
    for b in (0, 2, 3):
        s.len[b] -= 4
        pic.pic_page_free(s.pages, s.B, s.refs, s.table, b, int(s.len[b]))
    close(*s.decode(), s.dt)
    # requests leave, the rest moves together, and goes on
    for b in (1, 3):
        pic.pic_page_free(s.pages, s.B, s.refs, s.table, b)
        s.len[b] = 0
    pairs, n_used = pic.pic_page_compact(s.pages, s.B, s.refs, s.table)
    pic.pic_page_copy(s.model, s.pages, s.pk, s.pv, pairs)
    assert len(pairs) > 0 and s.table.max() < n_used
    s.same_cache()
    close(*s.decode(active=[True, False, True, False, True]), s.dt)
    s.same_cache()


def test_documents_of_a_workload_in_pages():
    """The 1-layer Llama shape: composed pages hold pic_compose's bits, and the suffix over them gives what it gives
    over the contiguous cache."""
    w = synth.get("llama8b_1layer")
    lay = S.pool_layout(w)
    dev, dt = torch.device("cuda", 0), torch.bfloat16
    s = Server((w.n_q_heads, w.n_kv_heads, w.head_dim), "bf16", 64, w.batch, 400, 4608, L=1)
    pool = [S.device_normal(w, name, (w.n_kv_heads, lay.pool_tokens, w.head_dim), 0, dev, dt)[None].contiguous()
            for name in ("pool_k", "pool_v")]
    blocks, ctx = pic.pic_plan_layout(lay.requests, lay.doc_offset, lay.doc_len, lay.doc_compile_pos, lay.pool_tokens)
    s.grow(ctx)
    at = pic.pic_page_blocks(s.pages, s.table, blocks)
    pic.pic_compose(s.model, *pool, lay.pool_tokens, s.dev(at.view(np.int32)), len(at), s.rope, s.mad, s.pk, s.pv, 1, 400 * 64)
    pic.pic_compose(s.model, *pool, lay.pool_tokens, s.dev(blocks.view(np.int32)), len(blocks), s.rope, s.mad, s.ck, s.cv, s.B, s.cap)
    s.len = np.asarray(ctx, np.int32).copy()
    s.same_cache()
    n, mx = w.n_suffix, int(ctx.max())
    q, k, v = s.rand(1, s.B, n, s.hq, s.d), s.rand(1, s.B, n, s.hkv, s.d), s.rand(1, s.B, n, s.hkv, s.d)
    s.grow(s.len + n)
    ws = torch.empty(max(pic.pic_prefill_workspace_bytes(s.model, s.B, n, mx), 16), dtype=torch.uint8, device=DEV)
    out, want = torch.empty_like(q), torch.empty_like(q)
    pic.pic_page_suffix_attn(s.model, s.pages, q, k, v, s.pk, s.pv, s.dev(s.table), s.B, s.dev(s.len), mx, n, out, ws)
    pic.pic_suffix_prefill_attn(s.model, q, k, v, s.ck, s.cv, s.B, s.cap, s.dev(s.len), mx, n, want, ws)
    # (two outputs rounded by 2^-8, root mean square 2^-8 / sqrt(3), and the contiguous call's bf16 shares)
    assert float((out.double() - want.double()).norm() / want.double().norm()) <= 2.0 ** -8 * 1.05
    s.len = s.len + n
    s.same_cache()


def _calls(x, out, ws):
    """A suffix, a few drafted tokens, a decode step and a page copy over the pages of `x` (see page_path.setup)."""
    pic.pic_page_suffix_attn(x["m"], x["pg"], x["q"], x["k"], x["v"], x["pk"], x["pv"], x["table"], x["B"], x["len"], x["mx"], x["n"],
                             out[0], ws[0], x["nv"])
    pic.pic_page_suffix_attn(x["m"], x["pg"], x["q3"], x["k3"], x["v3"], x["pk"], x["pv"], x["table"], x["B"], x["len"], x["mx"], 3,
                             out[1], ws[1])
    pic.pic_page_decode_attn(x["m"], x["pg"], x["q1"], x["k1"], x["v1"], x["pk"], x["pv"], x["table"], x["B"], x["len"], 0, x["mx"],
                             out[2], ws[2])
    pic.pic_page_copy(x["m"], x["pg"], x["pk"], x["pv"], x["pairs"])


def _state(seed, B=3, n=33, P=16, hq=16, hkv=4, d=128):
    from page_path import setup
    s = setup(hq, hkv, d, "bf16", P, [2500, 40, -1][:B], [n, 5, n][:B], n=n, L=2, seed=seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    f = lambda *z: torch.randn(z, generator=g, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    x = dict(m=s.model, pg=s.pages, q=s.q, k=s.k, v=s.v, pk=torch.nan_to_num(s.pk), pv=torch.nan_to_num(s.pv), table=s.table, B=B,
             len=s.len, mx=s.max_ctx, n=n, nv=s.n_valid, q3=f(2, B, 3, hq, d), k3=f(2, B, 3, hkv, d), v3=f(2, B, 3, hkv, d),
             q1=f(2, B, hq, d), k1=f(2, B, hkv, d), v1=f(2, B, hkv, d))
    free = sorted(set(range(s.pages.n_pages)) - set(s.table_host.ravel().tolist()))
    x["pairs"] = [[int(s.table_host[0, 0]), free[0]], [int(s.table_host[1, 1]), free[1]]]   # onto pages nobody reads
    out = [torch.zeros_like(x[i]) for i in ("q", "q3", "q1")]
    m = x["m"]
    ws = [torch.empty(max(b, 16), dtype=torch.uint8, device=DEV) for b in (
        pic.pic_prefill_workspace_bytes(m, B, n, x["mx"]), pic.pic_prefill_workspace_bytes(m, B, 3, x["mx"]),
        pic.pic_decode_workspace_bytes(m, B, x["mx"] + 1))]
    return x, out, ws


def test_graph_replays_match_eager():
    x, out, ws = _state(1)
    keep = x["pk"].clone(), x["pv"].clone()
    _calls(x, out, ws)
    want = [o.clone() for o in out] + [x["pk"].clone(), x["pv"].clone()]
    x["pk"].copy_(keep[0]), x["pv"].copy_(keep[1])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        _calls(x, out, ws)
    for rep in range(4):
        for o in out:
            o.zero_()
        for w in ws:
            w.fill_(0xFF)
        x["pk"].copy_(keep[0]), x["pv"].copy_(keep[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out + [x["pk"], x["pv"]], want):
            assert torch.equal(a, b), rep
        _calls(x, out, ws)   # the program's own eager work in between
    # lengths are read on replay: a request that has left is left alone
    x["len"][0] = -1
    for o in out:
        o.zero_()   # (what `want` holds where padding left it)
    graph.replay()
    torch.cuda.synchronize()
    for o, w in zip(out, want):
        assert (o[:, 0] == 0).all() and torch.equal(o[:, 1], w[:, 1])


def test_two_streams_at_once():
    states = [_state(seed) for seed in (5, 6)]
    want = []
    for x, out, ws in states:
        keep = x["pk"].clone(), x["pv"].clone()
        _calls(x, out, ws)
        want.append([o.clone() for o in out] + [x["pk"].clone(), x["pv"].clone()])
        x["pk"].copy_(keep[0]), x["pv"].copy_(keep[1])
        for o in out:
            o.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(3):
        for (x, out, ws), st in zip(states, streams):
            with torch.cuda.stream(st):
                _calls(x, out, ws)
    torch.cuda.synchronize()
    for (x, out, ws), w in zip(states, want):
        for a, b in zip(out + [x["pk"], x["pv"]], w):
            assert torch.equal(a, b)
