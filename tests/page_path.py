"""Shared set-up of the paged-cache GPU tests: a batch whose cached tokens lie in shuffled pages, every
other row of the page buffers holding NaN, and the attention of its new tokens in 64 bits."""
import math
from types import SimpleNamespace

import numpy as np
import torch

import paper_2607_28069_amd as pic

DEV = "cuda"
SENTINEL = 7.5


def setup(hq, hkv, d, dtype, P, ctx, new, n=None, L=1, spare=3, seed=0, slack=0, pairing="half", value_scale=1.0):
    """ctx: cached tokens per request, negative for padding of the batch; new: its new tokens of the n a
    row of the inputs holds; slack: how far max_ctx lies above the longest context."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    f = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=dt)  # noqa: E731
    B, n = len(ctx), n or max(max(new), 1)
    x = SimpleNamespace(L=L, B=B, n=n, hq=hq, hkv=hkv, d=d, P=P, dtype=dtype, dt=dt, ctx=list(ctx), new=list(new))
    x.max_ctx = max(max(ctx), 0) + slack
    lens = [c + v if c >= 0 else 0 for c, v in zip(ctx, new)]
    need = [-(-m // P) for m in lens]
    n_pages = sum(need) + spare
    cap = -(-(x.max_ctx + n) // P)
    x.pages = pic.Pages.of(n_pages, P, cap)
    order, at = np.random.default_rng(seed).permutation(n_pages), 0
    table = np.full((B, cap), -1, np.int32)
    for b in range(B):
        table[b, : need[b]] = order[at: at + need[b]]
        at += need[b]
    x.table_host, x.table = table, torch.from_numpy(table).to(DEV)
    x.q, x.k, x.v = f(L, B, n, hq, d), f(L, B, n, hkv, d), f(L, B, n, hkv, d) * value_scale
    x.pk = torch.full((L, hkv, n_pages * P, d), float("nan"), dtype=dt, device=DEV)
    x.pv = x.pk.clone()
    x.K, x.V = [], []
    for b in range(B):   # [L, Hkv, tokens, D], the new tokens last
        k, v = f(L, hkv, max(ctx[b], 0), d), f(L, hkv, max(ctx[b], 0), d) * value_scale
        r = rows(x, b, 0, max(ctx[b], 0))
        x.pk[:, :, r], x.pv[:, :, r] = k, v
        m = new[b] if ctx[b] >= 0 else 0
        x.K.append(torch.cat([k, x.k[:, b, :m].transpose(1, 2)], 2))
        x.V.append(torch.cat([v, x.v[:, b, :m].transpose(1, 2)], 2))
    x.len = torch.tensor(list(ctx), dtype=torch.int32, device=DEV)
    x.n_valid = torch.tensor(list(new), dtype=torch.int32, device=DEV)
    x.out = torch.full((L, B, n, hq, d), SENTINEL, dtype=dt, device=DEV)
    x.model = pic.Model.of(L, hq, hkv, d, dtype, 5e5, pairing)
    x.pairing = pairing
    return x


def rows(x, b, lo, hi):
    t = np.arange(lo, hi)
    return torch.from_numpy(x.table_host[b, t // x.P].astype(np.int64) * x.P + t % x.P).to(DEV)


def rope_table(x):
    mad = x.max_ctx + x.n
    t = torch.empty(pic.pic_rope_table_bytes(x.model, mad) // 4, dtype=torch.float32, device=DEV)
    pic.pic_rope_table_init(x.model, mad, t)
    return t, mad


def turn(x, rope):
    """The queries and new keys of `x` turned to their slots by rows of the table: keys as pic_rerotate_keys rounds
    them, in x.k and x.K, queries in 64 bits in x.q.  Returns the queries as pic_rerotate_keys rounds them."""
    table, mad = rope
    pos = torch.tensor([[max(c, 0) + i for i in range(x.n)] for c in x.ctx], dtype=torch.int32, device=DEV)
    interleaved = x.pairing == "interleaved"
    cs = table.view(-1, x.d // 2, 2)[pos.long()].double()[:, :, None]   # [B, n, 1, D / 2, 2], every layer's
    q = x.q.double()
    a, b = (q[..., ::2], q[..., 1::2]) if interleaved else (q[..., : x.d // 2], q[..., x.d // 2:])
    a, b = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
    rounded = x.q.clone()
    for t, h in ((rounded, x.hq), (x.k, x.hkv)):
        pic.pic_rerotate_keys(x.model, t, t, x.L * x.B * x.n, h, pos.repeat(x.L, 1, 1).contiguous(), table, mad)
    x.q = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    for i in range(x.B):
        m = x.new[i] if x.ctx[i] >= 0 else 0
        x.K[i] = torch.cat([x.K[i][:, :, : x.K[i].shape[2] - m], x.k[:, i, :m].transpose(1, 2)], 2)
    return rounded


def decode(x, step=0, n_splits=0, ws="query", rope=None, scale=0.0, **kw):
    """The contexts of `x` are base_len + step: base_len is given as the context less the step."""
    base = torch.where(x.len >= 0, x.len - step, x.len)
    if ws == "query":
        ws = torch.full((max(pic.pic_decode_workspace_bytes(x.model, x.B, x.max_ctx + 1, n_splits), 16),), 0xFF,
                        dtype=torch.uint8, device=DEV)
    head = (x.model, x.pages, x.q, x.k, x.v, x.pk, x.pv, x.table, x.B, base, step, x.max_ctx - step)
    if rope:
        pic.pic_page_decode_attn_rope(*head, *rope, x.out, ws, n_splits, scale, **kw)
    else:
        pic.pic_page_decode_attn(*head, x.out, ws, n_splits, scale, **kw)
    return x.out


def suffix(x, ws="query", rope=None, scale=0.0, n_valid="given", **kw):
    if ws == "query":
        ws = torch.full((max(pic.pic_prefill_workspace_bytes(x.model, x.B, x.n, x.max_ctx), 16),), 0xFF,
                        dtype=torch.uint8, device=DEV)
    head = (x.model, x.pages, x.q, x.k, x.v, x.pk, x.pv, x.table, x.B, x.len, x.max_ctx, x.n)
    nv = x.n_valid if isinstance(n_valid, str) else n_valid
    if rope:
        pic.pic_page_suffix_attn_rope(*head, *rope, x.out, ws, nv, scale, **kw)
    else:
        pic.pic_page_suffix_attn(*head, x.out, ws, nv, scale, **kw)
    return x.out


def reference(x, scale=0.0):
    """(out, sum of p |v|, largest sum of |q k| scale) in 64 bits, [L, B, n, Hq, D] and scalars per row;
    rows of padding hold the sentinel."""
    sc = scale or 1 / math.sqrt(x.d)
    rep = x.hq // x.hkv
    out = torch.full((x.L, x.B, x.n, x.hq, x.d), SENTINEL, dtype=torch.float64, device=DEV)
    mag, score = torch.zeros_like(out), torch.zeros_like(out[..., :1])
    for b in range(x.B):
        m = x.new[b] if x.ctx[b] >= 0 else 0
        if m == 0:
            continue
        K, V = x.K[b].double(), x.V[b].double()
        q = x.q[:, b, :m].double().view(x.L, m, x.hkv, rep, x.d).permute(0, 2, 1, 3, 4).reshape(x.L, x.hkv, m * rep, x.d)
        s = (q @ K.transpose(-1, -2) * sc).view(x.L, x.hkv, m, rep, -1)
        a = (q.abs() @ K.abs().transpose(-1, -2) * sc).view(x.L, x.hkv, m, rep, -1)
        pos = x.ctx[b] + torch.arange(m, device=DEV)
        hide = torch.arange(K.shape[2], device=DEV) > pos[:, None]
        p = s.masked_fill(hide[:, None], -math.inf).softmax(-1)
        seen = ~hide[:, None]
        put = lambda y: y.permute(0, 2, 1, 3, 4).reshape(x.L, m, x.hq, -1)  # noqa: E731
        pv = p.view(x.L, x.hkv, m * rep, -1)
        out[:, b, :m] = put((pv @ V).view(x.L, x.hkv, m, rep, x.d))
        mag[:, b, :m] = put((pv @ V.abs()).view(x.L, x.hkv, m, rep, x.d))
        score[:, b, :m] = put((a * seen).amax(-1, keepdim=True))
    return out, mag, score


def check(x, scale=0.0, decoded=False, turned=False):
    """Outputs within the rounding of their arithmetic (u = 2^-24 the float32 half step, T the keys):
      float32   scores: D products summed, off by D u sum|q k| scale; probabilities off by that
                relative to themselves, in numerator and denominator; sums of T terms by T u each
      bf16      besides: the output rounded (2^-8); in a prefill also each probability (2^-8), which the
                numerator and the denominator see, and a split's share (2^-11 in half precision, whose
                smallest step is 2^-24 of the row's largest value); in a decode the probabilities are two
                bfloat16 terms (2^-16)
      turned    (x.q in 64 bits) queries turned in float32 and then two bfloat16 terms: 2^-16 of each, and of
                the float32 turn 2^-22 of its pair, so scores off by 2^-16 sum|q k| scale
    rows of padding untouched, page rows holding exactly the tokens, everything else as it was."""
    ref, mag, score = reference(x, scale)
    got = x.out.double()
    T = max([k.shape[2] for k in x.K] + [1])
    u = 2.0 ** -24
    tol = (2 * x.d * u * score + 2 * (T + 16) * u) * mag + 1e-30
    if x.dtype == "bf16":
        tol = tol + (2 * 2.0 ** -16 if decoded else 2 * 2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()
        tol = tol + (0 if decoded else 2.0 ** -25 * mag.sum(-1, keepdim=True))
    if turned:
        tol = tol + 2 * 2.0 ** -16 * (1 + 2.0 ** -4) * score * mag
    pad = torch.ones((x.B, x.n), dtype=torch.bool, device=DEV)
    for b in range(x.B):
        pad[b, : x.new[b] if x.ctx[b] >= 0 else 0] = False
    assert (x.out[:, pad] == SENTINEL).all(), "rows of padding were written"
    live = ~pad
    assert torch.isfinite(got[:, live]).all(), "not finite: a slot nobody sees was read"
    err = (got - ref).abs()
    bad = (err > tol)[:, live]
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs off, worst {float((err / tol)[:, live].max()):.2f} of the bound"
    if live.any():
        rel = float(err[:, live].norm() / ref[:, live].norm())
        # float32 sums wander by the root of their terms; each of the one or two bf16 roundings is 2^-8 / sqrt(3)
        # in the 2-norm, independent of one another (a share's 2^-11 in what two leave of 2^-8)
        most = 2 * u * (math.sqrt(x.d) * float(score.max()) + math.sqrt(T) + 8)
        most += 2.0 ** -8 / (math.sqrt(3) if decoded else 1) if x.dtype == "bf16" else 0
        most += 2 * 2.0 ** -16 * float(score.max()) if turned else 0
        assert rel <= most, (rel, most)
    check_pages(x)


def check_pages(x):
    want_k, want_v = torch.full_like(x.pk, float("nan")), torch.full_like(x.pv, float("nan"))
    for b in range(x.B):
        r = rows(x, b, 0, x.K[b].shape[2])
        want_k[:, :, r], want_v[:, :, r] = x.K[b], x.V[b]
    i = torch.int32 if x.dtype == "f32" else torch.int16
    for got, want in ((x.pk, want_k), (x.pv, want_v)):
        assert (got.view(i) == want.view(i)).all(), "page rows differ from the tokens they should hold"


def contiguous(x, cap=None):
    """The cached tokens (the new ones left out) as caches [L][B][Hkv][cap][D]; every other slot NaN."""
    cap = cap or x.pages.table_cap * x.P
    ck = torch.full((x.L, x.B, x.hkv, cap, x.d), float("nan"), dtype=x.dt, device=DEV)
    cv = ck.clone()
    for b in range(x.B):
        m = x.ctx[b]
        ck[:, b, :, :m], cv[:, b, :, :m] = x.K[b][:, :, :m], x.V[b][:, :, :m]
    return ck, cv, cap
