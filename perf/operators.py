"""The operators of the paged cache: what is measured of them, and their plain forms.

A program that serves from a paged cache holds K and V pages [layers][kv heads][n_pages * page_tokens][head_dim]
and a page table [batch][table_cap]: slot t of request b is row table[b][t // P] * P + t % P of every (layer, kv head)
stream, P = page_tokens.  It appends and attends:

  decode   one new token per request: its K/V go to slot p = base_len[b] + step, its query heads attend over
           slots [0, p]; requests with a negative base_len are padding of the batch and stay as they are
  suffix   n_suffix new tokens per request after ctx_len[b] cached ones, token i at slot ctx_len[b] + i, which
           attends over [0, ctx_len[b] + i]; tokens from n_valid[b] on are padding
  copy     pages copied onto other pages in every layer and kv head, K and V: the copies that a fork's first
           write or a compaction asks for

"rope" cases bring queries and new keys unrotated.  Plain forms are elementary torch operations in 32 bits (angles
in 64); exact() is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
# (query heads, kv heads, head_dim, rope theta): the attention shapes of perf/cases.py
SHAPES = {
    "llama8b": (32, 8, 128, 5e5),
    "qwen7b": (28, 4, 128, 1e6),
    "llama_hd64": (32, 8, 64, 5e5),
    "small": (16, 4, 64, 1e4),
    "tiny": (4, 2, 64, 1e4),
}


def listed():
    return [
        # the tiny float32 request's decode step: one workgroup's worth of work, all latency
        dict(name="decode_tiny_f32", kind="decode", shape="tiny", dtype="f32", layers=1, batch=1, ctx=288, ragged=0.0,
             step=1, idle=0, page=16, rope=False, pairing="half"),
        # one user's 10K context in a 32-layer model, one layer of the step: short, split over the length
        dict(name="decode_lone_10k", kind="decode", shape="llama8b", dtype="bf16", layers=1, batch=1, ctx=10496, ragged=0.0,
             step=3, idle=0, page=64, rope=False, pairing="half"),
        # 16 such requests, tokens rotated by the call
        dict(name="decode_llama_16x10k_rope", kind="decode", shape="llama8b", dtype="bf16", layers=1, batch=16, ctx=10496,
             ragged=0.0, step=17, idle=0, page=64, rope=True, pairing="half"),
        # a full decode batch: 64 requests of up to 16K, uneven
        dict(name="decode_llama_64x16k", kind="decode", shape="llama8b", dtype="bf16", layers=1, batch=64, ctx=16384,
             ragged=0.25, step=100, idle=0, page=64, rope=False, pairing="half"),
        # long uneven contexts in pages of 16 tokens, seven query heads per kv head
        dict(name="decode_qwen_32k_page16", kind="decode", shape="qwen7b", dtype="bf16", layers=1, batch=8, ctx=33001,
             ragged=0.5, step=7, idle=0, page=16, rope=False, pairing="half"),
        # a padded batch of short chats at head_dim 64, two layers in one call, interleaved rotary pairs
        dict(name="decode_hd64_padded", kind="decode", shape="llama_hd64", dtype="bf16", layers=2, batch=48, ctx=701,
             ragged=0.9, step=0, idle=11, page=32, rope=True, pairing="interleaved"),
        # one layer of a batch's suffix prefill: 128 query tokens over about 10K of context
        dict(name="suffix_llama_16x10k", kind="suffix", shape="llama8b", dtype="bf16", layers=1, batch=16, ctx=10368,
             ragged=0.0, suffix=128, pad=0.0, page=64, rope=False, pairing="half"),
        # 32K contexts of uneven length, 256 query tokens, wide pages
        dict(name="suffix_qwen_32k", kind="suffix", shape="qwen7b", dtype="bf16", layers=1, batch=8, ctx=32749, ragged=0.25,
             suffix=256, pad=0.0, page=128, rope=False, pairing="half"),
        # follow-up turns of uneven length, padded to the longest, tokens rotated by the call, pages of 16
        dict(name="suffix_hd64_padded_rope", kind="suffix", shape="llama_hd64", dtype="bf16", layers=1, batch=5, ctx=4161,
             ragged=0.5, suffix=67, pad=0.9, page=16, rope=True, pairing="half"),
        # a small float32 model
        dict(name="suffix_small_f32", kind="suffix", shape="small", dtype="f32", layers=1, batch=4, ctx=2077, ragged=0.25,
             suffix=61, pad=0.0, page=32, rope=False, pairing="half"),
        # one answer sampled 16 times: 15 forks' first write copies the last page, in all 32 layers
        dict(name="copy_fork_16", kind="copy", shape="llama8b", dtype="bf16", layers=32, pairs=15, pages=64, page=64),
        # a pool compacted after requests have left: 208 of 512 pages move, in all 28 layers
        dict(name="copy_compact", kind="copy", shape="qwen7b", dtype="bf16", layers=28, pairs=208, pages=512, page=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "suffix", "suffix", "copy"])
    f32 = rng.random() < 0.2
    shape = rng.choice(["tiny", "small"]) if f32 else rng.choice(["llama8b", "llama8b", "qwen7b", "llama_hd64"])
    hq, hkv, d, _ = SHAPES[shape]
    c = dict(kind=kind, shape=shape, dtype="f32" if f32 else "bf16", page=rng.choice([16, 32, 64, 64, 128, 256]))
    if kind == "copy":
        layers = _log(rng, 1, 32)
        page_bytes = layers * hkv * c["page"] * d * (4 if f32 else 2)
        pairs = _log(rng, 1, max(1, min(2000, int(7.5e8 / page_bytes))))
        return dict(c, layers=layers, pairs=pairs, pages=2 * pairs + rng.randint(0, pairs))
    rope = not f32 and rng.random() < 0.4
    c.update(rope=rope, pairing=rng.choice(["half", "half", "interleaved"]) if rope else "half", layers=rng.choice([1, 1, 1, 2]),
             ragged=rng.choice([0.0, 0.0, 0.25, 0.5, 0.9]))
    if kind == "decode":
        batch = _log(rng, 1, 4 if f32 else 64)
        top = min(4096 if f32 else 33000, int(3.5e9 / (hkv * d * 4 * batch * c["layers"])))
        return dict(c, batch=batch, ctx=_log(rng, 1, top), step=rng.randint(0, 255),
                    idle=rng.choice([0, 0, rng.randint(0, batch - 1)]))
    batch, suffix = (_log(rng, 1, 4), _log(rng, 1, 64)) if f32 else (_log(rng, 1, 16), _log(rng, 1, 256))
    top = min(2048 if f32 else 32768, int((2e9 if f32 else 9e11) / (4 * hq * d * batch * suffix * c["layers"])))
    return dict(c, batch=batch, ctx=_log(rng, 1, max(top, 2)), suffix=suffix, pad=rng.choice([0.0, 0.0, 0.5, 0.9]))


# ------------------------------------------------------------------------------------------
# layouts: lengths are fixed by the case, so that the work does not depend on the seed; which page
# holds what does
# ------------------------------------------------------------------------------------------

def _ctx(case):
    """Tokens each request has cached: the longest is case["ctx"], the others up to a share `ragged` shorter;
    -1 for the padding of a decode batch."""
    r = random.Random(3)
    c = [case["ctx"]] + [case["ctx"] - int(r.random() * case["ragged"] * case["ctx"]) for _ in range(case["batch"] - 1)]
    for b in r.sample(range(1, case["batch"]), case.get("idle", 0)):
        c[b] = -1
    return c


def _valid(case):
    """New tokens of each request of a suffix batch (0 among them where the padding is deep)."""
    r = random.Random(4)
    n = case["suffix"]
    v = [n] + [n - int(r.random() * case["pad"] * (n + 1)) for _ in range(case["batch"] - 1)]
    if case["pad"] > 0.8 and len(v) > 2:
        v[-1] = 0
    return v


def _lens(case):
    """Slots each request occupies once the new tokens are stored."""
    if case["kind"] == "decode":
        return [c + case["step"] + 1 if c >= 0 else 0 for c in _ctx(case)]
    return [c + v for c, v in zip(_ctx(case), _valid(case))]


def _es(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    hq, hkv, d, _ = SHAPES[case["shape"]]
    L, es = case["layers"], _es(case)
    if case["kind"] == "copy":
        return {"bytes": 4 * case["pairs"] * L * hkv * case["page"] * d * es, "flops": 0}
    lens = _lens(case)
    new = [1 if n else 0 for n in lens] if case["kind"] == "decode" else _valid(case)
    # a request without new tokens is not read
    cached = sum(n - v for n, v in zip(lens, new) if v)
    seen = sum(v * (n - v) + v * (v + 1) // 2 for n, v in zip(lens, new))
    return {"bytes": L * d * es * (hkv * (2 * cached + 4 * sum(new)) + 2 * hq * sum(new)), "flops": 4 * L * hq * d * seen}


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------

def _randn(seed, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 777)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    return lambda *shape: torch.randn(shape, generator=g, device=DEV, dtype=dt)


def _dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype)).to(DEV)


def prepare(case, seed):
    hq, hkv, d, theta = SHAPES[case["shape"]]
    L, P, randn, r = case["layers"], case["page"], _randn(seed, case["dtype"]), np.random.default_rng(seed)
    s = dict(case=dict(case), theta=theta, scale=1.0 / math.sqrt(d), shape=(L, hq, hkv, d))
    if case["kind"] == "copy":
        at = r.permutation(case["pages"])
        s["pairs"] = np.ascontiguousarray(at[: 2 * case["pairs"]].reshape(-1, 2).astype(np.int32))
        s["n_pages"] = case["pages"]
        s["src"], s["dst"] = _dev(s["pairs"][:, 0], np.int64), _dev(s["pairs"][:, 1], np.int64)
    else:
        B, lens, ctx = case["batch"], _lens(case), _ctx(case)
        n = 1 if case["kind"] == "decode" else case["suffix"]
        need = [-(-x // P) for x in lens]
        s["n_pages"] = sum(need) + max(1, sum(need) // 16)
        order, table, at = r.permutation(s["n_pages"]), np.full((B, max(need)), -1, np.int32), 0
        for b in range(B):
            table[b, : need[b]] = order[at: at + need[b]]
            at += need[b]
        s.update(B=B, n=n, max_len=max(lens), max_ctx=max(ctx), table=_dev(table), table_cap=table.shape[1], ctx=_dev(ctx))
        # (request, token) of every new token that is one, and its slot
        off = case["step"] if case["kind"] == "decode" else 0
        new = [1 if c >= 0 else 0 for c in ctx] if case["kind"] == "decode" else _valid(case)
        at = [(b, i, ctx[b] + off + i) for b in range(B) for i in range(new[b])]
        s["at_b"], s["at_i"], s["at_pos"] = (_dev([x[j] for x in at], np.int64) for j in range(3))
        if case["kind"] == "suffix":
            s["n_valid"] = _dev(new)
        s["q"], s["k"], s["v"] = randn(L, B, n, hq, d), randn(L, B, n, hkv, d), randn(L, B, n, hkv, d)
        s["out"] = randn(L, B, n, hq, d) / 32   # what padding rows hold before and after: the size of an average of values
    s["pages_k"], s["pages_v"] = randn(L, hkv, s["n_pages"] * P, d), randn(L, hkv, s["n_pages"] * P, d)
    if own:
        import paper_2607_28069_amd as pic
        s["model"] = m = pic.Model.of(L, hq, hkv, d, case["dtype"], theta, case.get("pairing", "half"))
        s["pages"] = pic.Pages.of(s["n_pages"], P, s.get("table_cap", 0))
        if case["kind"] != "copy":
            bytes_ = (pic.pic_decode_workspace_bytes(m, B, s["max_len"]) if case["kind"] == "decode" else
                      pic.pic_prefill_workspace_bytes(m, B, n, s["max_ctx"]))
            s["ws"] = torch.empty(max(bytes_, 16), dtype=torch.uint8, device=DEV)
        if case.get("rope"):
            s["mad"] = s["max_ctx"] + (case["step"] if case["kind"] == "decode" else n)
            s["rope"] = torch.empty(pic.pic_rope_table_bytes(m, s["mad"]) // 4, dtype=torch.float32, device=DEV)
            pic.pic_rope_table_init(m, s["mad"], s["rope"])
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "copy":
        L, _, hkv, d = s["shape"]
        for x in (s["pages_k"], s["pages_v"]):
            p = x.view(L, hkv, s["n_pages"], -1)
            p[:, :, s["dst"]] = p[:, :, s["src"]]
        return {"pages_k": s["pages_k"], "pages_v": s["pages_v"]}
    return _attend(s, case)


def _run_own(s, case):
    import paper_2607_28069_amd as pic
    kind = case["kind"]
    if kind == "copy":
        pic.pic_page_copy(s["model"], s["pages"], s["pages_k"], s["pages_v"], s["pairs"])
        return {"pages_k": s["pages_k"], "pages_v": s["pages_v"]}
    head = (s["model"], s["pages"], s["q"], s["k"], s["v"], s["pages_k"], s["pages_v"], s["table"], s["B"], s["ctx"])
    rope = (s["rope"], s["mad"]) if case["rope"] else ()
    if kind == "decode":
        call = pic.pic_page_decode_attn_rope if case["rope"] else pic.pic_page_decode_attn
        call(*head, case["step"], s["max_ctx"], *rope, s["out"], s["ws"])
    else:
        call = pic.pic_page_suffix_attn_rope if case["rope"] else pic.pic_page_suffix_attn
        call(*head, s["max_ctx"], s["n"], *rope, s["out"], s["ws"], s["n_valid"])
    return {"out": s["out"], "pages_k": s["pages_k"], "pages_v": s["pages_v"]}


def _turn(x, pos, theta, pairing):
    """Rows x [L, N, heads, D] turned to positions pos [N]: angles in 64 bits, products in 32."""
    d = x.shape[-1]
    inv = float(theta) ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    ang = pos.to(torch.float64)[:, None] * inv
    c, sn = ang.cos().float()[None, :, None], ang.sin().float()[None, :, None]
    x = x.float()
    if pairing == "half":
        a, b = x[..., : d // 2], x[..., d // 2:]
        return torch.cat([a * c - b * sn, a * sn + b * c], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)


def _attend(s, case):
    L, hq, hkv, d = s["shape"]
    P, B, n, T = case["page"], s["B"], s["n"], s["max_len"]
    dt, ab, ai, ap = s["q"].dtype, s["at_b"], s["at_i"], s["at_pos"]
    q, k, v = s["q"][:, ab, ai].float(), s["k"][:, ab, ai], s["v"][:, ab, ai]   # [L, N, heads, D]
    if case["rope"]:
        q, k = _turn(q, ap, s["theta"], case["pairing"]), _turn(k, ap, s["theta"], case["pairing"]).to(dt)
    # the new tokens into their slots
    row = s["table"][ab, ap // P].long() * P + ap % P
    s["pages_k"][:, :, row] = k.transpose(1, 2)
    s["pages_v"][:, :, row] = v.transpose(1, 2)
    # every request's slots, gathered: [L, Hkv, B, T, D]
    slot = torch.arange(T, device=DEV)
    rows = s["table"][:, slot // P].long().clamp(min=0) * P + slot % P
    keys, vals = s["pages_k"][:, :, rows].float(), s["pages_v"][:, :, rows].float()
    qp = torch.zeros((L, B, n, hq, d), device=DEV)
    qp[:, ab, ai] = q
    pos = torch.zeros((B, n), dtype=torch.int64, device=DEV)
    pos[ab, ai] = ap
    rep = hq // hkv
    qp = qp.view(L, B, n, hkv, rep, d).permute(0, 3, 1, 4, 2, 5).reshape(L, hkv, B, rep * n, d)
    w = qp @ keys.transpose(-1, -2) * s["scale"]
    hidden = (slot > pos[..., None]).repeat(1, rep, 1)                           # [B, rep * n, T]
    w = w.masked_fill_(hidden, -math.inf)
    w = (w - w.amax(-1, keepdim=True)).exp_()
    o = (w @ vals) / w.sum(-1, keepdim=True)
    o = o.view(L, hkv, B, rep, n, d).permute(0, 2, 4, 1, 3, 5).reshape(L, B, n, hq, d)
    s["out"][:, ab, ai] = o[:, ab, ai].to(dt)
    return {"out": s["out"], "pages_k": s["pages_k"], "pages_v": s["pages_v"]}


# ------------------------------------------------------------------------------------------
# the definition in 64 bits: request by request, layer by layer
# ------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    L, hq, hkv, d = s["shape"]
    P = case["page"]
    if case["kind"] == "copy":
        moved = torch.arange(s["n_pages"], device=DEV)   # page -> the page its contents come from
        for a, b in s["pairs"].tolist():
            moved[b] = a
        take = lambda x: x.view(L, hkv, s["n_pages"], P, d).index_select(2, moved).reshape(x.shape).double()  # noqa: E731
        return {"pages_k": take(s["pages_k"]), "pages_v": take(s["pages_v"])}
    ctx, table = s["ctx"].tolist(), s["table"].long()
    step = case.get("step", 0)
    new = [1 if c >= 0 else 0 for c in ctx] if case["kind"] == "decode" else s["n_valid"].tolist()
    out, pk, pv = s["out"].double(), s["pages_k"].double(), s["pages_v"].double()
    half = torch.arange(d // 2, device=DEV, dtype=torch.float64)
    for b, nv in enumerate(new):
        if nv == 0:
            continue
        first = ctx[b] + step
        pos = torch.arange(first, first + nv, device=DEV)
        slots = torch.arange(first + nv, device=DEV)
        rows = table[b, slots.div(P, rounding_mode="floor")] * P + slots.remainder(P)
        for l in range(L):
            q, k, v = (s[x][l, b, :nv].double() for x in "qkv")               # [nv, heads, D]
            if case["rope"]:
                z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                                pos[:, None] * (-2.0 * half / d * math.log(s["theta"])).exp())[:, None]

                def turn(x):
                    if case["pairing"] == "half":
                        y = torch.complex(x[..., : d // 2], x[..., d // 2:]) * z
                        return torch.cat([y.real, y.imag], -1)
                    return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2)) * z).flatten(-2)

                q, k = turn(q), turn(k)
            pk[l][:, rows[first:]] = k.transpose(0, 1)
            pv[l][:, rows[first:]] = v.transpose(0, 1)
            for g in range(hkv):
                kk, vv = pk[l, g, rows], pv[l, g, rows]
                qq = q[:, g * (hq // hkv):(g + 1) * (hq // hkv)]               # [nv, rep, D]
                sc = (qq.reshape(-1, d) @ kk.T).view(nv, -1, len(slots)) * s["scale"]
                sc = sc.masked_fill(slots[None, None] > pos[:, None, None], -math.inf)
                out[l, b, :nv, g * (hq // hkv):(g + 1) * (hq // hkv)] = sc.softmax(-1) @ vv
    return {"out": out, "pages_k": pk, "pages_v": pv}
