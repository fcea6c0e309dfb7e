"""More operators of a program that serves from a paged cache: what is measured of them, and their plain forms.

Pages, page tables and slots are those of a paged cache: K and V pages [layers][kv heads][n_pages * page_tokens][head_dim],
slot t of request b in row table[b][t // P] * P + t % P of every (layer, kv head) stream, P = page_tokens.

  decode   one new token per request of a batch whose requests share long prefixes: requests of a group (neighbours in
           the batch) hold the same K/V in slots [0, shared_len), in pages they share.  The new token's K/V go to slot
           p = base_len[b] + step, its query heads attend over slots [0, p]; a negative base_len is padding
  suffix   the same for n_suffix tokens per request (drafted tokens, short questions), token i at ctx_len[b] + i; tokens
           from n_valid[b] on are padding
  norm     queries and keys of new tokens as a projection leaves them: each head divided by its root mean square, times
           a weight, then turned to its position: the first rope_dim elements of a head in pairs (halves or
           interleaved), with frequencies stretched for long contexts (yarn) or not; values are laid out beside them
  grow     page tables made ready for new tokens from the requests' lengths, lowest free page first; a partly filled
           page that is shared gives way to one of the request's own, and is copied where the case has layers

Plain forms are elementary torch operations in 32 bits (angles in 64); exact() is the definition in 64 bits.
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
EPS = 1e-6
YARN = (8.0, 8192.0, 32.0, 1.0)   # factor, original positions, beta_fast, beta_slow


def listed():
    return [
        # two answers sampled from one short prompt: all latency
        dict(name="decode_pair_2k", kind="decode", shape="llama8b", layers=1, batch=2, groups=1, shared=2065, ragged=0.0,
             own=33, step=1, idle=0, page=64),
        # 16 questions about the same ten documents, a step of their answers
        dict(name="decode_llama_16x10k", kind="decode", shape="llama8b", layers=1, batch=16, groups=1, shared=10368,
             ragged=0.0, own=228, step=17, idle=0, page=64),
        # a full batch of samples from one 16K context
        dict(name="decode_llama_64x16k", kind="decode", shape="llama8b", layers=1, batch=64, groups=1, shared=16384,
             ragged=0.0, own=300, step=5, idle=0, page=64),
        # four sets of documents of uneven length, their requests side by side, places left empty, pages of 16 tokens
        dict(name="decode_qwen_groups_32k", kind="decode", shape="qwen7b", layers=1, batch=37, groups=4, shared=32749,
             ragged=0.5, own=611, step=0, idle=5, page=16),
        # drafted tokens checked: 5 per request, padded, head_dim 64, two layers in one call
        dict(name="suffix_hd64_drafts", kind="suffix", shape="llama_hd64", layers=2, batch=12, groups=2, shared=4161,
             ragged=0.25, own=97, suffix=5, pad=0.9, page=32),
        # 16 short questions arrive at once over the same ten documents
        dict(name="suffix_llama_16x10k", kind="suffix", shape="llama8b", layers=1, batch=16, groups=1, shared=10368,
             ragged=0.0, own=0, suffix=24, pad=0.0, page=64),
        # one step of a small decode batch, slices of one projection: a launch
        dict(name="norm_decode_7", kind="norm", shape="qwen7b", dtype="bf16", layers=1, batch=7, tokens=1, ctx=33001,
             fused=True, pad=0.0, rope_dim=128, pairing="half", yarn=False, order="keep"),
        # a batch's suffix tokens on their way into the prefill, padded, stretched frequencies
        dict(name="norm_suffix_yarn", kind="norm", shape="llama8b", dtype="bf16", layers=1, batch=16, tokens=131, ctx=30011,
             fused=True, pad=0.5, rope_dim=128, pairing="half", yarn=True, order="keep"),
        # 64 documents of 1024 tokens being compiled, half of each head turned, interleaved pairs
        dict(name="norm_documents", kind="norm", shape="llama8b", dtype="bf16", layers=1, batch=64, tokens=1024, ctx=0,
             fused=False, pad=0.0, rope_dim=64, pairing="interleaved", yarn=False, order="keep"),
        # a small float32 model, half of each head turned, its pairs laid out for composition
        dict(name="norm_small_f32", kind="norm", shape="small", dtype="f32", layers=2, batch=4, tokens=61, ctx=2077,
             fused=False, pad=0.0, rope_dim=32, pairing="half", yarn=False, order="pairs"),
        # one decode step of a full batch: a request in 64 comes to a page's end
        dict(name="grow_decode_64", kind="grow", shape="llama8b", layers=0, batch=64, ctx=16384, ragged=0.25, tokens=1,
             pages=20000, page=64, forked=0),
        # 15 forks of one request write for the first time: pages of their own and the copies, in all 32 layers
        dict(name="grow_fork_copy_16", kind="grow", shape="llama8b", layers=32, batch=16, ctx=1001, ragged=0.0, tokens=7,
             pages=80, page=64, forked=15),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "suffix", "suffix", "norm", "norm", "grow"])
    if kind == "norm":
        f32 = rng.random() < 0.25
        shape = rng.choice(["tiny", "small"]) if f32 else rng.choice(["llama8b", "qwen7b", "llama_hd64"])
        d, pairing = SHAPES[shape][2], rng.choice(["half", "interleaved"])
        batch, tokens = _log(rng, 1, 64), rng.choice([1, _log(rng, 1, 1024)])
        return dict(kind=kind, shape=shape, dtype="f32" if f32 else "bf16", layers=rng.choice([1, 1, 2]) if tokens < 500 else 1,
                    batch=batch, tokens=tokens, ctx=rng.choice([0, _log(rng, 1, 33000)]), fused=rng.random() < 0.5,
                    pad=rng.choice([0.0, 0.5, 0.9]), rope_dim=rng.choice([d, d, d // 2, d // 4, 16, 48]), pairing=pairing,
                    yarn=rng.random() < 0.3, order=rng.choice(["keep", "pairs"]) if pairing == "half" else "keep")
    if kind == "grow":
        page, layers = rng.choice([16, 32, 64, 128]), rng.choice([0, 0, 2, 8])
        batch, tokens = _log(rng, 1, 32 if layers else 64), rng.choice([1, _log(rng, 1, 300)])
        forked = rng.randint(0, batch - 1) if batch > 1 else 0
        ctx = _log(rng, 1, 2000 if layers else 33000)
        need = batch * (-(-(ctx + tokens) // page) + 1)
        return dict(kind=kind, shape=rng.choice(["llama_hd64", "qwen7b"]), layers=layers, batch=batch, ctx=ctx,
                    ragged=rng.choice([0.0, 0.25, 0.9]), tokens=tokens, pages=need + rng.randint(0, 1 + need // 2), page=page,
                    forked=forked)
    c = dict(kind=kind, shape=rng.choice(["llama8b", "llama8b", "qwen7b", "llama_hd64"]), layers=rng.choice([1, 1, 1, 2]),
             page=rng.choice([16, 32, 64, 64, 128, 256]), ragged=rng.choice([0.0, 0.25, 0.5, 0.9]))
    hq, hkv, d, _ = SHAPES[c["shape"]]
    batch = _log(rng, 2, 64 if kind == "decode" else 16)
    c.update(batch=batch, groups=rng.choice([1, 1, min(batch, rng.randint(2, 4))]))
    n = 1 if kind == "decode" else _log(rng, 2, 32)
    top = int((1.6e10 if kind == "decode" else 5.5e10) / (4 * hq * d * batch * n * c["layers"]))
    c.update(shared=_log(rng, 33, min(33000, top)))
    c.update(own=min(_log(rng, 1, 2000), max(1, (top - c["shared"]) // 2)))
    if kind == "decode":
        return dict(c, step=rng.randint(0, 63), idle=rng.choice([0, 0, rng.randint(0, batch - 2)]))
    return dict(c, suffix=n, pad=rng.choice([0.0, 0.0, 0.5, 0.9]))


# ------------------------------------------------------------------------------------------
# layouts: lengths are fixed by the case, so that the work does not depend on the seed; which page
# holds what does
# ------------------------------------------------------------------------------------------

def _starts(case):
    """First request of each group, and the batch's end: groups of uneven size."""
    r = random.Random(5)
    return [0] + sorted(r.sample(range(1, case["batch"]), case["groups"] - 1)) + [case["batch"]]


def _shared(case):
    """Slots the requests of each group share: the longest is case["shared"], the others up to a share `ragged` shorter."""
    r = random.Random(6)
    return [case["shared"]] + [case["shared"] - int(r.random() * case["ragged"] * case["shared"]) for _ in range(case["groups"] - 1)]


def _group_of(case):
    s = _starts(case)
    return [g for g in range(case["groups"]) for _ in range(s[g], s[g + 1])]


def _ctx(case):
    """Tokens each request has cached: its group's prefix and up to case["own"] of its own; -1 for padding (never the first)."""
    r, shared = random.Random(3), _shared(case)
    c = [shared[g] + (case["own"] if b == 0 else int(r.random() * (case["own"] + 1))) for b, g in enumerate(_group_of(case))]
    for b in r.sample(range(1, case["batch"]), case.get("idle", 0)):
        c[b] = -1
    return c


def _valid(batch, n, pad):
    """New tokens of each request of a padded batch (0 among them where the padding is deep)."""
    r = random.Random(4)
    v = [n] + [n - int(r.random() * pad * (n + 1)) for _ in range(batch - 1)]
    if pad > 0.8 and len(v) > 2:
        v[-1] = 0
    return v


def _new(case):
    """New tokens of each request of a decode or suffix case."""
    if case["kind"] == "decode":
        return [1 if c >= 0 else 0 for c in _ctx(case)]
    return _valid(case["batch"], case["suffix"], case["pad"])


def _norm_base(case):
    r = random.Random(7)
    return [case["ctx"]] + [case["ctx"] - int(r.random() * 0.5 * case["ctx"]) for _ in range(case["batch"] - 1)]


def _grow_lens(case):
    """Lengths of a grow case: request 0, then its forks (the same length), then others of their own."""
    r = random.Random(8)
    return [case["ctx"] if b <= case["forked"] else max(1, case["ctx"] - int(r.random() * case["ragged"] * case["ctx"]))
            for b in range(case["batch"])]


def _es(case):
    return 4 if case.get("dtype") == "f32" else 2


def work(case):
    hq, hkv, d, _ = SHAPES[case["shape"]]
    L, es = case["layers"], _es(case)
    if case["kind"] == "norm":
        tokens = L * sum(_valid(case["batch"], case["tokens"], case["pad"]))
        return {"bytes": 2 * tokens * (hq + 2 * hkv) * d * es, "flops": tokens * (hq + hkv) * d * 8}
    if case["kind"] == "grow":
        P, lens = case["page"], _grow_lens(case)
        entries = sum(-(-(n + case["tokens"]) // P) - n // P for n in lens)
        copies = case["forked"] if case["ctx"] % P else 0
        return {"bytes": 4 * (2 * len(lens) + 4 * entries) + 4 * copies * L * hkv * P * d * 2, "flops": 0}
    ctx, new, group, shared = _ctx(case), _new(case), _group_of(case), _shared(case)
    off = case.get("step", 0)
    seen = cached = 0
    for c, v, g in zip(ctx, new, group):
        if v:   # a request without new tokens is not read
            cached += c + off - shared[g]
            seen += v * (c + off) + v * (v + 1) // 2
    cached += sum(shared[g] for g in {g for g, v in zip(group, new) if v})
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


def _inv_freq(case, theta, d):
    """(frequencies of the turned pairs, factor on the turned elements), in 64 bits."""
    n = case["rope_dim"]
    f = theta ** (-2.0 * np.arange(n // 2) / n)
    if not case["yarn"]:
        return f, 1.0
    factor, orig, fast, slow = YARN
    at = lambda turns: n * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), n - 1)
    ramp = np.clip((np.arange(n // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
    return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1


def prepare(case, seed):
    return {"norm": _prepare_norm, "grow": _prepare_grow}.get(case["kind"], _prepare_attn)(dict(case), seed)


def _prepare_attn(case, seed):
    hq, hkv, d, theta = SHAPES[case["shape"]]
    L, P, randn, r = case["layers"], case["page"], _randn(seed, "bf16"), np.random.default_rng(seed)
    B, n = case["batch"], 1 if case["kind"] == "decode" else case["suffix"]
    ctx, new, start, shared = _ctx(case), _new(case), _starts(case), _shared(case)
    off = case.get("step", 0)
    s = dict(case=case, scale=1.0 / math.sqrt(d), shape=(L, hq, hkv, d), B=B, n=n, max_ctx=max(ctx), max_shared=max(shared))
    lens = [c + off + v if v else max(c, 0) + off for c, v in zip(ctx, new)]
    # pages: a group's whole pages of the prefix once, every request's others its own
    whole = [x // P for x in shared]
    group = _group_of(case)
    need = [max(-(-x // P), -(-shared[g] // P)) for x, g in zip(lens, group)]
    total = sum(whole) + sum(k - whole[g] for k, g in zip(need, group))
    s["n_pages"] = total + max(1, total // 16)
    order, table, at = r.permutation(s["n_pages"]), np.full((B, max(need)), -1, np.int32), 0
    for g in range(case["groups"]):
        table[start[g]:start[g + 1], : whole[g]] = order[at: at + whole[g]]
        at += whole[g]
    for b, g in enumerate(group):
        table[b, whole[g]: need[b]] = order[at: at + need[b] - whole[g]]
        at += need[b] - whole[g]
    s["pages_k"], s["pages_v"] = randn(L, hkv, s["n_pages"] * P, d), randn(L, hkv, s["n_pages"] * P, d)
    # the part of a prefix in a page that a request has for itself holds the same
    src, dst = [], []
    for b, g in enumerate(group):
        for t in range(whole[g] * P, shared[g]):
            src.append(table[start[g], t // P] * P + t % P)
            dst.append(table[b, t // P] * P + t % P)
    if src:
        src, dst = _dev(src, np.int64), _dev(dst, np.int64)
        for x in (s["pages_k"], s["pages_v"]):
            x[:, :, dst] = x[:, :, src]
    s.update(table=_dev(table), table_cap=table.shape[1], ctx=_dev(ctx), start=_dev(start), shared=_dev(shared),
             n_valid=_dev(new), max_group=max(b - a for a, b in zip(start, start[1:])), max_own=max(1, max(
                 x - shared[g] for x, g in zip(lens, group))))
    # (request, token) of every new token that is one, and its slot
    at = [(b, i, ctx[b] + off + i) for b in range(B) for i in range(new[b])]
    s["at_b"], s["at_i"], s["at_pos"] = (_dev([x[j] for x in at], np.int64) for j in range(3))
    s["group"], s["in_group"] = _dev(group, np.int64), _dev([b - start[g] for b, g in enumerate(group)], np.int64)
    s["q"], s["k"], s["v"] = randn(L, B, n, hq, d), randn(L, B, n, hkv, d), randn(L, B, n, hkv, d)
    s["out"] = randn(L, B, n, hq, d) / 32   # what padding rows hold before and after: the size of an average of values
    if own:
        import paper_2607_28069_amd as pic
        s["model"] = m = pic.Model.of(L, hq, hkv, d, "bf16", theta)
        s["pages"] = pic.Pages.of(s["n_pages"], P, s["table_cap"])
        s["groups"] = pic.Shared.of(case["groups"], s["max_group"], s["max_shared"])
        need = pic.pic_page_shared_workspace_bytes(m, s["groups"], B, n, s["max_ctx"] + off)
        s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return s


def _prepare_norm(case, seed):
    hq, hkv, d, theta = SHAPES[case["shape"]]
    L, B, n, randn = case["layers"], case["batch"], case["tokens"], _randn(seed, case["dtype"])
    s = dict(case=case, shape=(L, hq, hkv, d), B=B, n=n)
    if case["fused"]:
        s["qkv"] = randn(L, B, n, (hq + 2 * hkv) * d) * 1.5
    else:
        s["qkv"] = (randn(L, B, n, hq, d) * 1.5, randn(L, B, n, hkv, d) * 1.5, randn(L, B, n, hkv, d))
    base, valid = _norm_base(case), _valid(B, n, case["pad"])
    s.update(max_base=max(base), base=_dev(base), n_valid=_dev(valid))
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 99)
    weight = lambda: 1 + 0.2 * torch.randn((L, d), generator=g, device=DEV)  # noqa: E731
    s["q_weight"], s["k_weight"] = weight(), weight()
    s["q"], s["k"], s["v"] = randn(L, B, n, hq, d), randn(L, B, n, hkv, d), randn(L, B, n, hkv, d)   # the call's outputs
    at = [(b, i, base[b] + i) for b in range(B) for i in range(valid[b])]
    s["at_b"], s["at_i"], s["at_pos"] = (_dev([x[j] for x in at], np.int64) for j in range(3))
    freq, s["rope_scale"] = _inv_freq(case, theta, d)
    s["freq"] = torch.from_numpy(freq).to(DEV)
    if own:
        import paper_2607_28069_amd as pic
        s["model"] = m = pic.Model.of(L, hq, hkv, d, case["dtype"], theta, case["pairing"])
        full = np.zeros(d // 2)
        if case["yarn"]:
            full, s["rope_scale"] = pic.pic_rope_yarn_freq(d, theta, *YARN, rope_dim=case["rope_dim"])
        else:
            full[: len(freq)] = freq
        s["mad"] = s["max_base"] + n
        s["rope"] = torch.empty(pic.pic_rope_table_bytes(m, s["mad"]) // 4, dtype=torch.float32, device=DEV)
        pic.pic_rope_table_init_freq(m, full, s["mad"], s["rope"])
        s["how"] = pic.QkNorm.of(s["q_weight"], s["k_weight"], EPS, case["rope_dim"], case["order"], s["rope_scale"])
    return s


def _prepare_grow(case, seed):
    hq, hkv, d, theta = SHAPES[case["shape"]]
    B, P, n, L = case["batch"], case["page"], case["tokens"], case["layers"]
    lens, r = _grow_lens(case), np.random.default_rng(seed)
    cap = max(-(-(x + n) // P) for x in lens)
    table, refs, order, at = np.full((B, cap), -1, np.int32), np.zeros(case["pages"], np.int32), r.permutation(case["pages"]), 0
    for b, x in enumerate(lens):
        k = -(-x // P)
        if 0 < b <= case["forked"]:
            table[b, :k] = table[0, :k]
        else:
            table[b, :k] = order[at: at + k]
            at += k
        refs[table[b, :k]] += 1
    s = dict(case=case, shape=(L, hq, hkv, d), B=B, n=n, cap=cap, refs0=_dev(refs), table0=_dev(table), lens=_dev(lens))
    s["refs"], s["table"] = s["refs0"].clone(), s["table0"].clone()
    s["pairs"], s["ready"] = _dev(np.zeros((B, 2))), _dev(np.zeros(B))
    s["result"] = _dev(np.zeros(3))
    if L:
        randn = _randn(seed, "bf16")
        s["pages_k"], s["pages_v"] = randn(L, hkv, case["pages"] * P, d), randn(L, hkv, case["pages"] * P, d)
    if own:
        import paper_2607_28069_amd as pic
        s["model"] = pic.Model.of(L, hq, hkv, d, "bf16", theta)
        s["pages"] = pic.Pages.of(case["pages"], P, cap)
        s["ws"] = torch.empty(max(16, pic.pic_page_grow_workspace_bytes(s["pages"], B, n)), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if kind == "norm":
        return _run_norm(s)
    if kind == "grow":
        return _run_grow(s)
    return _run_attn_own(s) if own else _attend(s)


def _run_attn_own(s):
    import paper_2607_28069_amd as pic
    case = s["case"]
    head = (s["model"], s["pages"], s["groups"], s["q"], s["k"], s["v"], s["pages_k"], s["pages_v"], s["table"], s["B"],
            s["start"], s["shared"], s["ctx"])
    if case["kind"] == "decode":
        pic.pic_page_shared_decode_attn(*head, case["step"], s["max_ctx"], s["out"], s["ws"])
    else:
        pic.pic_page_shared_suffix_attn(*head, s["max_ctx"], s["n"], s["out"], s["ws"], s["n_valid"])
    return {"out": s["out"], "pages_k": s["pages_k"], "pages_v": s["pages_v"]}


def _attend(s):
    case = s["case"]
    L, hq, hkv, d = s["shape"]
    P, B, n, S, T = case["page"], s["B"], s["n"], s["max_shared"], s["max_own"]
    dt, ab, ai, ap, rep = s["q"].dtype, s["at_b"], s["at_i"], s["at_pos"], hq // hkv
    n_groups, most = case["groups"], s["max_group"]
    # the new tokens into their slots
    row = s["table"][ab, ap // P].long() * P + ap % P
    s["pages_k"][:, :, row] = s["k"][:, ab, ai].transpose(1, 2)
    s["pages_v"][:, :, row] = s["v"][:, ab, ai].transpose(1, 2)
    q = s["q"].float().view(L, B, n, hkv, rep, d).permute(0, 3, 1, 4, 2, 5)                    # [L, Hkv, B, rep, n, D]
    pos = torch.zeros((B, n), dtype=torch.int64, device=DEV)
    pos[ab, ai] = ap
    # over a group's prefix, all of its requests' queries side by side: [L, Hkv, groups, most * rep * n, S]
    slot = torch.arange(S, device=DEV)
    rows = s["table"][s["start"][:-1].long()][:, slot // P].long().clamp(min=0) * P + slot % P
    qg = torch.zeros((L, hkv, n_groups, most, rep, n, d), device=DEV)
    qg[:, :, s["group"], s["in_group"]] = q
    wp = qg.view(L, hkv, n_groups, most * rep * n, d) @ s["pages_k"][:, :, rows].float().transpose(-1, -2) * s["scale"]
    wp = wp.masked_fill_(slot >= s["shared"][:, None, None], -math.inf)
    # over each request's own slots: [L, Hkv, B, rep * n, T]
    slot = s["shared"].long()[s["group"]][:, None] + torch.arange(T, device=DEV)               # [B, T]
    at = (slot // P).clamp(max=s["table_cap"] - 1)
    rows_o = s["table"].gather(1, at).long().clamp(min=0) * P + slot % P
    wo = q.reshape(L, hkv, B, rep * n, d) @ s["pages_k"][:, :, rows_o].float().transpose(-1, -2) * s["scale"]
    wo = wo.masked_fill_((slot[:, None] > pos[..., None]).repeat(1, rep, 1), -math.inf)
    # joined by their maxima and sums
    mp = wp.amax(-1, keepdim=True)
    wp = (wp - mp).exp_()
    op = (wp @ s["pages_v"][:, :, rows].float()).view(L, hkv, n_groups, most, rep * n, d)[:, :, s["group"], s["in_group"]]
    mp, lp = (x.view(L, hkv, n_groups, most, rep * n, 1)[:, :, s["group"], s["in_group"]] for x in (mp, wp.sum(-1, keepdim=True)))
    mo = wo.amax(-1, keepdim=True).clamp(min=-1e30)
    wo = (wo - mo).exp_()
    m = torch.maximum(mp, mo)
    fp, fo = (mp - m).exp(), (mo - m).exp()
    o = (op * fp + (wo @ s["pages_v"][:, :, rows_o].float()) * fo) / (lp * fp + wo.sum(-1, keepdim=True) * fo)
    o = o.view(L, hkv, B, rep, n, d).permute(0, 2, 4, 1, 3, 5).reshape(L, B, n, hq, d)
    s["out"][:, ab, ai] = o[:, ab, ai].to(dt)
    return {"out": s["out"], "pages_k": s["pages_k"], "pages_v": s["pages_v"]}


def _split(s):
    """Queries, keys and values [L, B, n, heads, D] of the projection's outputs."""
    L, hq, hkv, d = s["shape"]
    if not s["case"]["fused"]:
        return s["qkv"]
    x = s["qkv"].view(L, s["B"], s["n"], hq + 2 * hkv, d)
    return x[..., :hq, :], x[..., hq: hq + hkv, :], x[..., hq + hkv:, :]


def _run_norm(s):
    case = s["case"]
    q, k, v = _split(s)
    if own:
        import paper_2607_28069_amd as pic
        pic.pic_qk_norm_rope(s["model"], s["how"], q, k, v, s["B"], s["n"], s["rope"], s["mad"], s["q"], s["k"], s["v"],
                             base_len=s["base"], max_base_len=s["max_base"], n_valid=s["n_valid"])
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    ab, ai, ap, r, d = s["at_b"], s["at_i"], s["at_pos"], case["rope_dim"], s["shape"][3]
    ang = ap.to(torch.float64)[:, None] * s["freq"]
    c, sn = ((f.float() * s["rope_scale"])[None, :, None] for f in (ang.cos(), ang.sin()))
    for x, w, out in ((q, s["q_weight"], s["q"]), (k, s["k_weight"], s["k"])):
        x = x[:, ab, ai].float()                                                              # [L, N, heads, D]
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w[:, None, None]
        t, rest = x[..., :r], x[..., r:]
        if case["pairing"] == "half":
            a, b = t[..., : r // 2], t[..., r // 2:]
            a, b = a * c - b * sn, a * sn + b * c
            y = (torch.cat([a, rest[..., : (d - r) // 2], b, rest[..., (d - r) // 2:]], -1) if case["order"] == "pairs" else
                 torch.cat([a, b, rest], -1))
        else:
            a, b = t[..., 0::2], t[..., 1::2]
            y = torch.cat([torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2), rest], -1)
        out[:, ab, ai] = y.to(out.dtype)
    s["v"][:, ab, ai] = v[:, ab, ai]
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def _run_grow(s):
    case, P, B, n, cap = s["case"], s["case"]["page"], s["B"], s["n"], s["cap"]
    # (every pass starts from the same tables)
    s["refs"].copy_(s["refs0"])
    s["table"].copy_(s["table0"])
    got = {x: s[x] for x in ("refs", "table", "pairs", "ready", "result")}
    if case["layers"]:
        got.update(pages_k=s["pages_k"], pages_v=s["pages_v"])
    if own:
        import paper_2607_28069_amd as pic
        pic.pic_page_grow_async(s["pages"], B, s["refs"], s["table"], s["lens"], n, s["pairs"], s["ready"], s["result"], s["ws"])
        if case["layers"]:
            pic.pic_page_copy_async(s["model"], s["pages"], s["pages_k"], s["pages_v"], s["pairs"], B)
        return got
    refs, table, lens = s["refs"], s["table"], s["lens"].long()[:, None]
    i = torch.arange(cap, device=DEV)
    todo = (i >= lens // P) & (i < (lens + n + P - 1) // P)                                   # [B, cap] entries that are looked at
    partly = (i == lens // P) & (lens % P != 0)
    held = todo & (table >= 0)
    # of those that hold the same page, in order, all but as many as it has other references take one of their own
    page = torch.where(held, table, case["pages"]).flatten().long()
    by, where = page.sort(stable=True)
    first = torch.searchsorted(by, by)
    rank = torch.empty_like(where)
    rank[where] = torch.arange(len(by), device=DEV) - first
    count = torch.cat([refs, refs.new_ones(1)])
    leaves = (held.flatten() & (count[page] - rank > 1)).view(B, cap)
    takes = leaves | (todo & ~held)
    refs.scatter_add_(0, table.clamp(min=0).flatten().long(), -leaves.flatten().int())
    free = (s["refs0"] == 0)
    lowest = torch.where(free, torch.arange(case["pages"], device=DEV), case["pages"]).sort().values
    new = lowest[(takes.flatten().cumsum(0) - 1).clamp(min=0)].view(B, cap)
    taken = torch.zeros(case["pages"] + 1, dtype=torch.int32, device=DEV)
    taken[torch.where(takes, new, case["pages"]).flatten()] = 1
    refs += taken[:-1]
    copies = (leaves & partly).flatten()
    to = torch.where(copies, copies.cumsum(0) - 1, B)
    pairs = torch.full((B + 1, 2), -1, dtype=torch.int32, device=DEV)
    pairs[to] = torch.stack([table.flatten(), new.flatten().int()], -1)
    s["pairs"].copy_(torch.where((torch.arange(B, device=DEV) < copies.sum())[:, None], pairs[:B], -1))
    table.copy_(torch.where(takes, new.int(), table))
    s["ready"].copy_(s["lens"])
    s["result"][0] = 0
    s["result"][1] = copies.sum()
    s["result"][2] = takes.sum()
    if case["layers"]:
        # (pairs that are none copy what the first one does, or a page onto itself)
        L, _, hkv, d = s["shape"]
        src, dst = (torch.where(s["pairs"][:, 0] >= 0, s["pairs"][:, j], s["pairs"][0, j].clamp(min=0)).long() for j in (0, 1))
        for x in (s["pages_k"], s["pages_v"]):
            p = x.view(L, hkv, case["pages"], -1)
            p[:, :, dst] = p[:, :, src]
    return got


# ------------------------------------------------------------------------------------------
# the definitions in 64 bits: request by request
# ------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "grow": _exact_grow}.get(case["kind"], _exact_attn)(s, case)


def _exact_attn(s, case):
    L, hq, hkv, d = s["shape"]
    P, ctx, table, new = case["page"], s["ctx"].tolist(), s["table"].long(), s["n_valid"].tolist()
    rep = hq // hkv
    out, pk, pv = s["out"].double(), s["pages_k"].double(), s["pages_v"].double()
    for b, nv in enumerate(new):
        if nv == 0:
            continue
        first = ctx[b] + case.get("step", 0)
        slots = torch.arange(first + nv, device=DEV)
        rows = table[b, slots.div(P, rounding_mode="floor")] * P + slots.remainder(P)
        hidden = slots[None, None] > torch.arange(first, first + nv, device=DEV)[:, None, None]
        for l in range(L):
            q, k, v = (s[x][l, b, :nv].double() for x in "qkv")               # [nv, heads, D]
            pk[l][:, rows[first:]] = k.transpose(0, 1)
            pv[l][:, rows[first:]] = v.transpose(0, 1)
            for g in range(hkv):
                sc = (q[:, g * rep:(g + 1) * rep].reshape(-1, d) @ pk[l, g, rows].T).view(nv, rep, -1) * s["scale"]
                out[l, b, :nv, g * rep:(g + 1) * rep] = sc.masked_fill(hidden, -math.inf).softmax(-1) @ pv[l, g, rows]
    return {"out": out, "pages_k": pk, "pages_v": pv}


def _exact_norm(s, case):
    L, hq, hkv, d = s["shape"]
    r, base, valid = case["rope_dim"], s["base"].tolist(), s["n_valid"].tolist()
    got = {x: s[x].double() for x in "qkv"}
    # where element e of a head goes
    to = list(range(d))
    if case["order"] == "pairs":
        low, rest = r // 2, (d - r) // 2
        to = [e if e < low else d // 2 + e - low if e < r else low + e - r if e < r + rest else d // 2 + low + e - r - rest
              for e in range(d)]
    to = torch.tensor(to, device=DEV)
    freq, _ = _inv_freq(case, SHAPES[case["shape"]][3], d)
    freq, scale = torch.from_numpy(freq).to(DEV), s["rope_scale"]
    for x, name, w in zip(_split(s), "qkv", (s["q_weight"], s["k_weight"], None)):
        for b, nv in enumerate(valid):
            y = x[:, b, :nv].double()                                                         # [L, nv, heads, D]
            if w is not None:
                y = y / ((y * y).sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()[:, None, None]
                z = torch.polar(torch.full((), scale, dtype=torch.float64, device=DEV),
                                torch.arange(base[b], base[b] + nv, device=DEV)[:, None] * freq)[:, None]
                if case["pairing"] == "half":
                    t = torch.complex(y[..., : r // 2], y[..., r // 2: r]) * z
                    t = torch.cat([t.real, t.imag], -1)
                else:
                    t = torch.view_as_real(torch.view_as_complex(y[..., :r].reshape(*y.shape[:-1], r // 2, 2)) * z).flatten(-2)
                y = torch.empty_like(y).index_copy_(3, to, torch.cat([t, y[..., r:]], -1))
            got[name][:, b, :nv] = y
    return got


def _exact_grow(s, case):
    P, refs, table, lens = case["page"], s["refs0"].tolist(), s["table0"].tolist(), s["lens"].tolist()
    free = [p for p, n in enumerate(refs) if n == 0]
    pairs, taken = [], 0
    for b, x in enumerate(lens):
        for i in range(x // P, -(-(x + s["n"]) // P)):
            p = table[b][i]
            if p >= 0 and refs[p] == 1:
                continue
            if p >= 0:
                refs[p] -= 1
                if i == x // P and x % P:
                    pairs.append([p, free[taken]])
            table[b][i] = free[taken]
            refs[free[taken]] = 1
            taken += 1
    got = dict(refs=_dev(refs), table=_dev(table), pairs=_dev(pairs + [[-1, -1]] * (s["B"] - len(pairs))), ready=s["lens"],
               result=_dev([0, len(pairs), taken]))
    if case["layers"]:
        L, _, hkv, d = s["shape"]
        moved = torch.arange(case["pages"], device=DEV)   # page -> the page its contents come from
        for a, b in pairs:
            moved[b] = a
        for x in ("pages_k", "pages_v"):
            got[x] = s[x].view(L, hkv, case["pages"], P, d).index_select(2, moved).reshape(s[x].shape).double()
    return got
