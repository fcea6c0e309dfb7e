"""Host side of shared prefixes, page tables grown on the device and norms with rotation: every refusal, and the
frequencies of a stretched rotation (none of which needs a GPU)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic

INVALID, UNSUPPORTED, WORKSPACE, CAPACITY, MISALIGNED, RANGE = -1, -2, -3, -4, -5, -6


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(pic.LIB_PATH):
        from paper_2607_28069_amd.build import build
        build()
    return pic.load()


@pytest.fixture(scope="module")
def p():
    """An address (of host memory: a call that is refused reads nothing of it)."""
    buf = ctypes.create_string_buffer(1 << 16)
    yield (ctypes.addressof(buf) + 15) & ~15


MODEL = pic.Model.of(1, 4, 2, 64, "bf16", 1e4)


def shared(p, decode, **kw):
    a = dict(model=MODEL, pages=pic.Pages.of(8, 16, 4), groups=pic.Shared.of(1, 2, 20), q=p, k=p, v=p, pk=p, pv=p, table=p, batch=2,
             start=p, len=p, lens=p, max=10, step=0, nv=None, n=3, scale=0.0, out=p, ws=p, ws_bytes=0)
    a.update(kw)
    head = (ctypes.byref(a["model"]), ctypes.byref(a["pages"]), ctypes.byref(a["groups"]) if a["groups"] else None, a["q"], a["k"],
            a["v"], a["pk"], a["pv"], a["table"], a["batch"], a["start"], a["len"], a["lens"])
    tail = (a["scale"], a["out"], a["ws"], a["ws_bytes"], None)
    if decode:
        return pic.load().pic_page_shared_decode_attn(*head, a["step"], a["max"], *tail)
    return pic.load().pic_page_shared_suffix_attn(*head, a["max"], a["nv"], a["n"], *tail)


@pytest.mark.parametrize("decode", [True, False])
def test_shared_refusals(p, decode):
    call = lambda **kw: shared(p, decode, **kw)  # noqa: E731
    M, G, S = pic.Model, pic.Pages, pic.Shared
    assert call() == WORKSPACE
    assert call(ws=None, ws_bytes=1 << 20) == WORKSPACE
    assert call(ws=p + 8, ws_bytes=1 << 20) == MISALIGNED
    assert call(model=M.of(1, 4, 2, 80, "bf16", 1e4)) == UNSUPPORTED
    assert call(pages=G.of(8, 24, 4)) == UNSUPPORTED
    assert call(pages=G.of(0, 16, 4)) == RANGE
    assert call(groups=None) == INVALID
    for bad in (S.of(0, 2, 20), S.of(-1, 2, 20), S.of(1, -1, 20), S.of(1, 2, -1)):
        assert call(groups=bad) == INVALID
    assert call(groups=S.of(1, 2, 65)) == CAPACITY        # past the page table
    assert call(groups=S.of(2, 2, 20), start=None) == INVALID
    assert call(groups=S.of(1, 2, 20), start=None) == WORKSPACE
    assert call(max=64) == CAPACITY
    assert call(max=2**31 - 1) == CAPACITY
    for k in ("batch", "max"):
        assert call(**{k: -1}) == INVALID
    for s in (-1.0, float("nan"), float("inf")):
        assert call(scale=s) == INVALID
    for k in ("q", "k", "v", "pk", "pv", "out"):
        assert call(**{k: None}) == INVALID
        assert call(**{k: p + 8}) == MISALIGNED
    for k in ("table", "lens", "len"):
        assert call(**{k: None}) == INVALID
    assert call(batch=0, q=None) == 0
    assert call(model=M.of(0, 4, 2, 64, "bf16", 1e4)) == 0
    assert call(batch=1 << 30) == UNSUPPORTED
    assert call(groups=S.of(1 << 24, 2, 20)) == UNSUPPORTED
    many = 2**31 - 1
    assert call(batch=many, model=M.of(many, many, 1, 64, "bf16", 1e4)) == UNSUPPORTED
    if decode:
        assert call(step=-1) == INVALID
        assert call(step=60) == CAPACITY
    else:
        assert call(n=-1) == INVALID
        assert call(n=60) == CAPACITY
        assert call(n=0) == 0
    wide = G.of(8, 1024, 1 << 21)
    assert call(pages=wide, max=2**30, batch=0) == CAPACITY


def test_shared_workspace_query():
    q = lambda m=MODEL, s=pic.Shared.of(1, 4, 1000), b=4, n=1, c=2000: pic.pic_page_shared_workspace_bytes(m, s, b, n, c)  # noqa: E731
    assert q() > 0 and q(b=0) == 0 and q(n=0) == 0
    assert q(b=-1) == 0 and q(c=-1) == 0 and q(c=2**31 - 1) == 0 and q(s=pic.Shared.of(0, 1, 1)) == 0
    assert q(m=pic.Model.of(1, 4, 2, 64, "f32", 1e4)) == 0
    assert q(m=pic.Model.of(1, 4, 2, 80, "bf16", 1e4)) == 0


@pytest.mark.parametrize("model", [(1, 32, 8, 128), (2, 28, 4, 128), (1, 4, 2, 64), (32, 32, 8, 128), (1, 1, 1, 64)])
def test_one_workspace_serves_smaller_calls(model):
    """What is asked for at the largest sizes is enough at every size before them: each step of a decode loop, fewer requests,
    fewer tokens, shorter prefixes."""
    m = pic.Model.of(*model, "bf16", 1e4)
    for groups, batch, n in (((1, 2, 2048), 2, 1), ((4, 12, 8192), 37, 1), ((70, 3, 640), 140, 1), ((1, 64, 16384), 64, 1), ((2, 8, 0), 16, 3),
                             ((1, 16, 1000), 16, 131), ((2, 0, 500), 4, 1), ((1, 3, 4000), 200, 2)):
        need = lambda b=batch, t=n, s=groups[2], c=20000: pic.pic_page_shared_workspace_bytes(  # noqa: E731
            m, pic.Shared.of(*groups[:2], s), b, t, c)
        for sizes in ([need(c=c) for c in [*range(0, 700), *range(701, 20000, 61)]], [need(b=b) for b in range(1, batch + 1)],
                      [need(t=t) for t in range(1, n + 1)], [need(s=s) for s in range(0, groups[2] + 1, 16)]):
            assert sizes == sorted(sizes) and sizes[0] > 0


def test_shared_binding_refusals():
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    pages, groups = pic.Pages.of(8, 16, 4), pic.Shared.of(2, 2, 20)
    for start, length, name in ((i32(2), i32(2), "group_start"), (i32(3).long(), i32(2), "group_start"), (i32(3), i32(1), "shared_len"),
                                (i32(3), i32(2).float(), "shared_len")):
        with pytest.raises(ValueError, match=name):
            pic.pic_page_shared_decode_attn(MODEL, pages, groups, None, None, None, None, None, None, 2, start, length, None, 0, 10, None)
        with pytest.raises(ValueError, match=name):
            pic.pic_page_shared_suffix_attn(MODEL, pages, groups, None, None, None, None, None, None, 2, start, length, None, 10, 1, None)


def test_copy_listed_binding_refusals():
    model, pages = pic.Model.of(1, 2, 2, 64, "f32", 1e4), pic.Pages.of(4, 16, 0)
    for pairs in (torch.zeros((2, 2), dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int64)):
        with pytest.raises(ValueError, match="pairs"):
            pic.pic_page_copy_async(model, pages, None, None, pairs, 3)


def test_grow_refusals(p):
    def call(pages=pic.Pages.of(8, 16, 4), batch=2, refs=p, table=p, lens=p, offset=0, nv=None, n=3, pairs=p, ready=p, result=p, ws=p,
             ws_bytes=1 << 12):
        return pic.load().pic_page_grow_async(ctypes.byref(pages), batch, refs, table, lens, offset, nv, n, pairs, ready, result, ws,
                                              ws_bytes, None)

    G = pic.Pages.of
    need = pic.pic_page_grow_workspace_bytes(G(8, 16, 4), 2, 3)
    assert need > 0
    assert call(ws_bytes=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=p + 4) == MISALIGNED
    assert call(pages=G(8, 24, 4)) == UNSUPPORTED and call(pages=G(-1, 16, 4)) == INVALID and call(pages=G(8, 16, -4)) == INVALID
    for k in ("batch", "offset", "n"):
        assert call(**{k: -1}) == INVALID
    for k in ("refs", "table", "lens", "pairs", "ready", "result"):
        assert call(**{k: None}) == INVALID
    for k in ("refs", "table", "pairs", "ready", "result"):
        assert call(**{k: p + 4}) == MISALIGNED
    assert call(pages=G(8, 16, 1 << 24), batch=1 << 10, n=1 << 28) == UNSUPPORTED
    assert pic.pic_page_grow_workspace_bytes(G(8, 16, 1 << 24), 1 << 10, 1 << 28) == 0
    assert pic.pic_page_grow_workspace_bytes(G(8, 17, 4), 2, 3) == 0


def test_copy_listed_refusals(p):
    def call(model=MODEL, pages=pic.Pages.of(8, 16, 0), k=p, v=p, pairs=p, cap=2):
        return pic.load().pic_page_copy_async(ctypes.byref(model), ctypes.byref(pages), k, v, pairs, cap, None)

    assert call(cap=-1) == INVALID and call(cap=0, k=None) == 0
    assert call(k=None) == INVALID and call(v=p + 8) == MISALIGNED and call(pairs=None) == INVALID and call(pairs=p + 8) == MISALIGNED
    assert call(pages=pic.Pages.of(8, 15, 0)) == UNSUPPORTED and call(pages=pic.Pages.of(0, 16, 0)) == 0
    assert call(model=pic.Model.of(0, 4, 2, 64, "bf16", 1e4)) == 0
    assert call(model=pic.Model.of(1, 4, 2, 96, "bf16", 1e4)) == UNSUPPORTED


def test_norm_refusals(p):
    def call(model=MODEL, how=None, q=p, qs=0, k=p, ks=0, v=p, vs=0, batch=2, lens=p, max=10, offset=0, nv=None, n=3, table=p, mad=12,
             qo=p, ko=p, vo=p, eps=1e-6, rope_dim=0, order=0, scale=1.0, qw=p, kw=p):
        x = pic.QkNorm(qw, kw, eps, rope_dim, order, scale)
        return pic.load().pic_qk_norm_rope(ctypes.byref(model), ctypes.byref(x) if how is None else None, q, qs, k, ks, v, vs, batch,
                                           lens, max, offset, nv, n, table, mad, qo, ko, vo, None)

    assert call(how=False) == INVALID
    assert call(model=pic.Model.of(1, 4, 2, 80, "bf16", 1e4)) == UNSUPPORTED
    for k in ("batch", "max", "offset", "n"):
        assert call(**{k: -1}) == INVALID
    for e in (-1.0, float("nan"), float("inf")):
        assert call(eps=e) == INVALID
    assert call(scale=float("nan")) == INVALID and call(order=2) == INVALID
    for r in (8, 72, -16, 80, 24):
        assert call(rope_dim=r) == UNSUPPORTED
    assert call(mad=11) == RANGE and call(mad=-1) == RANGE and call(mad=(1 << 20) + 1) == RANGE
    assert call(offset=1) == RANGE and call(lens=None, mad=1) == RANGE
    assert call(n=2**31 - 1, max=2**31 - 1) == RANGE
    assert call(table=p + 8) == MISALIGNED
    for x in "qkv":
        assert call(**{x + "o": None}) == INVALID
        assert call(**{x: p + 8}) == MISALIGNED and call(**{x + "o": p + 8}) == MISALIGNED
        assert call(**{x + "s": 64}) == INVALID           # less than a row
        assert call(**{x + "s": 300}) == MISALIGNED
        assert call(**{x + "s": 264}) == INVALID          # in place, not dense
    assert call(qw=p + 4) == MISALIGNED and call(kw=p + 4) == MISALIGNED
    assert call(q=None, k=None, v=None) == 0 and call(n=0, q=None) == 0 and call(batch=0) == 0
    assert call(batch=1 << 30, lens=None) == UNSUPPORTED
    assert call(model=pic.Model.of(70000, 4, 2, 64, "bf16", 1e4)) == UNSUPPORTED


def test_norm_binding_refusals():
    q = torch.zeros(2, 3, 4, 64)
    how = pic.QkNorm(None, None, 1e-6, 0, 0, 1.0)
    rows = pic._token_rows
    for bad in (q[..., :3, :], q[..., :32], q.transpose(0, 1), q.transpose(2, 3), torch.zeros(4, 3, 8, 128)[::2, :, :4, ::2]):
        with pytest.raises(ValueError):
            rows(bad, 4, 64, "q", -1)
    assert rows(q, 4, 64, "q", -1) == (q.data_ptr(), 256)
    wide = torch.zeros(2, 3, 5 * 64)
    assert rows(wide[..., 64:].unflatten(-1, (4, 64)), 4, 64, "q", -1) == (wide.data_ptr() + 256, 320)
    with pytest.raises(ValueError, match="host"):
        rows(q, 4, 64, "q", 0)
    assert how.eps > 0
    with pytest.raises(ValueError, match="float32"):
        pic.QkNorm.of(torch.zeros(64, dtype=torch.bfloat16), None)


def test_yarn_frequencies():
    for d, r, theta, factor, orig, fast, slow in ((128, 0, 1e6, 4.0, 32768, 32, 1), (64, 32, 1e4, 8.0, 8192, 32, 1),
                                                  (128, 64, 5e5, 40.0, 4096, 32, 1), (128, 0, 1e4, 1.0, 4096, 16, 2)):
        got, scale = pic.pic_rope_yarn_freq(d, theta, factor, orig, fast, slow, rope_dim=r)
        n = r or d
        # the definition: pair i turns L theta_i / (2 pi) times over L positions
        at = lambda turns: n * math.log(orig / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), n - 1)
        want = np.zeros(d // 2)
        for i in range(n // 2):
            f = theta ** (-2.0 * i / n)
            keep = 1.0 if i < lo else 0.0 if i > hi else 1.0 - (i - lo) / max(hi - lo, 1e-3)
            want[i] = f * keep + f / factor * (1 - keep)
        assert np.allclose(got, want, rtol=1e-14, atol=0)
        assert scale == pytest.approx(0.1 * math.log(factor) + 1)
    for kw in (dict(factor=0.5), dict(beta_slow=0.0), dict(beta_fast=1.0), dict(theta=1.0), dict(original_max_position=0.0)):
        a = dict(theta=1e4, factor=4.0, original_max_position=4096.0, beta_fast=32.0, beta_slow=1.0)
        a.update(kw)
        with pytest.raises(pic.PicError) as e:
            pic.pic_rope_yarn_freq(128, **a)
        assert e.value.status == INVALID
    for d, r, st in ((96, 0, INVALID), (64, 128, UNSUPPORTED), (64, 24, UNSUPPORTED)):
        with pytest.raises(pic.PicError) as e:
            pic.pic_rope_yarn_freq(d, 1e4, 4.0, 4096.0, rope_dim=r)
        assert e.value.status == st

