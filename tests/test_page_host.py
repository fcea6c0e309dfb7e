"""Host side of the paged cache: bookkeeping calls against a model that follows every token, gather
blocks cut into pages, and every refusal (none of which needs a GPU)."""
import ctypes
import os

import numpy as np
import pytest
from hypothesis import given, settings
from hypothesis import strategies as st

import paper_2607_28069_amd as pic

INVALID, UNSUPPORTED, WORKSPACE, CAPACITY, MISALIGNED, RANGE = -1, -2, -3, -4, -5, -6


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(pic.LIB_PATH):
        from paper_2607_28069_amd.build import build
        build()
    return pic.load()


def fails(status, call, *args, **kw):
    with pytest.raises(pic.PicError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


class Book:
    """refs and table, the memory of one stream and, apart from them, the tokens every request should hold."""

    def __init__(self, n_pages, P, cap, batch):
        self.pages = pic.Pages.of(n_pages, P, cap)
        self.refs = np.zeros(n_pages, np.int32)
        self.table = np.full((batch, cap), -1, np.int32)
        self.mem = np.full(n_pages * P, -1, np.int64)
        self.want = [[] for _ in range(batch)]
        self.next = 0

    def state(self):
        return self.refs.copy(), self.table.copy()

    def copy(self, pairs):
        m = self.mem.reshape(self.pages.n_pages, -1)
        old = m.copy()
        src, dst = pairs[:, 0], pairs[:, 1]
        assert len(set(dst)) == len(dst) and not set(dst) & set(src)
        m[dst] = old[src]

    def check(self):
        P = self.pages.page_tokens
        held = np.bincount(self.table[self.table >= 0], minlength=self.pages.n_pages)
        assert (held == self.refs).all()
        for b, w in enumerate(self.want):
            rows = [self.table[b, t // P] * P + t % P for t in range(len(w))]
            assert [int(self.mem[r]) for r in rows] == w

    def grow(self, add):
        ln = [len(w) for w in self.want]
        before = self.state()
        try:
            pairs = pic.pic_page_grow(self.pages, self.refs, self.table, ln, [n + a for n, a in zip(ln, add)])
        except pic.PicError as e:
            assert e.status == CAPACITY
            assert all((x == y).all() for x, y in zip(before, self.state()))
            return False
        self.copy(pairs)
        P = self.pages.page_tokens
        for b, a in enumerate(add):
            for _ in range(a):
                t = len(self.want[b])
                page = self.table[b, t // P]
                assert self.refs[page] == 1   # a page that is written belongs to one request
                self.mem[page * P + t % P] = self.next
                self.want[b].append(self.next)
                self.next += 1
        return True


@settings(max_examples=60, deadline=None)
@given(st.data())
def test_bookkeeping_keeps_every_token(data):
    batch, P = data.draw(st.integers(1, 5)), 16
    k = Book(data.draw(st.integers(1, 24)), P, data.draw(st.integers(1, 8)), batch)
    for _ in range(data.draw(st.integers(1, 14))):
        op = data.draw(st.sampled_from(["grow", "grow", "fork", "free", "compact"]))
        if op == "grow":
            k.grow([data.draw(st.sampled_from([0, 1, 7, 15, 16, 17, 33])) for _ in range(batch)])
        elif op == "fork" and batch > 1:
            src, dst = data.draw(st.permutations(range(batch)))[:2]
            n = data.draw(st.integers(0, len(k.want[src])))
            if (k.table[dst] >= 0).any():
                fails(INVALID, pic.pic_page_fork, k.pages, batch, k.refs, k.table, src, n, dst)
            else:
                pic.pic_page_fork(k.pages, batch, k.refs, k.table, src, n, dst)
                k.want[dst] = k.want[src][:n]
        elif op == "free":
            b = data.draw(st.integers(0, batch - 1))
            keep = data.draw(st.integers(0, len(k.want[b])))
            pic.pic_page_free(k.pages, batch, k.refs, k.table, b, keep)
            k.want[b] = k.want[b][:keep]
        elif op == "compact":
            pairs, used = pic.pic_page_compact(k.pages, batch, k.refs, k.table)
            k.copy(pairs)
            assert (k.refs[:used] > 0).all() and (k.refs[used:] == 0).all()
        k.check()


def test_last_sharer_keeps_the_page():
    k = Book(8, 16, 4, 3)
    assert k.grow([20, 0, 0])
    for dst in (1, 2):
        pic.pic_page_fork(k.pages, 3, k.refs, k.table, 0, 20, dst)
        k.want[dst] = list(k.want[0])
    assert list(k.refs[:3]) == [3, 3, 0]
    assert k.grow([1, 1, 1])
    assert k.refs[0] == 3 and k.refs[1] == 1 and (k.refs[:4] > 0).all()
    k.check()
    # a fork that ends at a page border shares without a copy when it grows
    pic.pic_page_free(k.pages, 3, k.refs, k.table, 2)
    pic.pic_page_fork(k.pages, 3, k.refs, k.table, 0, 16, 2)
    k.want[2] = k.want[0][:16]
    pairs = pic.pic_page_grow(k.pages, k.refs, k.table, [0, 0, 16], [0, 0, 17])
    assert len(pairs) == 0


def test_a_grown_table_over_a_shared_whole_page_takes_a_new_one():
    # request 0 holds two pages for 16 tokens (grown ahead); the second is shared by a fork of 17 slots
    pages = pic.Pages.of(6, 16, 3)
    refs, table = np.zeros(6, np.int32), np.full((2, 3), -1, np.int32)
    pic.pic_page_grow(pages, refs, table, [0, 0], [32, 0])
    pic.pic_page_fork(pages, 2, refs, table, 0, 32, 1)
    pairs = pic.pic_page_grow(pages, refs, table, [16, 0], [20, 0])   # slots 16.. are written anew: nothing to copy
    assert len(pairs) == 0 and table[0, 1] != table[1, 1] and refs[table[0, 1]] == 1


def test_bookkeeping_refusals():
    pages = pic.Pages.of(4, 16, 2)
    refs, table = np.zeros(4, np.int32), np.full((2, 2), -1, np.int32)
    P = pic.Pages
    for bad in (P.of(4, 8, 2), P.of(4, 48, 2), P.of(4, 2048, 2), P.of(4, 0, 2), P.of(1 << 28, 16, 2)):
        r = np.zeros(max(bad.n_pages, 0) if bad.n_pages < 1 << 20 else 0, np.int32)
        st_ = pic.load().pic_page_free(ctypes.byref(bad), 2, r.ctypes.data, table.ctypes.data, 0, 0)
        assert st_ == UNSUPPORTED
    grow = lambda *a: pic.pic_page_grow(pages, refs, table, *a)  # noqa: E731
    fails(INVALID, grow, [-1, 0], [5, 0])
    fails(CAPACITY, grow, [0, 0], [33, 0])           # the table holds two pages per request
    fails(RANGE, grow, [5, 0], [6, 0])               # slot 5 sits in a page the request does not hold
    table[0, 0] = 9
    fails(RANGE, grow, [5, 0], [6, 0])
    table[0, 0] = 1
    fails(RANGE, grow, [5, 0], [6, 0])               # a page without a reference
    fails(RANGE, pic.pic_page_fork, pages, 2, refs, table, 0, 5, 1)
    fails(RANGE, pic.pic_page_free, pages, 2, refs, table, 0)
    fails(RANGE, pic.pic_page_compact, pages, 2, refs, table)
    table[0, 0] = -1
    fails(INVALID, pic.pic_page_fork, pages, 2, refs, table, 1, 0, 1)
    fails(RANGE, pic.pic_page_fork, pages, 2, refs, table, 2, 0, 1)
    fails(RANGE, pic.pic_page_fork, pages, 2, refs, table, 0, 0, -1)
    fails(CAPACITY, pic.pic_page_fork, pages, 2, refs, table, 0, 33, 1)
    fails(INVALID, pic.pic_page_fork, pages, 2, refs, table, 0, -1, 1)
    fails(RANGE, pic.pic_page_free, pages, 2, refs, table, 2)
    fails(INVALID, pic.pic_page_free, pages, 2, refs, table, 0, -1)
    refs[3] = 1
    fails(INVALID, pic.pic_page_compact, pages, 2, refs, table)   # held from outside the table
    refs[3] = 0
    assert (refs == 0).all() and (table == -1).all()
    with pytest.raises(ValueError):
        pic.pic_page_free(pages, 2, refs[:3], table, 0)
    with pytest.raises(ValueError):
        pic.pic_page_free(pages, 2, refs, table.astype(np.int64), 0)
    with pytest.raises(ValueError):
        pic.pic_page_free(pages, 2, refs, table.T, 0)
    # a compaction with too little room for its pairs says how many it needs and changes nothing
    pic.pic_page_grow(pages, refs, table, [0, 0], [16, 16])
    pic.pic_page_free(pages, 2, refs, table, 0)
    before = refs.copy(), table.copy()
    n, used = ctypes.c_int32(0), ctypes.c_int32(0)
    assert pic.load().pic_page_compact(ctypes.byref(pages), 2, refs.ctypes.data, table.ctypes.data, None, 0,
                                       ctypes.byref(n), ctypes.byref(used)) == CAPACITY
    assert n.value == 1 and (refs == before[0]).all() and (table == before[1]).all()


@settings(max_examples=60, deadline=None)
@given(st.data())
def test_blocks_cut_at_page_borders(data):
    P = data.draw(st.sampled_from([16, 32, 64, 128]))
    batch = data.draw(st.integers(1, 3))
    lens = np.array(data.draw(st.lists(st.integers(1, 150), min_size=1, max_size=6)))
    offs = np.concatenate([[0], np.cumsum(lens)[:-1]])
    reqs = [data.draw(st.lists(st.integers(0, len(lens) - 1), max_size=4)) for _ in range(batch)]
    blocks, ctx = pic.pic_plan_layout(reqs, offs, lens, np.zeros_like(lens), int(lens.sum()))
    need = [-(-int(c) // P) for c in ctx]
    pages = pic.Pages.of(max(sum(need), 1) + 3, P, max(need + [1]))
    order = np.random.default_rng(data.draw(st.integers(0, 99))).permutation(pages.n_pages)
    table, at = np.full((batch, pages.table_cap), -1, np.int32), 0
    for b in range(batch):
        table[b, : need[b]] = order[at: at + need[b]]
        at += need[b]
    got = {}
    for b in pic.pic_page_blocks(pages, table, blocks):
        assert b["request"] == 0 and 1 <= b["n_tokens"] <= 64
        assert b["dst_slot"] // P == (b["dst_slot"] + b["n_tokens"] - 1) // P
        for t in range(b["n_tokens"]):
            assert int(b["dst_slot"]) + t not in got
            got[int(b["dst_slot"]) + t] = (int(b["src_token"]) + t, int(b["delta"]))
    want = {}
    for b in blocks:
        for t in range(b["n_tokens"]):
            slot = int(b["dst_slot"]) + t
            want[int(table[b["request"], slot // P]) * P + slot % P] = (int(b["src_token"]) + t, int(b["delta"]))
    assert got == want


def test_blocks_refusals():
    blocks, _ = pic.pic_plan_layout([[0]], [0], [70], [0], 70)
    pages = pic.Pages.of(4, 32, 3)
    table = np.array([[2, 0, 3]], np.int32)
    assert len(pic.pic_page_blocks(pages, table, blocks)) == 3
    for bad in ([[2, -1, 3]], [[2, 4, 3]]):
        fails(RANGE, pic.pic_page_blocks, pages, np.array(bad, np.int32), blocks)
    fails(RANGE, pic.pic_page_blocks, pic.Pages.of(4, 32, 2), table[:, :2], blocks)   # slots past the table
    fails(RANGE, pic.pic_page_blocks, pages, np.zeros((0, 3), np.int32), blocks)
    with pytest.raises(ValueError):
        pic.pic_page_blocks(pages, table[:, :2], blocks)


# ---- the calls that launch: refused before anything is enqueued, so host addresses will do ----

BUF = 1 << 16


@pytest.fixture(scope="module")
def p():
    raw = ctypes.create_string_buffer(4096)
    a = ctypes.addressof(raw)
    p.raw = raw
    return a + (-a) % 256


def _attn(p, model=None, pages=None, name="pic_page_decode_attn", **kw):
    d = dict(q=p, k=p, v=p, pk=p, pv=p, table=p, batch=1, lens=p, step=0, max=15, n_valid=None, n=1, rope=p, mad=64,
             scale=0.0, splits=1, out=p, ws=None, ws_bytes=0)
    assert set(kw) <= set(d)
    d.update(kw)
    m = model if model is not None else pic.Model.of(1, 4, 2, 64, "bf16", 1e4)
    g = pages if pages is not None else pic.Pages.of(8, 16, 4)
    head = [ctypes.byref(m), ctypes.byref(g), d["q"], d["k"], d["v"], d["pk"], d["pv"], d["table"], d["batch"], d["lens"]]
    mid = [d["step"], d["max"]] if "decode" in name else [d["max"], d["n_valid"], d["n"]]
    if "rope" in name:
        mid += [d["rope"], d["mad"]]
    mid += [d["scale"]] + ([d["splits"]] if "decode" in name else [])
    return getattr(pic.load(), name)(*head, *mid, d["out"], d["ws"], d["ws_bytes"], None)


NAMES = ["pic_page_decode_attn", "pic_page_decode_attn_rope", "pic_page_suffix_attn", "pic_page_suffix_attn_rope"]


@pytest.mark.parametrize("name", NAMES)
def test_attention_refusals(p, name):
    call = lambda **kw: _attn(p, name=name, **kw)  # noqa: E731
    M, G = pic.Model, pic.Pages
    assert call(model=M.of(1, 4, 2, 80, "bf16", 1e4)) == UNSUPPORTED
    assert call(model=M.of(1, 4, 3, 64, "bf16", 1e4)) == INVALID
    assert call(pages=G.of(8, 24, 4)) == UNSUPPORTED
    assert call(pages=G.of(-1, 16, 4)) == INVALID
    assert call(pages=G.of(8, 16, -1)) == INVALID
    assert call(pages=G.of(1 << 27, 16, 4)) == UNSUPPORTED
    assert call(pages=G.of(0, 16, 4)) == RANGE
    assert call(max=64) == CAPACITY
    assert call(max=2**31 - 1) == CAPACITY
    for k in ("batch", "max"):
        assert call(**{k: -1}) == INVALID
    for s in (-1.0, float("nan"), float("inf")):
        assert call(scale=s) == INVALID
    for k in ("q", "k", "v", "pk", "pv", "out"):
        assert call(**{k: None}) == INVALID
        assert call(**{k: p + 8}) == MISALIGNED
    assert call(table=None) == INVALID
    assert call(lens=None) == INVALID
    assert call(batch=0) == 0 and call(batch=0, q=None) == 0
    assert call(model=M.of(0, 4, 2, 64, "bf16", 1e4)) == 0
    assert call(batch=1 << 30) == UNSUPPORTED   # query rows
    if "rope" in name:
        assert call(rope=None) == INVALID
        assert call(rope=p + 8) == MISALIGNED
        assert call(mad=14) == RANGE
        assert call(mad=(1 << 20) + 1) == RANGE
        assert call(model=M.of(1, 4, 2, 64, "f32", 1e4)) == UNSUPPORTED
    if "decode" in name:
        assert call(step=-1) == INVALID
        assert call(splits=-1) == INVALID
        assert call(step=60) == CAPACITY
        assert call(splits=2) == WORKSPACE
        assert call(splits=2, ws=p + 8, ws_bytes=1 << 20) == MISALIGNED
        # float32 and bf16 decode address rows with 64 bits: no limit below INT32_MAX rows
    else:
        assert call(n=-1) == INVALID
        assert call(n=50) == CAPACITY
        assert call(n=0) == 0
        assert call(pages=G.of(1 << 20, 16, 4)) == UNSUPPORTED   # a stream of 2^24 rows


@pytest.mark.parametrize("name", NAMES)
def test_attention_refuses_requests_past_2_30_slots(p, name):
    """Tables that name pages more than once can hold positions past those the pages have."""
    wide = pic.Pages.of(8, 1024, 1 << 21)
    assert _attn(p, name=name, pages=wide, max=2**30, batch=0) == CAPACITY
    assert _attn(p, name=name, pages=wide, max=2**31 - 1, batch=0) == CAPACITY
    at_limit = _attn(p, name=name, pages=wide, max=2**30 - 8, batch=0)
    assert at_limit == (RANGE if "rope" in name else 0)   # rope: no table is that long


def test_copy_refusals(p):
    m, g = pic.Model.of(1, 4, 2, 64, "bf16", 1e4), pic.Pages.of(8, 16, 0)

    def call(pairs, k=p, v=p, model=m, pages=g, n=None):
        a = np.ascontiguousarray(pairs, np.int32).reshape(-1, 2)
        return pic.load().pic_page_copy(ctypes.byref(model), ctypes.byref(pages), k, v, a.ctypes.data,
                                        len(a) if n is None else n, None)

    assert call([[0, 8]]) == RANGE
    assert call([[-1, 3]]) == RANGE
    assert call([[0, 1], [2, 1]]) == INVALID        # written twice
    assert call([[0, 1], [1, 2]]) == INVALID        # written and read
    assert call([[3, 3]]) == INVALID
    assert call([[0, 1]], n=9) == INVALID and call([[0, 1]], n=-1) == INVALID
    assert call([[0, 1]], k=None) == INVALID and call([[0, 1]], v=p + 8) == MISALIGNED
    assert call([[0, 1]], model=pic.Model.of(0, 4, 2, 64, "bf16", 1e4)) == 0
    assert call(np.zeros((0, 2)), k=None) == 0
    big = np.stack([np.arange(400), np.arange(400) + 400], 1)
    assert call(np.concatenate([big, [[0, 500]]]), pages=pic.Pages.of(1000, 16, 0)) == INVALID
    assert call(np.concatenate([big, [[700, 900]]]), pages=pic.Pages.of(1000, 16, 0)) == INVALID
