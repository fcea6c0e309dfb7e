"""Attention over pages for batches that share prefixes, against the definition in 64 bits: head layouts, page sizes,
groups of every size, shared lengths around the tiles, padding, several tokens per request, bad tables, what is not
finite, and the calls' refusals of too little workspace."""
import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, SENTINEL, check, check_pages, reference, rows
from shared_path import batch, decode, starts, suffix, workspace

pytestmark = pytest.mark.gpu


def right(x, **kw):
    """Probabilities over shared slots keep 16 bits up to 64 query rows of a group, and 8 beyond (one rounding of 2^-8 each, which
    the numerator and the denominator see: as in a prefill)."""
    check(x, decoded=x.shared.max_group * x.n * (x.hq // x.hkv) <= 64, **kw)


HEADS = [(4, 2, 64), (32, 8, 128), (28, 4, 128), (5, 1, 64), (3, 3, 128), (40, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("P", [16, 64, 256])
def test_decode(hq, hkv, d, P):
    # a group over 5 tiles and a bit, one of a single request, one that shares nothing, one with padding
    ctx = [333, 400, 333, 511, 70, 20, 0, 190, -1, 130]
    x = batch(hq, hkv, d, P, ctx, [1] * 10, [0, 4, 5, 7, 10], [333, 70, 0, 130])
    decode(x)
    right(x)


@pytest.mark.parametrize("shared", [1, 15, 63, 64, 65, 127, 128, 200])
@pytest.mark.parametrize("own", [0, 1, 63, 64])
def test_decode_borders(shared, own):
    for P in (16, 128):
        x = batch(8, 2, 128, P, [shared + own, shared, shared + own // 2], [1] * 3, [0, 3], [shared], slack=9)
        decode(x)
        right(x)


@pytest.mark.parametrize("sizes", [[2], [17], [33], [1, 40, 3], [16, 16, 16, 16]])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 2, 64)])
def test_decode_groups(sizes, hq, hkv, d):
    """Row tiles full, in part, and more than one; prefixes in many ranges."""
    r = np.random.default_rng(len(sizes))
    shared = [int(r.integers(600, 2100)) for _ in sizes]
    ctx = [s + int(r.integers(0, 150)) for s, n in zip(shared, sizes) for _ in range(n)]
    x = batch(hq, hkv, d, 32, ctx, [1] * len(ctx), starts(sizes), shared, L=2)
    decode(x, step=3)
    right(x)


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (4, 2, 64), (40, 1, 64)])
@pytest.mark.parametrize("n", [2, 5, 17, 70])
def test_suffix(hq, hkv, d, n):
    ctx = [700, 641, 640, 800, 0, 90, 90, -1]
    new = [n, 1, n // 2, 0, n, n - 1, n, n]
    x = batch(hq, hkv, d, 64, ctx, new, [0, 4, 5, 8], [640, 0, 90], n=n)
    suffix(x)
    right(x)


@pytest.mark.parametrize("n", [1, 33])
def test_suffix_row_tiles(n):
    x = batch(32, 4, 128, 16, [1300, 1290, 1300, 1281, 1300, 1500], [n] * 6, [0, 6], [1281], n=n, L=2)
    suffix(x, n_valid=None)
    right(x)


def test_no_groups_and_all_in_one():
    """Without starts the batch is one group; requests before the first start and after the last share nothing."""
    x = batch(8, 2, 128, 64, [200, 210, 250], [1] * 3, [0, 3], [200])
    decode(x, start=None)
    right(x)
    x = batch(8, 2, 128, 64, [200, 210, 250, 300, 100], [1] * 5, [0, 1, 4, 5], [0, 200, 0])
    x.start, x.shared_len = x.start[1:3].clone(), x.shared_len[1:2].clone()
    x.shared = pic.Shared.of(1, 3, 200)
    decode(x)
    right(x)


def test_bounds_below_the_lengths():
    """Requests past max_group in their group share nothing, and neither do slots past max_len: outputs are the same."""
    x = batch(8, 2, 128, 64, [400, 410, 450, 401], [1] * 4, [0, 4], [400])
    x.shared = pic.Shared.of(1, 2, 300)
    decode(x)
    right(x)


def test_requests_shorter_than_the_prefix():
    """Requests whose new tokens come before the end of the shared slots see their own slots only."""
    x = batch(8, 2, 128, 32, [500, 100, 63, 64, 0, 430], [1] * 6, [0, 6], [480])
    decode(x)
    right(x)
    x = batch(8, 2, 64, 32, [500, 100, 63, 64, 0, 430], [9] * 6, [0, 6], [480], n=9)
    suffix(x)
    right(x)


def test_prefix_held_by_padding():
    """The group's first request is padding of the batch: its page table row holds the prefix."""
    x = batch(8, 2, 128, 64, [330, 330, 350, 420], [1] * 4, [0, 4], [330])
    x.ctx[0] = -1
    x.K[0], x.V[0] = x.K[0][:, :, :330], x.V[0][:, :, :330]
    x.len[0] = -1
    decode(x)
    right(x)


def test_a_batch_of_padding():
    x = batch(8, 2, 128, 64, [-1, -1], [1, 1], [0, 2], [0])
    x.shared_len[0] = 64
    decode(x)
    right(x)


def test_the_same_bits_twice_and_with_a_larger_workspace():
    x = batch(32, 8, 128, 64, [1500, 1400, 1333, 1800], [1] * 4, [0, 4], [1333])
    a = decode(x).clone()
    x.out.fill_(SENTINEL)
    big = torch.full((4 * workspace(x, 1, x.max_ctx).numel(),), 0xFF, dtype=torch.uint8, device=DEV)
    assert (decode(x, ws=big) == a).all()
    need = pic.pic_page_shared_workspace_bytes(x.model, x.shared, x.B, 1, x.max_ctx)
    assert (big[need:] == 0xFF).all()
    with pytest.raises(pic.PicError) as e:
        decode(x, ws=big[: need - 16])
    assert e.value.status == -3


def test_scale():
    x = batch(8, 2, 128, 64, [300, 350], [1] * 2, [0, 2], [300])
    decode(x, scale=0.03)
    right(x, scale=0.03)


@pytest.mark.parametrize("n", [1, 3])
def test_f32_pages(n):
    x = batch(8, 2, 64, 16, [300, 350, 310], [n] * 3, [0, 3], [300], dtype="f32", n=n)
    (decode if n == 1 else suffix)(x, ws=None)
    check(x)


def test_rows_past_2_32_bytes():
    """Pages whose byte offsets in a stream pass 2^32."""
    P, n_pages = 1024, 17000
    if torch.cuda.mem_get_info()[0] < 3 * 2 * n_pages * P * 256:
        pytest.skip("too little memory")
    x = batch(4, 1, 128, P, [1000, 1010, 1300], [1] * 3, [0, 3], [1000])
    pk = torch.full((1, 1, n_pages * P, 128), float("nan"), dtype=x.dt, device=DEV)
    pv = pk.clone()
    up = n_pages - x.pages.n_pages
    pk[:, :, up * P:], pv[:, :, up * P:] = x.pk, x.pv
    x.pk, x.pv = pk, pv
    x.table_host = np.where(x.table_host >= 0, x.table_host + up, -1).astype(np.int32)
    x.table = torch.from_numpy(x.table_host).to(DEV)
    x.pages = pic.Pages.of(n_pages, P, x.pages.table_cap)
    decode(x)
    right(x)


def _odd(x, kind):
    """Values that are not finite, in a prefix, in a request's own slots and among the new tokens."""
    inf, nan = float("inf"), float("nan")
    a, b, c = {"inf": (inf, inf, inf), "nan": (nan, nan, nan), "both": (inf, -inf, nan)}[kind]

    def put(req, slot, dim, v):
        x.V[req][0, 0, slot, dim] = v
        if slot < x.ctx[req]:
            x.pv[0, 0, rows(x, req, slot, slot + 1), dim] = v
        else:
            x.v[0, req, slot - x.ctx[req], 0, dim] = v

    for r in range(3):
        put(r, 5, 3, a)             # in a shared tile
        put(r, 5, 4, a)
        put(r, 70, 4, b)            # an infinity of the other sign in the same head dim
        put(r, 129, 9, c)           # in the shared slots that each request reads
    put(1, 140, 17, b)              # one request's own
    put(2, x.ctx[2], 21, a)         # a new token
    if x.n > 1:
        put(0, x.ctx[0] + 1, 30, c)  # seen from the second token on


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("kind", ["inf", "nan", "both"])
def test_values_that_are_not_finite(n, kind):
    """Those a row sees are, in their head dim, summed up in place of the average; others change nothing."""
    x = batch(8, 1, 128, 64, [140, 150, 133], [n] * 3, [0, 3], [131], n=n)
    _odd(x, kind)
    (decode if n == 1 else suffix)(x)
    got = x.out.clone()
    fin = torch.isfinite(torch.stack([torch.isfinite(v).all() * 1.0 for v in x.V]))
    assert fin.all()
    odd = [torch.where(torch.isfinite(v), torch.zeros_like(v), v).double() for v in x.V]
    for b in range(3):
        for i in range(n):
            s = odd[b][0, 0, : x.ctx[b] + i + 1].sum(0)               # [D]: 0, an infinity or NaN
            o = got[0, b, i].double()
            bad = ~torch.isfinite(s)
            assert (torch.isfinite(o) == ~bad).all()
            w = s[bad].expand(x.hq, -1)
            assert ((o[:, bad] == w) | (o[:, bad].isnan() & w.isnan())).all()
    for b in range(3):
        x.V[b] = torch.where(torch.isfinite(x.V[b]), x.V[b], torch.zeros_like(x.V[b]))
    ref, mag, _ = reference(x)
    ok = torch.isfinite(got)
    assert ((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** (-14 if 3 * n * 8 <= 64 else -7) * mag + 1e-30)[ok].all()   # (see right())


def test_keys_that_are_not_finite():
    """A NaN in a visible key makes the outputs of its kv head NaN in the requests that see it, and no others."""
    x = batch(8, 2, 128, 64, [200, 260, 230, 90], [1] * 4, [0, 3, 4], [192, 0])
    x.pk[0, 1, rows(x, 1, 250, 251), 7] = float("nan")
    decode(x)
    assert x.out[0, 1, 0, 4:].isnan().all() and torch.isfinite(x.out[0, 1, 0, :4]).all()
    assert torch.isfinite(x.out[0, [0, 2, 3]]).all()
    x.pk[0, 0, rows(x, 0, 100, 101), 7] = float("nan")
    x.out.fill_(SENTINEL)
    decode(x)
    assert x.out[0, :3, 0, :4].isnan().all() and torch.isfinite(x.out[0, 3]).all()


def test_scores_far_apart():
    """One key far above all others: parts without it add nothing."""
    x = batch(4, 1, 64, 16, [200, 210], [1] * 2, [0, 2], [200])
    x.q.zero_()
    x.q[..., 0] = 1
    for b in range(2):
        x.K[b][..., 0] = -60000.0
        x.K[b][:, :, 130 + b, 0] = 0.0
        r = rows(x, b, 0, x.ctx[b])
        x.pk[:, :, r] = x.K[b][:, :, : x.ctx[b]]
        x.k[:, b, 0] = x.K[b][:, :, -1]
    for b in range(2):   # (rows that both hold: the last written)
        x.K[b][:, :, : x.ctx[b]] = x.pk[:, :, rows(x, b, 0, x.ctx[b])]
    decode(x)
    ref, mag, _ = reference(x)
    assert ((x.out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -14 * mag).all()


def test_streams_and_graph():
    """Captured, replayed with new inputs and other lengths, eager calls in between; then on a stream of its own."""
    x = batch(32, 8, 128, 64, [900, 910, 950, 980], [1] * 4, [0, 4], [900], slack=64)
    ws = workspace(x, 1, x.max_ctx)
    eager = decode(x, ws=ws).clone()
    right(x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        decode(x, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        decode(x, ws=ws)
    for it in range(4):
        x.out.fill_(SENTINEL)
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert (x.out == eager).all(), it
        x.out.fill_(SENTINEL)
        assert (decode(x, ws=ws) == eager).all()
    x.q.copy_(torch.randn_like(x.q))
    x.len[1] = x.ctx[1] = 905
    x.K[1] = torch.cat([x.K[1][:, :, :905], x.k[:, 1].transpose(1, 2)], 2)
    x.V[1] = torch.cat([x.V[1][:, :, :905], x.v[:, 1].transpose(1, 2)], 2)
    x.pk[:, :, rows(x, 1, 906, 911)] = float("nan")
    x.pv[:, :, rows(x, 1, 906, 911)] = float("nan")
    g.replay()
    torch.cuda.synchronize()
    replayed = x.out.clone()
    with torch.cuda.stream(side):
        x.out.fill_(SENTINEL)
        decode(x, ws=torch.empty_like(ws))
    torch.cuda.synchronize()
    assert (x.out == replayed).all()
    right(x)


def test_bad_tables_stay_in_bounds():
    """Entries, starts and lengths out of range read some page and store nothing outside: outputs are values or NaN, pages
    change only where a table entry is a page."""
    r = np.random.default_rng(0)
    for it in range(6):
        x = batch(8, 2, 64, 16, [300, 350, 310, 333, 200], [3] * 5, [0, 3, 5], [300, 200], n=3)
        torch.cuda.synchronize()
        x.table = torch.from_numpy(r.integers(-2**31, 2**31, x.table_host.shape).astype(np.int32)).to(DEV)
        x.start = torch.from_numpy(r.integers(-9, 9, 3).astype(np.int32)).to(DEV)
        x.shared_len = torch.from_numpy(r.integers(-2**31, 2**31, 2).astype(np.int32)).to(DEV)
        if it % 2:
            x.len = torch.from_numpy(r.integers(-2**31, 2**31, 5).astype(np.int32)).to(DEV)
            x.n_valid = torch.from_numpy(r.integers(-2**31, 2**31, 5).astype(np.int32)).to(DEV)
        before = x.pk.clone()
        suffix(x)
        torch.cuda.synchronize()
        assert (x.pk.view(torch.int16) == before.view(torch.int16)).all()


@pytest.mark.parametrize("sizes", [[1, 2, 1] * 24, [1] * 63 + [3], [2] * 62])
def test_many_groups(sizes):
    """Starts that one wave holds, and more of them."""
    B = sum(sizes)
    shared = [64 + 64 * (i % 3) + (i % 5) for i in range(len(sizes))]
    ctx = np.concatenate([[s + i + (7 * i) % 90 for i in range(n)] for n, s in zip(sizes, shared)]).tolist()
    x = batch(4, 2, 64, 16, ctx, [1] * B, starts(sizes), shared)
    decode(x)
    right(x)


@pytest.mark.parametrize("hq,hkv,d,L", [(16, 16, 128, 2), (64, 8, 128, 3)])
def test_a_batch_past_the_last_level_cache(hq, hkv, d, L):
    """Rows of more than 256 MB pass the caches by: the same outputs, from a plan of its own."""
    ctx, n_groups = [8200, 8300, 8400, 8500, 8600, 8700, 8800, 8900], 4
    x = batch(hq, hkv, d, 64, ctx, [1] * 8, [0, 2, 4, 6, 8], [8200, 8300, 8500, 8700], L=L)
    assert x.pk.numel() * 4 > 300e6
    decode(x)
    right(x)


@pytest.mark.parametrize("hq,hkv,d,L,sizes,n,shared", [(32, 8, 64, 2, [6, 6], 5, 1200), (32, 8, 128, 2, [4, 4], 4, 3000), (32, 8, 128, 1, [16], 8, 2000),
                                                       (8, 2, 128, 1, [8], 9, 2000), (32, 8, 128, 2, [8, 8], 9, 900)])
def test_parts_joined_in_every_way(hq, hkv, d, L, sizes, n, shared):
    """Few parts of many rows, some of many, many of few; requests of a group that others do not fill."""
    B = sum(sizes)
    ctx = [shared + (13 * b) % 50 for b in range(B)]
    ctx[-1] = 70
    x = batch(hq, hkv, d, 64, ctx, [1 + (b % n) for b in range(B)], starts(sizes), [shared] * len(sizes), n=n, L=L)
    suffix(x)
    right(x)


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, several times over."""
    xs = [batch(32, 8, 128, 64, [1500, 1400, 1333, 1800], [1] * 4, [0, 4], [1333]),
          batch(32, 8, 128, 32, [900, 910, 905, 950, 64, 77], [3] * 6, [0, 4, 6], [900, 64], n=3, seed=1)]
    want = [decode(xs[0]).clone(), suffix(xs[1]).clone()]
    ws = [workspace(x, x.n, x.max_ctx) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    for it in range(5):
        for x in xs:
            x.out.fill_(SENTINEL)
        torch.cuda.synchronize()
        for _ in range(4):
            with torch.cuda.stream(streams[0]):
                decode(xs[0], ws=ws[0])
            with torch.cuda.stream(streams[1]):
                suffix(xs[1], ws=ws[1])
        torch.cuda.synchronize()
        assert all((x.out == w).all() for x, w in zip(xs, want)), it
    for x in xs:
        right(x)
