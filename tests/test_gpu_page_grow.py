"""Page tables grown on the device, entry for entry what the host's call gives, its refusals among them; copies of listed
pages."""
import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def device_grow(pages, refs, table, lens, n, n_valid=None, offset=0, ws=None):
    """(refs, table, pairs, ready, result) after the call, as numpy arrays."""
    B = len(lens)
    r, t = dev(refs), dev(table)
    pairs, ready, result = dev(np.full((B, 2), 99)), dev(np.full(B, 99)), dev([9, 9, 9])
    need = pic.pic_page_grow_workspace_bytes(pages, B, n)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV) if ws is None else ws
    pic.pic_page_grow_async(pages, B, r, t, dev(lens), n, pairs, ready, result, ws, None if n_valid is None else dev(n_valid), offset)
    out = [x.cpu().numpy() for x in (r, t, pairs, ready, result)]
    assert (ws[need:] == 0xFF).all()
    return out


def compare(pages, refs, table, lens, n, n_valid=None, offset=0):
    """Against pic_page_grow on copies; returns the device's state and status."""
    lens = np.asarray(lens, np.int32)
    add = np.full(len(lens), n) if n_valid is None else np.clip(n_valid, 0, n)
    frm = np.where(lens < 0, 0, lens + offset)
    to = np.where(lens < 0, 0, frm + add)
    r, t = np.array(refs, np.int32), np.array(table, np.int32)
    status, pairs = 0, np.zeros((0, 2), np.int32)
    try:
        pairs = pic.pic_page_grow(pages, r, t, frm, to)
    except pic.PicError as e:
        status = e.status
    got = device_grow(pages, refs, table, lens, n, n_valid, offset)
    assert got[4][0] == status, (got[4], status)
    assert (got[0] == r).all() and (got[1] == t).all()
    want = np.full((len(lens), 2), -1, np.int32)
    want[: len(pairs)] = pairs
    assert (got[2] == want).all()
    assert (got[3] == (np.where(lens < 0, -1, lens) if status == 0 else -1)).all()
    if status == 0:
        taken = (t != np.asarray(table)).sum()
        assert got[4].tolist() == [0, len(pairs), taken]
    return r, t, status


def state(r, P, lens, cap, n_pages, share=()):
    """Tables over shuffled pages; share: (request, request it is a fork of, slots)."""
    pages = pic.Pages.of(n_pages, P, cap)
    refs, table, order, at = np.zeros(n_pages, np.int32), np.full((len(lens), cap), -1, np.int32), r.permutation(n_pages), 0
    forks = {d: (s, n) for d, s, n in share}
    for b, x in enumerate(lens):
        k = -(-max(x, 0) // P)
        if b in forks:
            s, n = forks[b]
            k = -(-n // P)
            table[b, :k] = table[s, :k]
        else:
            table[b, :k] = order[at: at + k]
            at += k
        refs[table[b, :k]] += 1
    return pages, refs, table


@pytest.mark.parametrize("P", [16, 64, 1024])
@pytest.mark.parametrize("n", [1, 7, 100])
def test_as_on_the_host(P, n):
    r = np.random.default_rng(P + n)
    for it in range(8):
        B = int(r.integers(1, 40))
        lens = r.integers(0, 300, B)
        share = []
        for d in range(1, B):
            if r.random() < 0.6:
                s = int(r.integers(0, d))
                if all(s != x[0] for x in share):
                    lens[d] = int(r.integers(0, lens[s] + 1))
                    share.append((d, s, int(lens[d])))
        cap = int(-(-(lens.max() + n) // P)) + 1
        pages, refs, table = state(r, P, lens, cap, B * (cap + 1) + 5, share)
        compare(pages, refs, table, lens, n)
        lens2 = np.where(r.random(B) < 0.3, -1, lens)
        nv = r.integers(-2, n + 3, B)
        rr, tt, _ = compare(pages, refs, table, lens2, n, nv)
        # on from there: pages already held past the length
        compare(pages, rr, tt, np.where(lens2 < 0, 0, lens2), n, offset=0)


def test_offset_is_a_step():
    r = np.random.default_rng(5)
    pages, refs, table = state(r, 16, [30, 32, 33], 8, 40)
    rr, tt, _ = compare(pages, refs, table, [20, 22, 23], 1, offset=10)
    compare(pages, rr, tt, [20, 22, -1], 1, offset=11)


def test_many_sharers():
    """The last of the sharers keeps the page, whole pages past the length give way without a copy."""
    r = np.random.default_rng(6)
    lens = [100] * 50
    pages, refs, table = state(r, 64, lens, 8, 300, [(d, 0, 100) for d in range(1, 50)])
    compare(pages, refs, table, lens, 300)
    compare(pages, refs, table, lens, 1)
    refs[table[0, 1]] += 3       # held by others too: all of these take their own
    compare(pages, refs, table, lens, 1)
    lens = [40] * 50             # entry 0 partly filled, entry 1 shared past the length
    compare(pages, refs, table, lens, 90)


def test_large_batches():
    """More requests, entries and pages than the workgroup has threads."""
    r = np.random.default_rng(7)
    B = 2500
    lens = r.integers(0, 64, B)
    pages, refs, table = state(r, 16, lens, 6, 4 * B + 7000)
    compare(pages, refs, table, lens, 30)
    pages, refs, table = state(r, 16, [5], 5000, 6000)
    compare(pages, refs, table, [5], 70001)


def test_large_forked_batches():
    """More requests than their places are kept of, more shared entries than threads, in several orders; and none at all."""
    r = np.random.default_rng(17)
    B = 4500
    lens = r.integers(0, 64, B)
    share = []
    for d in range(1, B, 2):
        lens[d] = int(r.integers(0, lens[d - 1] + 1))
        share.append((d, d - 1, int(lens[d])))
    pages, refs, table = state(r, 16, lens, 6, 3 * B, share)
    compare(pages, refs, table, lens, 30)
    rr, tt, _ = compare(pages, refs, table, lens, 1, r.integers(0, 2, B))
    compare(pages, rr, tt, lens, 20)
    lens = [100] * 1500
    pages, refs, table = state(r, 64, lens, 3, 2000, [(d, 0, 100) for d in range(1, 1500)])
    compare(pages, refs, table, lens, 50)
    few = refs.copy()
    few[np.flatnonzero(refs == 0)[1400:]] = 1                      # 1499 take one
    assert compare(pages, few, table, lens, 1)[2] == -4
    pairs, ready, result = dev(np.full((1, 2), 99)), dev([99]), dev([9, 9, 9])
    pages = pic.Pages.of(2000, 64, 3)
    ws = torch.empty(max(16, pic.pic_page_grow_workspace_bytes(pages, 0, 1)), dtype=torch.uint8, device=DEV)
    pic.pic_page_grow_async(pages, 0, None, None, None, 1, pairs[:0], ready[:0], result, ws)
    assert result.tolist() == [0, 0, 0] and pairs.tolist() == [[99, 99]] and ready.tolist() == [99]


def test_refusals_change_nothing():
    r = np.random.default_rng(8)
    lens = [30, 64, 10, 100]
    pages, refs, table = state(r, 16, lens, 7, 20)
    full = refs.copy()
    full[full == 0] = 5
    full[np.flatnonzero(refs == 0)[:3]] = 0
    assert compare(pages, full, table, lens, 40)[2] == -4          # 3 pages free
    assert compare(pages, refs, table, lens, 13)[2] == -4          # past the table
    assert compare(pages, refs, table, [30, 2**31 - 1 - 40, 10, -1], 40)[2] == -4
    bad = table.copy()
    bad[0, 1] = -1                                                 # the partly filled page is none
    assert compare(pages, refs, bad, lens, 1)[2] == -6
    for v in (20, -2, 2**31 - 1, -2**31):
        bad = table.copy()
        bad[3, 6] = v
        assert compare(pages, refs, bad, lens, 1)[2] == -6
    gone = refs.copy()
    gone[table[0, 1]] = 0
    assert compare(pages, gone, table, lens, 1)[2] == -6
    assert compare(pages, refs, table, [-1] * 4, 1)[2] == 0
    assert compare(pages, refs, table, lens, 0)[2] == 0
    assert compare(pic.Pages.of(0, 16, 0), [], np.zeros((2, 0)), [3, 4], 1)[2] == -4


def test_graph_of_steps():
    """One captured step replayed until pages run out: the same tables as the host's, then refused and nothing changed."""
    r = np.random.default_rng(9)
    lens = np.array([30, 47, 16, 1], np.int32)
    pages, refs, table = state(r, 16, lens, 12, 20)
    rd, td, ld = dev(refs), dev(table), dev(lens)
    pairs, ready, result = dev(np.zeros((4, 2))), dev(np.zeros(4)), dev(np.zeros(3))
    ws = torch.empty(pic.pic_page_grow_workspace_bytes(pages, 4, 1), dtype=torch.uint8, device=DEV)

    def step():
        pic.pic_page_grow_async(pages, 4, rd, td, ld, 1, pairs, ready, result, ws)
        ld.add_(1)

    keep = [x.clone() for x in (rd, td, ld)]
    step()
    for x, y in zip((rd, td, ld), keep):
        x.copy_(y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    failed = 0
    for it in range(120):
        try:
            pic.pic_page_grow(pages, refs, table, lens, lens + 1)
            status = 0
        except pic.PicError as e:
            status = e.status
        lens = lens + 1
        g.replay()
        torch.cuda.synchronize()
        assert result[0].item() == status
        assert (rd.cpu().numpy() == refs).all() and (td.cpu().numpy() == table).all()
        failed += status != 0
    assert 0 < failed < 120


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,d,L,hkv", [(16, 64, 1, 1), (64, 128, 3, 2), (1024, 64, 2, 1)])
def test_copy_listed(dtype, P, d, L, hkv):
    r = np.random.default_rng(P)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    for n, cap in ((0, 0), (0, 5), (1, 1), (37, 64), (70, 200)):
        n_pages = 2 * n + 3
        pages = pic.Pages.of(n_pages, P, 0)
        k, v = (torch.randn((L, hkv, n_pages * P, d), device=DEV).to(dt) for _ in "kv")
        order = r.permutation(n_pages)[: 2 * n].reshape(-1, 2)
        listed = r.choice(np.array([-1, -7, n_pages, 2**31 - 1, -2**31]), (cap, 2)).astype(np.int64)
        if cap:
            listed[:, 0] = np.where(r.random(cap) < 0.5, listed[:, 0], 0)      # one of the two no page: skipped
        at = np.sort(r.choice(cap, n, replace=False)) if n else []
        listed[at] = order
        want = []
        for x in (k, v):
            y = x.clone().view(L, hkv, n_pages, P * d)
            y[:, :, order[:, 1]] = y[:, :, order[:, 0]].clone()
            want.append(y.view_as(x))
        pic.pic_page_copy_async(pic.Model.of(L, hkv, hkv, d, dtype, 1e4), pages, k, v, dev(listed) if cap else dev(np.zeros((1, 2))), cap)
        assert (k == want[0]).all() and (v == want[1]).all()
