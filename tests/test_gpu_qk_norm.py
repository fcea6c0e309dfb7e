"""Norms of queries and keys with the rotation, against the definition in 64 bits: types, heads, pairings, parts of a
head, orders, strides, padding; and keys so stored, moved on by the other calls."""
import numpy as np
import pytest
import torch

import paper_2607_28069_amd as pic

pytestmark = pytest.mark.gpu
DEV = "cuda"
SENTINEL = 7.5


def place(d, r, order):
    """Where element e of a head goes."""
    if order == "keep":
        return list(range(d))
    rest = [e for e in range(d) if not (e < r // 2 or d // 2 <= e < d // 2 + r // 2)]   # places left
    return list(range(r // 2)) + list(range(d // 2, d // 2 + r // 2)) + rest


def reference(x, w, eps, pos, freq, scale, r, pairing, order):
    """Heads x [..., N, heads, D] at positions pos [N], in 64 bits; w [D] or None."""
    y = x.double()
    if w is not None:
        y = y / ((y * y).mean(-1, keepdim=True) + eps).sqrt() * w.double()
    if freq is not None:
        ang = pos.double()[:, None] * torch.from_numpy(freq[: r // 2]).to(DEV)
        c, s = ang.cos()[:, None], ang.sin()[:, None]
        a, b = (y[..., : r // 2], y[..., r // 2: r]) if pairing == "half" else (y[..., 0:r:2], y[..., 1:r:2])
        a, b = scale * (a * c - b * s), scale * (a * s + b * c)
        t = torch.cat([a, b], -1) if pairing == "half" else torch.stack([a, b], -1).flatten(-2)
        y = torch.cat([t, y[..., r:]], -1)
    if pairing == "half":
        y = torch.empty_like(y).index_copy_(y.dim() - 1, torch.tensor(place(y.shape[-1], r, order), device=DEV), y)
    return y


def tolerance(want, pair, f32):
    """u = 2^-24: the sum of D squares off by (D + 2) u / 2 after the root, quotient, products and the turn's three
    roundings with the table's: at most 90 u of the element's pair; the store half a step."""
    u = 2.0 ** -24
    return 90 * u * pair + (0 if f32 else 2.0 ** -8) * want.abs() + 1e-30


def run(hq, hkv, d, dtype, B, n, r=None, pairing="half", order="keep", layers=1, base=None, n_valid=None, offset=0, fused=False,
        weights=True, rope=True, scale=1.0, parts="qkv", in_place=False, eps=1e-5, size=1.0, per_layer=False, seed=0):
    r = r or d
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    heads = dict(q=hq, k=hkv, v=hkv)
    model = pic.Model.of(layers, hq, hkv, d, dtype, 1e4, pairing, per_layer_tables=per_layer)
    total = sum(heads.values())
    if fused:
        wide = (rand(layers, B, n, total * d + 16) * size).to(dt)
        cut = wide[..., 8: 8 + total * d].unflatten(-1, (total, d))
        ins = dict(q=cut[..., :hq, :], k=cut[..., hq: hq + hkv, :], v=cut[..., hq + hkv:, :])
    else:
        ins = {x: (rand(layers, B, n, h, d) * size).to(dt) for x, h in heads.items()}
    ins = {x: t if x in parts else None for x, t in ins.items()}
    before = {x: None if t is None else t.clone() for x, t in ins.items()}
    outs = {x: (ins[x] if in_place else torch.full((layers, B, n, h, d), SENTINEL, dtype=dt, device=DEV)) if x in parts else None
            for x, h in heads.items()}
    w = {x: (1 + 0.3 * rand(layers, d)) if weights else None for x in "qk"}
    base_h = [0] * B if base is None else base
    first = [max(b, 0) + offset for b in base_h]
    mad = max(first) + n
    tables = layers if per_layer else 1
    freq = np.zeros((tables, d // 2))
    for t in range(tables):
        freq[t, : r // 2] = (1e4 + 5000 * t) ** (-2.0 * np.arange(r // 2) / r)
    table = None
    if rope:
        table = torch.empty(pic.pic_rope_table_bytes(model, mad) // 4, dtype=torch.float32, device=DEV)
        pic.pic_rope_table_init_freq(model, freq, mad, table)
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    pic.pic_qk_norm_rope(model, pic.QkNorm.of(w["q"], w["k"], eps, 0 if r == d else r, order, scale), ins["q"], ins["k"], ins["v"], B, n,
                         table, mad, outs["q"], outs["k"], outs["v"], base_len=i32(base), max_base_len=max(max(base_h), 0), offset=offset,
                         n_valid=i32(n_valid))
    torch.cuda.synchronize()
    for x in parts:
        got = outs[x]
        for b in range(B):
            m = n if n_valid is None else min(max(n_valid[b], 0), n)
            if base is not None and base[b] < 0:
                m = 0
            rest = got[:, b, m:]
            assert (rest == (before[x][:, b, m:] if in_place else SENTINEL)).all(), "rows of padding were written"
            if x == "v":
                assert (got[:, b, :m] == before[x][:, b, :m]).all()
                continue
            pos = torch.arange(first[b], first[b] + m, device=DEV)
            for l in range(layers):
                f = freq[l if per_layer else 0] if rope else None
                arg = (before[x][l, b, :m], None if w[x] is None else w[x][l], eps, pos, f, scale, r, pairing, order)
                want = reference(*arg)
                # the magnitude of each element's pair: both members' sizes without the turn's signs
                mag = reference(arg[0].double().abs(), None if w[x] is None else w[x][l].abs(), eps, torch.zeros_like(pos), f,
                                abs(scale), r, pairing, order)
                if pairing == "half":
                    at = torch.tensor(place(d, r, order), device=DEV)
                    back = mag[..., at]
                    back = torch.cat([(back[..., : r // 2] + back[..., r // 2: r]).repeat(*[1] * (back.dim() - 1), 2), back[..., r:]], -1)
                    mag = torch.empty_like(mag).index_copy_(mag.dim() - 1, at, back)
                else:
                    both = (mag[..., 0::2] + mag[..., 1::2]).repeat_interleave(2, -1)
                    mag = torch.cat([both[..., :r], mag[..., r:]], -1)
                err = (got[l, b, :m].double() - want).abs()
                assert (err <= tolerance(want, mag, dtype == "f32")).all(), (x, float((err / tolerance(want, mag, dtype == "f32")).max()))
    return outs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (32, 8, 128), (28, 4, 128), (5, 1, 64), (3, 3, 128), (1, 1, 128), (71, 1, 64)])
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_heads(dtype, hq, hkv, d, pairing):
    run(hq, hkv, d, dtype, 3, 7, pairing=pairing, base=[5, 0, 1000], layers=2)
    run(hq, hkv, d, dtype, 2, 1, pairing=pairing, base=[4097, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [16, 32, 48, 64, 80, 112, 128])
def test_part_of_the_head(dtype, d, r):
    if r > d:
        pytest.skip("the whole head and no more")
    for pairing, order in (("half", "keep"), ("half", "pairs"), ("interleaved", "keep"), ("interleaved", "pairs")):
        run(8, 2, d, dtype, 2, 5, r=r, pairing=pairing, order=order, base=[77, 2], scale=1.25)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slices_of_a_projection(dtype):
    run(8, 2, 128, dtype, 3, 9, base=[1, 2, 3], fused=True, layers=2)
    run(8, 2, 64, dtype, 4, 1, base=[1, 2, 3, 4], fused=True, pairing="interleaved")
    for parts in ("q", "k", "v", "qk", "qv", "kv"):
        run(8, 2, 64, dtype, 2, 5, base=[9, 0], fused=parts != "kv", parts=parts)


def test_padding_and_positions():
    run(8, 2, 128, "bf16", 5, 11, base=[0, -1, 30, -7, 5], n_valid=[11, 4, 0, 11, 3])
    run(8, 2, 128, "bf16", 3, 11, n_valid=[-4, 99, 7])              # without lengths: positions from offset
    run(8, 2, 128, "bf16", 3, 6, offset=1000)
    run(8, 2, 128, "bf16", 3, 6, base=[4, 0, 9], offset=17)
    run(8, 2, 128, "bf16", 1, 1)


def test_norm_only_rotation_only():
    run(8, 2, 128, "bf16", 2, 5, base=[50, 3], rope=False)
    run(8, 2, 128, "f32", 2, 5, base=[50, 3], weights=False)
    run(8, 2, 128, "bf16", 2, 5, base=[50, 3], weights=False, rope=False, order="pairs", r=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    for order in ("keep", "pairs"):
        run(32, 8, 128, dtype, 4, 33, base=[9, 8, 7, 6], in_place=True, order=order, r=64, n_valid=[33, 0, 5, 32])


def test_per_layer_tables_and_sizes():
    run(8, 2, 64, "bf16", 3, 5, base=[11, 700, 3], layers=3, per_layer=True)
    run(8, 2, 128, "f32", 2, 5, base=[11, 7], size=1e6)
    run(8, 2, 128, "f32", 2, 5, base=[11, 7], size=1e-4)            # eps counts
    run(8, 2, 128, "bf16", 1, 4000, layers=2)
    run(8, 2, 64, "bf16", 700, 1, base=list(range(700)))
    run(32, 8, 128, "bf16", 40, 131, base=list(range(40)), n_valid=[131 - 3 * i for i in range(40)], fused=True)


def test_rows_of_zeros_and_not_finite():
    q = torch.zeros((1, 1, 4, 2, 64), dtype=torch.bfloat16, device=DEV)
    q[0, 0, 1, 0, 3] = float("inf")
    q[0, 0, 2, 1, 3] = float("nan")
    out = torch.empty_like(q)
    m = pic.Model.of(1, 2, 1, 64, "bf16", 1e4)
    one = torch.ones((1, 64), device=DEV)
    pic.pic_qk_norm_rope(m, pic.QkNorm.of(one, None, 1e-6), q, None, None, 1, 4, None, 0, out, None, None)
    assert (out[0, 0, [0, 3]] == 0).all() and out[0, 0, 1, 0, 3].isnan() and (out[0, 0, 1, 1] == 0).all()
    assert out[0, 0, 2, 1].isnan().all() and (out[0, 0, 2, 0] == 0).all()


def test_keys_in_the_order_of_pairs_move_on():
    """A third of each head turned in halves: laid out by pairs, pic_rerotate_keys moves such keys from position to
    position, and scores are those of the order kept."""
    d, r, n = 128, 32, 12
    m = pic.Model.of(1, 4, 4, d, "f32", 1e4)
    freq = np.zeros(d // 2)
    freq[: r // 2] = 1e4 ** (-2.0 * np.arange(r // 2) / r)
    mad = 5000
    table = torch.empty(pic.pic_rope_table_bytes(m, mad) // 4, dtype=torch.float32, device=DEV)
    pic.pic_rope_table_init_freq(m, freq, mad, table)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k = (torch.randn((1, 1, n, 4, d), generator=g, device=DEV) for _ in "qk")
    w = torch.randn((2, d), generator=g, device=DEV)
    got = {}
    for order in ("keep", "pairs"):
        for at in (0, 3000):
            qo, ko = torch.empty_like(q), torch.empty_like(k)
            pic.pic_qk_norm_rope(m, pic.QkNorm.of(w[:1].contiguous(), w[1:].contiguous(), 1e-6, r, order), q, k, None, 1, n, table, mad,
                                 qo, ko, None, offset=at)
            got[order, at] = qo, ko
    moved = torch.empty_like(k)
    delta = torch.full((n,), 3000, dtype=torch.int32, device=DEV)
    pic.pic_rerotate_keys(m, got["pairs", 0][1], moved, n, 4, delta, table, mad)
    # (two turns of 3 roundings and a table value each, of elements of some 10 at most)
    assert (moved - got["pairs", 3000][1]).abs().max() <= 16 * 10 * 2.0 ** -24
    scores = {o: got[o, 3000][0].double() @ got[o, 0][1].double().transpose(-1, -2) for o in ("keep", "pairs")}
    assert (scores["keep"] == scores["pairs"]).all() or (scores["keep"] - scores["pairs"]).abs().max() < 1e-11


def test_graph():
    m = pic.Model.of(1, 8, 2, 128, "bf16", 1e4)
    table = torch.empty(pic.pic_rope_table_bytes(m, 100) // 4, dtype=torch.float32, device=DEV)
    pic.pic_rope_table_init(m, 100, table)
    q, k = torch.randn((1, 3, 2, 8, 128), device=DEV).bfloat16(), torch.randn((1, 3, 2, 2, 128), device=DEV).bfloat16()
    qo, ko, lens = torch.empty_like(q), torch.empty_like(k), torch.tensor([3, 4, 5], dtype=torch.int32, device=DEV)
    how = pic.QkNorm.of(torch.ones((1, 128), device=DEV), None)
    call = lambda: pic.pic_qk_norm_rope(m, how, q, k, None, 3, 2, table, 100, qo, ko, None, base_len=lens, max_base_len=90)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for it in range(3):
        lens += 1
        call()
        want = qo.clone(), ko.clone()
        qo.zero_(), ko.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert (qo == want[0]).all() and (ko == want[1]).all()
