"""What the Python binding refuses of shared prefixes and norms with rotation: tensors that hold fewer entries, or others, than
the call reads or writes (no GPU: every refusal comes before the device is asked)."""
import pytest
import torch

import paper_2607_28069_amd as pic

MODEL = pic.Model.of(2, 4, 2, 64, "bf16", 1e4)
PAGES, GROUPS = pic.Pages.of(8, 16, 4), pic.Shared.of(2, 2, 20)


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


@pytest.mark.parametrize("name", ["page_table", "lens", "n_valid"])
@pytest.mark.parametrize("bad", ["short", "int64", "float32"])
@pytest.mark.parametrize("decode", [True, False])
def test_shared_refuses_lengths_and_tables(name, bad, decode):
    n = {"page_table": 3 * 4, "lens": 3, "n_valid": 3}
    a = {k: i32(v) for k, v in n.items()}
    a[name] = i32(n[name] - 1) if bad == "short" else a[name].to(getattr(torch, bad))
    head = (MODEL, PAGES, GROUPS, None, None, None, None, None, a["page_table"], 3, i32(3), i32(2), a["lens"])
    want = {"lens": "base_len" if decode else "ctx_len"}.get(name, name)
    if decode:
        if name != "n_valid":
            with pytest.raises(ValueError, match=want):
                pic.pic_page_shared_decode_attn(*head, 0, 10, None)
        return
    with pytest.raises(ValueError, match=want):
        pic.pic_page_shared_suffix_attn(*head, 10, 1, None, n_valid=a["n_valid"])


HOW = pic.QkNorm(None, None, 1e-6, 0, 0, 1.0)


def norm(**kw):
    b = torch.bfloat16
    a = dict(q=torch.zeros(2, 3, 5, 4, 64, dtype=b), k=torch.zeros(2, 3, 5, 2, 64, dtype=b), v=torch.zeros(2, 3, 5, 2, 64, dtype=b), batch=3, n=5,
             table=torch.zeros(11 * 64), mad=10, qo=torch.zeros(2, 3, 5, 4, 64, dtype=b), ko=torch.zeros(2, 3, 5, 2, 64, dtype=b),
             vo=torch.zeros(2, 3, 5, 2, 64, dtype=b), lens=i32(3), nv=i32(3), how=HOW, model=MODEL)
    a.update(kw)
    pic.pic_qk_norm_rope(a["model"], a["how"], a["q"], a["k"], a["v"], a["batch"], a["n"], a["table"], a["mad"], a["qo"], a["ko"], a["vo"],
                         base_len=a["lens"], max_base_len=5, n_valid=a["nv"])


@pytest.mark.parametrize("x", "qkv")
def test_norm_refuses_rows(x):
    heads = 4 if x == "q" else 2
    for at in (x, x + "o"):
        with pytest.raises(ValueError, match=f"{x}: at least {2 * 15 * heads * 64} elements"):     # one layer of two
            norm(**{at: torch.zeros(1, 3, 5, heads, 64, dtype=torch.bfloat16)})
        with pytest.raises(ValueError, match=f"{x}: at least .*bfloat16 expected"):
            norm(**{at: torch.zeros(2, 3, 5, heads, 64)})
        with pytest.raises(ValueError, match=f"{x}: at least .*float32 expected"):
            norm(model=pic.Model.of(2, 4, 2, 64, "f32", 1e4), **{y: None for y in "qkv" if y != x})


def test_norm_refuses_tables_lengths_and_weights():
    with pytest.raises(ValueError, match="base_len"):
        norm(lens=i32(2))
    with pytest.raises(ValueError, match="base_len"):
        norm(lens=i32(3).long())
    with pytest.raises(ValueError, match="n_valid"):
        norm(nv=i32(2))
    with pytest.raises(ValueError, match="table"):
        norm(table=torch.zeros(11 * 64 - 1))
    with pytest.raises(ValueError, match="table"):
        norm(model=pic.Model.of(2, 4, 2, 64, "bf16", 1e4, per_layer_tables=True))
    how = pic.QkNorm(None, None, 1e-6, 0, 0, 1.0)
    how.n_weights = 64
    with pytest.raises(ValueError, match="weights"):
        norm(how=how)


def test_token_rows_refuse_one_row_for_all():
    """A step of 0 from token to token stands for dense rows in the call, which would read past the one row there is."""
    one = torch.zeros(1, 4, 64)
    for t in (one.expand(5, 4, 64), one.expand(2, 5, 4, 64)):
        with pytest.raises(ValueError, match="one place"):
            pic._token_rows(t, 4, 64, "q", -1)
    assert pic._token_rows(one, 4, 64, "q", -1)[1] == 0
    assert pic._token_rows(torch.zeros(0, 4, 64), 4, 64, "q", -1)[0] is not None
