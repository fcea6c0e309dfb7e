"""A workspace larger than the query names: the rest of it is left alone, the outputs are those of one of the size named."""
import pytest
import torch

import paper_2607_28069_amd as pic
from page_path import DEV, decode, setup, suffix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 8, 128, 1, [700]), (32, 8, 128, 4, [900, 800]), (4, 4, 128, 2, [714] * 3),
                                            (32, 8, 64, 5, [2900] * 4), (32, 8, 128, 4, [2600] * 16), (32, 8, 128, 40, [9001, 20]),
                                            (32, 8, 128, 128, [6000] * 8)])
def test_the_rest_of_a_workspace_is_left_alone(hq, hkv, d, n, ctx):
    x, y = (setup(hq, hkv, d, "bf16", 64, ctx, [n] * len(ctx)) for _ in range(2))
    named = pic.pic_prefill_workspace_bytes(x.model, x.B, n, x.max_ctx)
    ws = torch.full((named + (64 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
    suffix(x, ws=ws)
    assert (ws[named:] == 0xA5).all()
    suffix(y)
    assert torch.equal(x.out, y.out)
    if named == 0:
        y.out.fill_(0)
        suffix(y, ws=ws[8:])   # (misaligned: as if there were none)
        assert (ws == 0xA5).all() and torch.equal(x.out, y.out)
    x.out.fill_(0)
    if n == 1:
        decode(x, ws=ws)
        named = max(named, pic.pic_decode_workspace_bytes(x.model, x.B, x.max_ctx + 1, 0))
        assert (ws[named:] == 0xA5).all()
