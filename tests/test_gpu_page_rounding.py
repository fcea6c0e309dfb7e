"""How often the bf16 calls over pages round, by the way that their launch takes (page_cases.py): the output alone in decode
and in the kernel of few rows, the probabilities besides in the prefill, with or without shares; and the bits of
the contiguous call where both calls do the same."""
import math

import pytest
import torch

import paper_2607_28069_amd as pic
from page_cases import F32_SHARES, FEW, HALF_SHARES, WHOLE
from page_path import DEV, check, contiguous, decode, reference, rope_table, setup, suffix, turn

pytestmark = pytest.mark.gpu


def batch(case):
    hq, hkv, d, b, n, ctx = case
    return setup(hq, hkv, d, "bf16", 64, [ctx - 7 * i % 40 for i in range(b)], [n] * b)


def rounded(x, times):
    """The outputs' error in the 2-norm is that of `times` roundings to bfloat16.  One is off by up to 2^-8 of the next lower
    power of two, evenly: 2^-8 / sqrt(3) of it in the root mean square, and relative to values whose mantissas m are
    spread by their logarithm that times sqrt(mean of m^-2) = sqrt(3 / (8 ln 2)).  Independent ones add in squares; a
    tenth more for the sample, and less than 2^-11 for all that is kept finer."""
    ref, _, _ = reference(x)
    rel = float((x.out.double() - ref).norm() / ref.norm())
    most = 1.1 * math.sqrt(times) * 2.0 ** -8 / math.sqrt(3) * math.sqrt(3 / (8 * math.log(2))) + 2.0 ** -13
    assert rel <= most, (rel, most)


@pytest.mark.parametrize("case", FEW)
@pytest.mark.parametrize("rope", [False, True])
def test_few_rows_round_the_output_alone(case, rope):
    x = batch(case)
    r = rope_table(x) if rope else None
    suffix(x, rope=r)
    if rope:
        turn(x, r)
    check(x, decoded=True, turned=rope)
    rounded(x, 1)


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (32, 8, 64), (40, 1, 128)])
@pytest.mark.parametrize("n_splits", [1, 5, 8])
@pytest.mark.parametrize("rope", [False, True])
def test_decode_rounds_the_output_alone(hq, hkv, d, n_splits, rope):
    x = batch((hq, hkv, d, 6, 1, 3000))
    r = rope_table(x) if rope else None
    decode(x, n_splits=n_splits, rope=r)
    if rope:
        turn(x, r)
    check(x, decoded=True, turned=rope)
    rounded(x, 1)


@pytest.mark.parametrize("case", WHOLE + F32_SHARES + HALF_SHARES)
def test_prefill_rounds_probabilities_and_output(case):
    x = batch(case)
    suffix(x)
    check(x)
    rounded(x, 2)


@pytest.mark.parametrize("case", [c for c in WHOLE + HALF_SHARES if c[2] == 64])
def test_prefill_turned_queries_round_no_more_at_head_dim_64(case):
    x = batch(case)
    r = rope_table(x)
    suffix(x, rope=r)
    turn(x, r)
    check(x, turned=True)
    rounded(x, 2)


@pytest.mark.parametrize("case,rope", [(c, False) for c in WHOLE + F32_SHARES] + [(c, True) for c in WHOLE + F32_SHARES if c[2] == 128])
def test_bits_of_the_contiguous_call(case, rope):
    """Unsplit, or in float32 shares, of equal contexts (ranges over pages are of a request's own keys); queries turned by
    the call at head_dim 128 (at 64 they keep two terms over pages)."""
    hq, hkv, d, b, n, ctx = case
    x = setup(hq, hkv, d, "bf16", 64, [ctx] * b, [n] * b)
    ck, cv, cap = contiguous(x)
    r = rope_table(x) if rope else None
    suffix(x, rope=r)
    ws = torch.empty(max(pic.pic_prefill_workspace_bytes(x.model, b, n, ctx), 16), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(x.out)
    args = (x.model, x.q, x.k, x.v, ck, cv, b, cap, x.len, ctx, n)
    if rope:
        pic.pic_suffix_prefill_attn_rope(*args, *r, out, ws)
    else:
        pic.pic_suffix_prefill_attn(*args, out, ws)
    assert torch.equal(out.view(torch.int16), x.out.view(torch.int16))
