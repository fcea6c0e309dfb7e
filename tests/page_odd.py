"""Inputs of the bf16 calls over pages that are not finite: where they go, and which outputs have to follow."""
import math

import torch

from page_path import DEV, rope_table, rows, setup

INF, NAN = math.inf, math.nan


def put_value(x, b, slot, g, c, value):
    """Head dim c of slot `slot`'s value in kv head g, cached or new."""
    if slot < x.ctx[b]:
        x.pv[0, g, rows(x, b, slot, slot + 1), c] = value
    else:
        x.v[0, b, slot - x.ctx[b], g, c] = value


def put_key(x, b, slot, g, value):
    if slot < x.ctx[b]:
        x.pk[0, g, rows(x, b, slot, slot + 1)] = value
    else:
        x.k[0, b, slot - x.ctx[b], g] = value


def same_but(x, want, slack=None):
    """x's outputs are `want`, bit for bit, or finite ones to within `slack` of each other."""
    nan, fin = torch.isnan(want), torch.isfinite(want)
    assert torch.equal(torch.isnan(x.out), nan)
    if slack is None:
        fin = torch.zeros_like(fin)
    bits = torch.int32 if x.out.dtype == torch.float32 else torch.int16
    assert torch.equal(x.out[~nan & ~fin].view(bits), want[~nan & ~fin].view(bits))
    err = (x.out[fin].double() - want[fin].double()).abs()
    assert (err <= (slack(want.double())[fin] if slack else 0)).all()


def rounded_anew(x):
    """Two results of the same scores whose running maxima moved at other tiles: each rounds probabilities by 2^-8 at
    most, in numerator and denominator, and a share by 2^-11, of values no larger than those of the batch; and the
    output by 2^-8."""
    most = float(max(v[v.isfinite()].abs().max() for v in x.V).double())
    return lambda want: 2 * ((2 * 2.0 ** -8 + 2.0 ** -11) * most + 2.0 ** -8 * want.abs())


def rescaled(x):
    """Shares in half precision, scaled by the row's largest finite value, here another one: what is below 2^-14 of that
    is off by 2^-25 of it in either scale, and the output then rounds to a neighbour, 2^-7 away."""
    most = float(max(v[v.isfinite()].abs().max() for v in x.V).double())
    return lambda want: 2.0 ** -7 * want.abs() + 2 * 2.0 ** -25 * most


def value_case(call, args, bad, queries=1.0, rope=False, slack=None):
    """bad: (request, slot, kv head, head dim, value).  The outputs of the tokens that see a value that is not finite
    are the sum of those they see, in its head dim; all others are as if it were finite."""
    x, y = (setup(*args) for _ in range(2))
    for z in (x, y):
        z.q *= queries
    for item in bad:
        put_value(x, *item)
    r = rope_table(x) if rope else None
    call(x, rope=r)
    call(y, rope=r)
    assert torch.isfinite(y.out).all()
    want, rep = y.out.clone(), x.hq // x.hkv
    odd = torch.zeros_like(want)
    for b, slot, g, c, v in bad:
        odd[0, b, max(slot - x.ctx[b], 0): x.new[b], g * rep: (g + 1) * rep, c] += v
    want[odd != 0] = odd[odd != 0]
    same_but(x, want, slack and slack(y))


def key_case(call, args, bad, rope=False):
    x, y = (setup(*args) for _ in range(2))
    rep = x.hq // x.hkv
    for item in bad:
        put_key(x, *item, NAN)
    r = rope_table(x) if rope else None
    call(x, rope=r)
    call(y, rope=r)
    assert torch.isfinite(y.out).all()
    want = y.out.clone()
    for b, slot, g in bad:
        want[0, b, max(slot - x.ctx[b], 0): x.new[b], g * rep: (g + 1) * rep] = NAN
    same_but(x, want, rounded_anew(y))
