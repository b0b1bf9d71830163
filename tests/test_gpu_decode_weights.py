"""attn_decode's weights in fp16 where the steps of 4-bit values differ widely from token to token, and where one token has nearly
all of the weight: what is small beside the largest weight still counts in full."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    from paper_2506_05413_b200 import build, binding
    build.build()
    binding.load()
    return binding


@pytest.fixture(scope="module")
def au():
    import attention_util
    return attention_util


def _first_key_stands_out(au, gen, n, by):
    """Keys of which the first scores `by` above the rest (whose scores spread by about 1) for a query of ones in value 0."""
    k = au.pu.rows(gen, n, 256, 1.0)
    k[0] = 0
    k[0, 0::128] = by
    k[1:, 0::128] = 0
    return k


def _query(au, gen, heads):
    q = au.pu.rows(gen, 1, heads * 128, 1.0 / math.sqrt(128))
    q[:, 0::128] = 1
    return q


@pytest.mark.parametrize("n", [333, 5000])
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("by", [0.0, 2.0])
def test_rows_of_zeros_beside_small_values(sr, au, n, size, by):
    """A constant row has the step 1, many times the others'.  One in eight here, the first among them.
    Roundings of weights and result, each 2^-12 in the mean square at most, on values of either sign: 1e-3 is thrice that;
    values of 1e-4 are 2^-13 and the result's last place 2^-24, whose rounding
    adds 2^-25.8 a value in the mean square."""
    import torch
    gen = au.generator(n)
    v = au.pu.rows(gen, n, 256, size)
    v[::8] = 0
    cache, table, slots = au.paged(gen, [n], 2, 128, 16, 4, keys=lambda n: _first_key_stands_out(au, gen, n, by), values=lambda n: v)
    q = _query(au, gen, 8)
    y = au.decode(sr, q, cache, table, [n], scale=1.0)
    k, w = cache.get(slots[0])
    want, bound = au.attend(q, k, w, 128, 2, 1.0, None, *au.steps(cache, slots[0]))
    assert bool(((y.double() - want).abs() <= bound).all())
    floor = 2.0 ** -25.5 * math.sqrt(want.numel()) / float(want.norm())
    assert au.off(y, want) <= 1e-3 + floor, (au.off(y, want), floor)


@pytest.mark.parametrize("bits,down", [(4, 16), (16, 26)])
def test_many_small_weights_beside_a_large_one(sr, au, bits, down):
    """One token with nearly all of the weight and a value of zero; the others' weights are some 2^-down of it, and all that shows
    (with 4 bits the zeros' step of 1 takes six more places)."""
    import torch
    gen = au.generator(7)
    n = 150                                               # one warp's share
    by = down * math.log(2)
    v = au.pu.rows(gen, n, 256, 0.05) + 1
    v[0] = 0
    lengths = [n] * 700                                   # more segments than warps take in one round
    q = _query(au, gen, 8).repeat(len(lengths), 1)
    keys = _first_key_stands_out(au, gen, n, by)
    cache, table, slots = au.paged(gen, lengths, 2, 128, 16, bits, keys=lambda n: keys, values=lambda n: v, clip=1.0)
    y = au.decode(sr, q, cache, table, lengths, scale=1.0)
    k, w = cache.get(slots[0])
    want, bound = au.attend(q[:1], k, w, 128, 2, 1.0, None, *au.steps(cache, slots[0]))
    for b in (0, 1, 350, 699):
        assert bool(((y[b:b + 1].double() - want).abs() <= bound).all()), b
