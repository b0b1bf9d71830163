"""attn_decode's division of long and of many sequences over warps and CTAs: every tile of keys counts once, and outputs of long
sequences are near the plain form in the 2-norm, where a lost or doubled tile would show."""
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


@pytest.mark.parametrize("bits,D,H,kv", [(16, 128, 8, 2), (16, 64, 3, 3), (4, 128, 8, 2), (4, 128, 24, 2)])
@pytest.mark.parametrize("lengths", [[20000], [9001, 3, 777], [131, 4000, 1, 2049, 0, 65], list(range(40, 340, 4))])
@pytest.mark.parametrize("place", [0, 11, 31])
def test_every_tile_counts_once(sr, au, lengths, bits, D, H, kv, place):
    """With a scale of 0 all weights are equal and a value's output is the mean of its column.  One key of each tile (the one at
    `place`, or the tile's last) holds a power of two in a column of its own, eight tiles to a column: the column's sum tells which
    of them were counted.  Weights, values and sums are exact with fp16; a 4-bit value is rounded once in its step and once in its
    weight, so a sum of at most 255 is off by at most 255 * 2^-10, and the result's rounding adds 255 * 2^-11: below a half."""
    import torch
    gen = au.generator(place)
    tile = 32 if bits == 4 else 16
    zeros = lambda n: torch.zeros(n, kv * D, device=au.DEV)  # noqa: E731
    cache, table, slots = au.paged(gen, lengths, kv, D, 16, bits, values=zeros, clip=1.0)
    q = au.pu.rows(gen, len(lengths), H * D)
    most = max(-(-n // tile) for n in lengths)
    for first in range(0, most, 8 * D):                   # tiles first .. first + 8 D - 1 are told apart
        sums = torch.zeros(len(lengths), kv, D, dtype=torch.float64, device=au.DEV)
        for b, n in enumerate(lengths):
            if n == 0:
                continue
            t = torch.arange(min(first, -(-n // tile)), min(first + 8 * D, -(-n // tile)), device=au.DEV)
            v = torch.zeros(n, kv, D, device=au.DEV)
            for h in range(kv):
                column, power = (t + 17 * h) % D, 2.0 ** ((t - first) // D)
                v[(t * tile + place).clamp_max(n - 1).minimum(t * tile + tile - 1), h, column] = power
                sums[b, h].index_add_(0, column, power.double())
            k, _ = cache.get(slots[b])
            cache.put(slots[b], k, v.reshape(n, kv * D), 1.0)
        y = au.decode(sr, q, cache, table, lengths, scale=0.0).double().reshape(len(lengths), kv, H // kv, D)
        count = torch.tensor(lengths, device=au.DEV).double()[:, None, None, None]
        got = y * count
        assert bool(((got - sums[:, :, None]).abs() < 0.5).all()), float((got - sums[:, :, None]).abs().max())
        assert sr.device_status() == 0


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("lengths,H,kv,D", [([9001], 8, 2, 128), ([20000, 6000], 8, 2, 128), ([131072], 4, 1, 128), ([40000], 24, 2, 64),
                                            ([700 + 11 * i for i in range(40)], 8, 2, 128)])
def test_long_sequences_in_the_2_norm(sr, au, lengths, H, kv, D, bits):
    """Roundings of the result and of each weight, 2^-12 in the mean square at most, on values of either sign: 1e-3 is thrice their
    sum.  A tile of 32 keys among 131072 is 2^-6 of the norm."""
    gen = au.generator(lengths[0])
    cache, table, slots = au.paged(gen, lengths, kv, D, 16, bits)
    q = au.pu.rows(gen, len(lengths), H * D)
    y = au.decode(sr, q, cache, table, lengths)
    assert sr.device_status() == 0
    au.check(y, q, cache, slots, close=1e-3)
