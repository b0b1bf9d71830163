"""attn_decode at the longest length that the call takes: just below 2^31 tokens, where a count of keys rounded up to whole tiles
no longer fits 32 bits.  The table names the same few pages over and over, so the cache itself is small."""
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


@pytest.mark.parametrize("short", [0, 1, 15, 17])
def test_almost_2_to_the_31_tokens(sr, au, short):
    """Every page counts equally often, but for the last ones, so the output is that over the pages once.  Sums in fp32 over
    28339 tiles of a warp, two products each, may be off by 56678 * 2^-24 = 0.34 % of the values' weighted size, numerator and
    denominator alike: 1 % with the roundings of weights and result, 2^-11 each, beside it."""
    import torch
    gen = au.generator(31)
    page, pages, H, D = 16, 8, 2, 128
    longest = (1 << 31) - page
    cache = au.pu.Cache(pages, page, 1, D, 4)
    slots = torch.arange(pages * page, device=au.DEV)
    cache.put(slots, au.pu.rows(gen, len(slots), D), au.pu.rows(gen, len(slots), D) + 0.5)
    table = (torch.arange(longest // page, device=au.DEV, dtype=torch.int32) % pages)[None]
    q = au.pu.rows(gen, 1, H * D)
    y = au.decode(sr, q, cache, table, [longest - short])
    assert sr.device_status() == 0
    k, v = cache.get(slots)
    want, _ = au.attend(q, k, v, D, 1, 1 / math.sqrt(D))
    size, _ = au.attend(q, k, v.abs(), D, 1, 1 / math.sqrt(D))
    assert bool(((y.double() - want).abs() <= 1e-2 * size).all()), float(((y.double() - want).abs() / size).max())
