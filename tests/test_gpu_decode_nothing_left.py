"""attn_decode where every token of a sequence is left out (its pages lie outside the cache): such a sequence has no token, so
its output is 0, wherever its pieces meet: within a warp, within a CTA, across CTAs."""
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


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("lengths,gone", [
    ([5], [0]), ([9, 7, 30], [1]),                      # a warp has the whole sequence
    ([250], [0]), ([250, 3, 200], [0, 2]),              # pieces of one CTA
    ([20000], [0]), ([20000, 40, 9000, 1], [0, 1]),     # pieces of many CTAs
])
def test_all_pages_out_of_range_give_zero(sr, au, lengths, gone, bits):
    import torch
    gen = au.generator(len(lengths))
    cache, table, slots = au.paged(gen, lengths, 2, 128, 16, bits)
    q = au.pu.rows(gen, len(lengths), 8 * 128)
    sr.device_status()
    for b in gone:
        table[b] = torch.where(torch.arange(table.shape[1], device=au.DEV) % 2 == 0, -1, cache.k.shape[0]).int()
    y = au.decode(sr, q, cache, table, lengths)
    assert sr.device_status() == 34
    for b in gone:
        assert bool((y[b] == 0).all()), b
    kept = [b for b in range(len(lengths)) if b not in gone]
    if kept:
        au.check(y[kept], q[kept], cache, [slots[b] for b in kept])


@pytest.mark.parametrize("bits", [4, 16])
def test_a_cache_without_pages_gives_zero(sr, au, bits):
    import torch
    cache = au.pu.Cache(0, 16, 2, 128, bits)
    q = au.pu.rows(au.generator(1), 2, 4 * 128)
    sr.device_status()
    y = au.decode(sr, q, cache, torch.zeros(2, 400, dtype=torch.int32, device=au.DEV), [6400, 3])
    assert sr.device_status() == 34 and bool((y == 0).all())


@pytest.mark.parametrize("bits", [4, 16])
def test_pieces_without_tokens_beside_pieces_with_some(sr, au, bits):
    """Only the last, only the first, and only a middle page of a long sequence is there."""
    import torch
    gen = au.generator(3)
    n = 12000
    cache, table, slots = au.paged(gen, [n, n, n], 2, 128, 16, bits)
    q = au.pu.rows(gen, 3, 8 * 128)
    sr.device_status()
    left = [n // 16 - 1, 0, 333]
    for b, at in enumerate(left):
        keep = table[b, at].clone()
        table[b] = -1
        table[b, at] = keep
    y = au.decode(sr, q, cache, table, [n, n, n])
    assert sr.device_status() == 34
    au.check(y, q, cache, [slots[b][16 * at:16 * at + 16] for b, at in enumerate(left)])


def test_scores_of_minus_infinity_are_not_missing_tokens(sr, au):
    """Tokens that are there, all with a score of minus infinity: the softmax has no value, and the output says so."""
    import torch
    gen = au.generator(4)
    cache, table, slots = au.paged(gen, [40], 2, 128, 16, 16)
    q = torch.ones(1, 4 * 128, dtype=torch.float16, device=au.DEV)
    cache.k[..., 0] = -float("inf")
    y = au.decode(sr, q, cache, table, [40])
    assert sr.device_status() == 0 and bool(torch.isnan(y).all())
