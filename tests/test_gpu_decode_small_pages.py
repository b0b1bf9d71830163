"""attn_decode over 4-bit and fp16 caches with pages of 1, 2 and 4 tokens: a tile's copies are then more than a warp has lanes, and
with pages of 1 the steps and zero points come by plain loads."""
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
@pytest.mark.parametrize("page", [1, 2, 4])
@pytest.mark.parametrize("H,kv,D", [(8, 2, 128), (4, 2, 64), (24, 2, 128), (20, 2, 64)])
@pytest.mark.parametrize("lengths", [[1], [0, 1, 2, 3, 31, 32, 33, 64, 65, 97], [4001, 5, 600]])
def test_small_pages(sr, au, lengths, H, kv, D, page, bits):
    import torch
    gen = au.generator(page + len(lengths))
    cache, table, slots = au.paged(gen, lengths, kv, D, page, bits, fill=float("nan"))
    q = au.pu.rows(gen, len(lengths), H * D)
    for _ in range(3):
        y = au.decode(sr, q, cache, table, lengths)
        assert sr.device_status() == 0
        au.check(y, q, cache, slots)
        again = au.decode(sr, q, cache, table, lengths)
        assert torch.equal(y, again)


@pytest.mark.parametrize("page", [1, 2])
def test_small_pages_out_of_range_are_left_out(sr, au, page):
    import torch
    gen = au.generator(page)
    n = 300
    cache, table, slots = au.paged(gen, [n], 2, 128, page, 4, fill=float("nan"))
    gone = torch.arange(table.shape[1], device=au.DEV) % 3 == 1
    table[0, gone] = -1
    q = au.pu.rows(gen, 1, 8 * 128)
    sr.device_status()
    y = au.decode(sr, q, cache, table, [n])
    assert sr.device_status() == 34
    left = slots[0][~gone[torch.arange(n, device=au.DEV) // page]]
    au.check(y, q, cache, [left])
