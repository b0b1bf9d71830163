"""attn_prefill where one key has nearly all of a row's weight: the many small weights beside it still count in full."""
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,down", [(3000, 22), (131072, 26), (131072, 29)])
def test_many_small_weights_beside_a_large_one(sr, au, D, n, down):
    """The first key scores `down` powers of two above the others and its value is zero, so that all of the output comes from
    the others.  Their scores spread by about 1, so their roundings are of either sign: a weight of 2^-29 beside the largest
    keeps two bits and more, its error is below 2^-3 of it in the mean, and below 1e-3 in a sum of 131072; the rest of 2e-3 is
    for the result's rounding and for sums in fp32 over 8192 products of 16 keys, 8192 * 2^-24 at most."""
    import torch
    gen = au.generator(n)
    H, kv, m = 4, 2, 3
    k = au.pu.rows(gen, n, kv * D)
    k[0] = 0
    k[0, 0::D] = down * math.log(2)
    k[1:, 0::D] = 0
    v = (au.pu.rows(gen, n, kv * D, 0.05).float() + 64).half()
    v[0] = 0
    q = au.pu.rows(gen, m, H * D, 1 / math.sqrt(D))
    q[:, 0::D] = 1
    ends = lambda x: torch.tensor([0, x], dtype=torch.int32, device=au.DEV)  # noqa: E731
    y = torch.full((m, H * D), float("nan"), dtype=torch.float16, device=au.DEV)
    sr.attn_prefill(q, k, v, ends(m), ends(n), y, head_dim=D, causal=False, scale=1.0)
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    want, _ = au.attend(q, k, v, D, kv, 1.0)
    assert au.off(y, want) <= 2e-3, au.off(y, want)


def test_weights_grow_past_what_the_type_holds_from_block_to_block(sr, au):
    """Scores that rise steadily, by 3, 11, 15.9 and 40 powers of two a block: the reference follows them."""
    import torch
    gen = au.generator(5)
    H, kv, D, m = 4, 2, 128, 70
    for rise in (3.0, 11.0, 15.9, 40.0):
        n = 64 * 12 + m
        k = au.pu.rows(gen, n, kv * D, 0.1)
        k[:, 0::D] = (torch.arange(n, device=au.DEV) // 64 * rise * math.log(2))[:, None].half()
        v = au.pu.rows(gen, n, kv * D)
        q = au.pu.rows(gen, m, H * D, 0.1)
        q[:, 0::D] = 1
        cq = torch.tensor([0, m], dtype=torch.int32, device=au.DEV)
        ck = torch.tensor([0, n], dtype=torch.int32, device=au.DEV)
        y = torch.empty(m, H * D, dtype=torch.float16, device=au.DEV)
        sr.attn_prefill(q, k, v, cq, ck, y, head_dim=D, causal=True, scale=1.0)
        seen = torch.ones(m, n, dtype=torch.bool, device=au.DEV).tril(n - m)
        want, bound = au.attend(q, k, v, D, kv, 1.0, seen)
        assert bool(((y.double() - want).abs() <= bound).all()), rise
