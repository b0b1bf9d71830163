"""Rows so long that their scales' offsets pass 32 bits: read back, and written by the gated block."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    from paper_2506_05413_b200 import build, binding
    build.build()
    binding.load()
    return binding


@pytest.fixture(scope="module")
def mu():
    import mx_util
    return mx_util


@pytest.mark.parametrize("k", [2 ** 29 + 2 ** 20, 2 ** 30])
def test_codes_read_back(sr, mu, k):
    """A row in groups of 16: groups past the 2^25th have their scales beyond 4 GB."""
    import torch
    g = mu.gen(1)
    q = torch.empty(1, k // 2, dtype=torch.uint8, device=mu.DEV).random_(0, 256, generator=g)
    s = torch.empty(128 * (k // 16), dtype=torch.uint8, device=mu.DEV).random_(30, 100, generator=g)
    y = torch.empty(1, k, dtype=torch.float16, device=mu.DEV)
    sr.mx_dequant(q, s, None, y, group=16)
    grid = torch.tensor(mu.GRID + [-x for x in mu.GRID], device=mu.DEV)
    for first in (0, 2 ** 28, 2 ** 29 - 2 ** 18, 2 ** 29, k - 2 ** 19):
        n = 2 ** 19
        groups = torch.arange(first // 16, (first + n) // 16, device=mu.DEV)
        byte = s[groups // 4 * 512 + groups % 4].int()
        unit = (1 + (byte & 7) / 8) * torch.exp2((byte >> 3).float() - 7)
        part = q[0, first // 2:(first + n) // 2]
        code = grid[torch.stack([part & 15, part >> 4], -1).reshape(-1).int()]
        assert torch.equal(y[0, first:first + n], (code * unit.repeat_interleave(16)).half()), first


def test_codes_of_the_gated_block(sr, mu):
    """More than 2^29 features in groups of 16: the last ones' scales are where their call alone puts them."""
    import torch
    f, k, last = 2 ** 29 + 256, 128, 256
    g = mu.gen(2)
    few, x = mu.random_coded(g, last, k, 16), mu.random_coded(g, 1, k, 16)
    q, s = torch.zeros(f, k // 2, dtype=torch.uint8, device=mu.DEV), torch.zeros(f * (k // 16), dtype=torch.uint8, device=mu.DEV)
    q[-last:], s[-last * (k // 16):] = few.q, few.s
    step = torch.ones(1, device=mu.DEV)
    codes, scales = torch.empty(1, f // 2, dtype=torch.uint8, device=mu.DEV), torch.zeros(128 * (f // 16), dtype=torch.uint8, device=mu.DEV)
    alone = mu.Coded(1, last, 16)
    kw = dict(group=16, x_step=x.step, h_step=step)
    sr.mx_glu(x.q, x.s, few.q, few.s, few.q, few.s, q_out=alone.q, scale_out=alone.s, **kw)
    sr.mx_glu(x.q, x.s, q, s, q, s, q_out=codes, scale_out=scales, **kw)
    want = alone.s[mu.place(1, last, 16)]
    groups = torch.arange((f - last) // 16, f // 16, device=mu.DEV)
    assert bool((want != 0).any()) and torch.equal(scales[groups // 4 * 512 + groups % 4], want[0])
    assert torch.equal(codes[:, -last // 2:], alone.q)
    groups = torch.arange(last // 16, device=mu.DEV)
    assert bool((scales[groups // 4 * 512 + groups % 4] == 0).all()) and bool((codes[:, :last // 2] & 0x77 == 0).all()) and sr.device_status() == 0
