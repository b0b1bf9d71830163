"""The gated block's codes in groups of 16 under steps of the caller's: of no particular form, and far too small for the values."""
import pytest

pytestmark = pytest.mark.gpu

BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]


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


def _codes(sr, mu, m, h, step):
    """h [F] fp32 in codes, for each of m tokens: a gate of 32 is its own SiLU in fp32, and products by powers of two are exact."""
    import torch
    f = h.numel()
    x, w, c = mu.Coded(m, 128, 16), mu.Coded(f, 128, 16), mu.Coded(m, f, 16)
    for t in (x, w):        # value 0 of every row is 1, the others 0: sums are 1
        t.q.zero_()
        t.q[:, 0] = 2
        t.s[mu.place(t.m, 128, 16)] = 56
    c.step = step.expand(m).contiguous()
    sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s, group=16, gate_step=torch.full((f,), 32.0, device=mu.DEV), up_step=h / 32, q_out=c.q, scale_out=c.s, h_step=c.step)
    return c


def _scales(mu):
    import torch
    return torch.tensor([(1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) if b >> 3 else (b & 7) / 512 for b in range(1, 127)], device=mu.DEV)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_borders_under_steps_of_no_particular_form(sr, mu, m):
    """A group for every scale and each distance of -2 to 2 units in the last place from the borders: the scale is that of the fp32 quotient
    of the group's largest value and 6 steps, codes are those of the fp32 quotients of its values and scale * step."""
    import torch
    g = mu.gen(m)
    for step in torch.cat([torch.rand(12, generator=g, device=mu.DEV) + 0.5, torch.tensor([1.0, 1.5, 4.0 / 3, 0.1, 1e-4, 3e-28, 7e20], device=mu.DEV)]):
        unit = (_scales(mu) * step)[:, None, None]                                     # rounded to fp32
        border = torch.tensor(BORDERS, device=mu.DEV) * unit                           # [126, 1, 7], rounded
        ulps = torch.arange(-2, 3, device=mu.DEV, dtype=torch.int32)[:, None]
        near = (border.view(torch.int32) + ulps).view(torch.float32)                   # [126, 5, 7]
        top = (6 * unit).expand(126, 5, 1)
        zero = torch.zeros(126, 5, 1, device=mu.DEV)
        h = torch.cat([torch.cat([top, near, -near, zero], 2).reshape(-1), torch.zeros(10 * 16, device=mu.DEV)])       # 640 groups
        c = _codes(sr, mu, m, h, step)
        v = h.reshape(640, 16)
        t = v.abs().amax(1) / (6 * step)
        byte = c.s[mu.place(m, h.numel(), 16)]
        assert bool((byte == t.to(torch.float8_e4m3fn).view(torch.uint8)).all())
        d = t.to(torch.float8_e4m3fn).float() * step
        q = torch.where(d[:, None] == 0, torch.zeros_like(v), v / d[:, None]).double()
        assert bool((c.codes().reshape(m, 640, 16) == mu.nearest(q, torch.ones_like(q))).all()), float(step)
    assert sr.device_status() == 0


@pytest.mark.parametrize("m", [1, 40, 300])
@pytest.mark.parametrize("step", [2.0 ** -100, 1e-30, 3e-20])
def test_values_far_beyond_the_steps_saturate_with_their_sign(sr, mu, m, step):
    """Quotients that no fp32 number holds among ordinary ones: a value beyond 2688 steps is 6 scales of its sign, the others are coded as ever."""
    import torch
    s = torch.tensor([step], device=mu.DEV)
    d = 448 * s
    far = torch.tensor([1e12, -1e12, 3e38, -3e38, 1e25, -1e25], device=mu.DEV)
    ordinary = torch.tensor([0.0, 0.6, -1.4, 2.2, -3.2, 4.4, -5.6, 0.1, 6.0, -6.0], device=mu.DEV) * d
    h = torch.cat([far, ordinary, far.flip(0), ordinary, ordinary, far * 1e-3]).repeat(8)
    h = h[:h.numel() // 128 * 128]
    c = _codes(sr, mu, m, h, s)
    v = h.double().reshape(-1, 16)
    scale = torch.full((v.shape[0], 1), 448.0, dtype=torch.float64, device=mu.DEV) * s.double()
    want = mu.nearest(v / scale, torch.ones_like(v)).reshape(-1)
    over = v.abs().amax(1) >= 2688 * s.double()
    assert bool(over.all()) and bool((c.s[mu.place(m, h.numel(), 16)] == 126).all())
    assert bool((c.codes() == want).all()) and sr.device_status() == 0
