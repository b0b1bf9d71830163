"""The gated block's values in front of codes, to the last bits of fp32: next to the borders between codes, which side they fall on."""
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


def _ones(mu, rows, group):
    """Rows of which value 0 alone is not 0 but 1: a product of two such rows is 1, so that a step is what the sum comes to."""
    c = mu.Coded(rows, 128, group)
    c.q.zero_()
    c.q[:, 0] = 2
    c.s[mu.place(rows, 128, group)] = 127 if group == 32 else 56
    c.step = None
    return c


def _codes(sr, mu, m, gate, up, group, step=1.0):
    """Codes of SiLU(gate) * up, both [F] fp32, for each of m tokens."""
    f = gate.numel()
    x, w, c = _ones(mu, m, group), _ones(mu, f, group), mu.Coded(m, f, group)
    import torch
    c.step = torch.full((m,), step, device=mu.DEV) if group == 16 else None
    sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s, group=group, gate_step=gate, up_step=up, q_out=c.q, scale_out=c.s, h_step=c.step)
    return c


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_values_next_to_a_border_are_coded_by_their_side(sr, mu, m, group):
    """fp32 allows h five units of 2^-24: two for the exponential's last place, one each for the sum, the quotient and the product.  Values
    seven units off a border, whatever the gate, belong to their side of it."""
    import torch
    g, f = mu.gen(m), 8192
    gate = (torch.rand(f, generator=g, device=mu.DEV) * 128 - 88.5).float()
    border = torch.tensor(BORDERS, dtype=torch.float64, device=mu.DEV)[torch.arange(f, device=mu.DEV) % 7]
    above = torch.arange(f, device=mu.DEV) // 7 % 2 == 1
    sign = 1 - 2.0 * (torch.arange(f, device=mu.DEV) // 14 % 2)
    silu = gate.double() / (1 + torch.exp(-gate.double()))
    up = (sign * border * (1 + torch.where(above, 8.0, -8.0) * 2.0 ** -24) / silu).float()
    h = silu * up.double()
    off = (h.abs() / border - 1) * 2.0 ** 24
    assert bool(((off >= 6.9) == above).all()) and bool((off.abs() >= 6.9).all())
    gate[::16], up[::16] = 32.0, 6.0 / 32          # sets the scale: a gate of 32 is its own SiLU
    h = torch.where(torch.arange(f, device=mu.DEV) % 16 == 0, torch.full_like(h, 6.0), h)
    c = _codes(sr, mu, m, gate, up, group)
    assert bool((c.units() == 1).all())
    assert bool((c.codes() == mu.nearest(h, torch.ones_like(h))).all()) and sr.device_status() == 0


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m", [1, 300])
def test_gates_at_the_ends_of_the_range(sr, mu, m, group):
    """exp(-gate) next to the largest fp32 number, infinite, and 0; infinite and NaN gates; zeros."""
    import torch
    inf, nan = float("inf"), float("nan")
    groups = [([-88.0, -87.5, -88.5, -87.0], 2.0 ** 120, None), ([-89.5, -100.0, -3e38, -95.0], 2.0 ** 120, 0.0), ([90.0, 3e38, 1e30, 200.0], 2.0 ** -100, None),
              ([inf, 1.0, 0.0, 2.0], 1.0, nan), ([-inf, 1.0, 0.0, 2.0], 1.0, nan), ([nan, 1.0, 0.0, 2.0], 1.0, nan), ([0.0, -0.0, 0.0, 0.0], 3.0, 0.0),
              ([1e-30, -1e-30, 2e-30, 5e-31], 2.0 ** 100, None)]
    gate, up, want = torch.zeros(8, 32), torch.ones(8, 32), torch.zeros(8, 32, dtype=torch.float64)
    for i, (values, u, result) in enumerate(groups):
        gate[i] = torch.tensor(values).repeat(8)
        up[i] = u
        silu = gate[i].double() / (1 + torch.exp(-gate[i].double()))
        want[i] = silu * u if result is None else result
    step = 2.0 ** 20
    c = _codes(sr, mu, m, gate.reshape(-1).to(mu.DEV), up.reshape(-1).to(mu.DEV), group, step)
    want = want.reshape(-1).to(mu.DEV).expand(m, 256)
    assert torch.equal(c.values().isnan(), want.isnan())
    ok = ~want.isnan()
    unit = c.units().repeat_interleave(group, 1)
    saturated = want.abs() > 6 * unit            # groups of 16 under a step that is too small for them
    near = (c.values() - want).abs() <= unit * c.codes().abs().clamp(min=1) / 4 + 5 * 2.0 ** -24 * want.abs()
    # the least scale of groups of 16 is 2^-9, so one up to 2^-10 is rounded to 0: largest values up to 6 steps times that are coded as 0
    lost = (want.abs() <= 6 * step * 2.0 ** -10) & (unit == 0) & (c.codes() == 0) if group == 16 else torch.zeros_like(ok)
    assert bool((near | lost | (saturated & (c.codes().abs() == 6)))[ok].all())
    if group == 32:
        for i in (0, 2, 7):          # and they are there: the largest keeps its two bits
            top = want[:, 32 * i:32 * i + 32].abs().amax(1)
            assert bool(((c.values()[:, 32 * i:32 * i + 32].abs().amax(1) / top - 1).abs() < 0.2).all())
