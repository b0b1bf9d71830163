"""The gated block's fp16 output at the ends of the gate's range."""
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


@pytest.mark.parametrize("m", [1, 40, 300])
def test_gates_whose_exponential_is_next_to_the_largest_number(sr, mu, m):
    """exp(-gate) is finite down to -88.7, and h an ordinary number where up is large; below, h is 0."""
    import torch
    f = 256
    x, w = mu.Coded(m, 128, 32), mu.Coded(f, 128, 32)
    for c in (x, w):                  # value 0 of every row is 1, the others 0: sums are 1, gates and ups the steps
        c.q.zero_()
        c.q[:, 0] = 2
        c.s[mu.place(c.m, 128, 32)] = 127
    gate = torch.linspace(-88.7, -80.0, f, device=mu.DEV)
    gate[::8] = torch.tensor([float("inf"), 3e38, 100.0, 20.0, -89.0, -3e38, 0.0, -0.0], device=mu.DEV).repeat(4)
    up = torch.full((f,), 2.0 ** 120, device=mu.DEV)
    up[::8] = torch.tensor([1.0, 1e-36, 3.0, 3.0, 1.0, 1e30, 2.0, 2.0], device=mu.DEV).repeat(4)
    h = torch.empty(m, f, dtype=torch.float16, device=mu.DEV)
    sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s, gate_step=gate, up_step=up, h_out=h)
    g, u = gate.double(), up.double()
    want = g / (1 + torch.exp(-g)) * u
    want[::8] = torch.tensor([float("inf"), 3e38 * 1e-36, 300.0, 60.0, 0.0, 0.0, 0.0, 0.0], dtype=torch.float64, device=mu.DEV).repeat(4)
    assert bool((h[:, ::64].isinf()).all())
    got, want = h.double().flatten(), want.expand(m, f).flatten()
    ok = ~want.isinf()
    # the exponential's argument is rounded: |g| / ln 2 units of 2^-24 of which the exponential makes ln 2, and few more
    bound = mu.half_bound(want, (8 + 2 * g.abs().expand(m, f).flatten()) * 2.0 ** -23 * want.abs())
    assert bool(((got - want).abs() <= bound)[ok].all()) and sr.device_status() == 0
