"""mx_quant and mx_dequant against their 64-bit definition: exact where nothing is rounded on the way, layouts, edges, refusals."""
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


def _run(sr, mu, x, group, **kw):
    c = mu.Coded(x.shape[0], x.shape[1], group)
    sr.mx_quant(x, c.q, c.s, c.step, group=group, **kw)
    return c


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m,k,pad,shift", [(1, 128, 0, 0), (1, 4096, 0, 0), (3, 384, 8, 8), (37, 896, 0, 0), (130, 640, 24, 8), (300, 14336, 0, 0),
                                           (5, 32768, 0, 0), (1700, 4096, 32, 16), (4097, 128, 0, 0), (257, 17408, 0, 0)])
def test_codes_of_fp16_values_are_those_of_the_definition(sr, mu, m, k, pad, shift, group):
    import torch
    x = mu.rows(mu.gen(m + k), m, k, pad=pad, shift=shift)
    if m > 2:
        x[1] = 0
        x[2, :group] = 0
        x[2, group:2 * group] *= 2.0 ** -12      # far below the row's largest
    c = _run(sr, mu, x, group)
    v = x.double()
    g = v.reshape(m, -1, group)
    top = g.abs().amax(2)
    if group == 32:
        unit = mu.scale_32(top)
    else:
        step = mu.step_16(top.amax(1))
        assert torch.equal(c.step.double(), step)
        unit = mu.e4m3(top / (6 * step[:, None])) * step[:, None]
    assert torch.equal(c.units(), unit)
    assert torch.equal(c.values(), mu.nearest(v, unit.repeat_interleave(group, 1)))
    # bytes of rows that are not there are left alone
    rest = torch.ones(c.s.numel(), dtype=torch.bool, device=mu.DEV)
    rest[mu.place(m, k, group)] = False
    assert bool((c.s[rest] == (255 if group == 32 else 127)).all())
    y = torch.full((m, k + 8), 7.0, dtype=torch.float16, device=mu.DEV)
    sr.mx_dequant(c.q, c.s, c.step, y[:, :k], group=group)
    assert torch.equal(y[:, :k], c.values().half()) and bool((y[:, k:] == 7).all())


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m,k,walsh,pre", [(1, 128, 32, False), (1, 4096, 128, True), (70, 896, 64, True), (70, 896, 32, True), (333, 14336, 128, True),
                                           (129, 384, 128, False), (2100, 1024, 64, False), (33, 2048, 0, True), (5, 20480, 128, True)])
def test_diagonal_and_rotation(sr, mu, m, k, walsh, pre, group):
    import torch
    g = mu.gen(k + walsh)
    x = mu.rows(g, m, k)
    d = torch.exp(torch.randn(k, generator=g, device=mu.DEV)) if pre else None
    c = _run(sr, mu, x, group, pre=d, walsh=walsh)
    v = x.double() * (d.double() if pre else 1)
    n = walsh or 1
    size = v.abs().reshape(m, -1, n).sum(2).repeat_interleave(n, 1) / n ** 0.5
    # the diagonal's product, an addition per stage and the norm (itself rounded), each half a unit of fp32 of what it comes to
    mu.check_codes(c, mu.walsh(v, walsh), (n.bit_length() + 2) * 2.0 ** -24 * size)


@pytest.mark.parametrize("group", [32, 16])
def test_infinities_and_nan_are_kept(sr, mu, group):
    import torch
    x = mu.rows(mu.gen(4), 6, 512)
    x[1, 40], x[2, 300], x[3, 511] = float("inf"), float("nan"), float("-inf")
    x[4, 64:96] = 65504
    v = _run(sr, mu, x, group).values()
    bad = torch.zeros(6, 512 // group, dtype=torch.bool, device=mu.DEV)
    for r, at in ((1, 40), (2, 300), (3, 511)):
        bad[r] = True if group == 16 else bad[r]
        bad[r, at // group] = True
    assert torch.equal(v.isnan(), bad.repeat_interleave(group, 1))
    y = torch.zeros(6, 512, dtype=torch.float16, device=mu.DEV)
    c = _run(sr, mu, x, group)
    sr.mx_dequant(c.q, c.s, c.step, y, group=group)
    assert torch.equal(y.isnan(), v.isnan())


@pytest.mark.parametrize("group", [32, 16])
def test_smallest_and_largest_values(sr, mu, group):
    """fp16 subnormals alone in a row, and a diagonal that takes values below what a scale reaches."""
    import torch
    x = torch.zeros(3, 128, dtype=torch.float16, device=mu.DEV)
    x[0, 3], x[1, 5] = 2.0 ** -24, -65504
    x[2] = torch.linspace(-1, 1, 128, device=mu.DEV).half()
    c = _run(sr, mu, x, group)
    # groups of 32: 2^-24 is 4 under 2^-26.  Groups of 16: a group's largest value is 6 scales, and the scale is within half a step of its
    # 3 bits, 2^-4 of it.
    got = float(c.values()[0, 3])
    assert got == float(c.values()[0].abs().sum()) and abs(got - 2.0 ** -24) <= (0 if group == 32 else 2.0 ** -4 * 2.0 ** -24)
    # 65504 is the largest: 4 under 2^14 (and 65504 above 3.5 of it) or 6 scales
    assert abs(float(c.values()[1, 5]) + 65504) <= (32 if group == 32 else 65504 / 16)
    tiny = torch.full((128,), 2.0 ** -126, device=mu.DEV)
    c = _run(sr, mu, x, group, pre=tiny)
    assert not bool(c.values().isnan().any()) and float(c.values().abs().max()) <= 2.0 ** -100


def test_streams_graphs_and_refusals(sr, mu):
    import torch
    x = mu.rows(mu.gen(1), 40, 512)
    want = _run(sr, mu, x, 32)
    c = mu.Coded(40, 512, 32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sr.mx_quant(x, c.q, c.s, group=32)
    side.synchronize()
    assert torch.equal(c.q, want.q) and torch.equal(c.s, want.s)
    graph, c = torch.cuda.CUDAGraph(), mu.Coded(40, 512, 32)
    y = torch.zeros(40, 512, dtype=torch.float16, device=mu.DEV)
    with torch.cuda.graph(graph):
        sr.mx_quant(x, c.q, c.s, group=32)
        sr.mx_dequant(c.q, c.s, None, y, group=32)
    x.mul_(-0.5)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want.values().half() * -0.5)
    before = sr.launch_count()
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=mu.DEV)  # noqa: E731
    for bad in (lambda: sr.mx_quant(x, u8(40, 255), c.s), lambda: sr.mx_quant(x, c.q, u8(100)), lambda: sr.mx_quant(x[:, ::2], u8(40, 128), c.s),
                lambda: sr.mx_quant(x, c.q, c.s, pre=torch.ones(100, device=mu.DEV)), lambda: sr.mx_dequant(c.q, c.s, None, y[:39]),
                lambda: sr.mx_quant(x, c.q, u8(20, 2048)[:, ::2])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sr.mx_quant(x.float(), c.q, c.s), lambda: sr.mx_quant(x, c.q.int(), c.s), lambda: sr.mx_quant(x, c.q, c.s, group="32")):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sr.mx_quant(x, c.q, c.s, torch.zeros(40, device=mu.DEV)), lambda: sr.mx_quant(x, c.q, u8(16384), group=16),
                lambda: sr.mx_quant(x, c.q, c.s, walsh=8)):
        with pytest.raises(sr.SmoothRotError):
            bad()
    assert sr.launch_count() == before and sr.device_status() == 0
    e = torch.zeros(0, 512, dtype=torch.float16, device=mu.DEV)
    sr.mx_quant(e, u8(0, 256), u8(0))
    sr.mx_dequant(u8(0, 256), u8(0), None, e)
    assert sr.launch_count() == before
