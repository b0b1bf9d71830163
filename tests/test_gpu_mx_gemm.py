"""mx_linear and mx_glu against 64-bit forms of the coded operands: sizes and edges of both kernels, groups, steps, both outputs of the
gated block, layouts, streams and replays, refusals."""
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


def _linear(sr, mu, x, w, pad=0):
    import torch
    y = torch.full((x.m, w.m + pad), 9.0, dtype=torch.float16, device=mu.DEV)
    sr.mx_linear(x.q, x.s, w.q, w.s, y[:, :w.m], group=x.group, x_step=x.step, w_step=w.step)
    return y


# one token, borders of the token tiles 16, 32, 64, 128 and of the pair's 256; channels that end inside a tile; a last half block of k;
# more blocks than the rings have stages; K split over 1, 2, 4 and 8 CTAs
SIZES = [(1, 8, 128), (1, 4096, 4096), (2, 136, 384), (16, 512, 1024), (17, 264, 2048), (32, 128, 8192), (33, 1000, 640), (64, 2056, 896), (65, 24, 14336),
         (128, 1288, 4096), (129, 136, 384), (256, 256, 256), (257, 520, 128), (300, 1000, 896), (700, 2816, 1024), (1100, 4096, 512), (130, 64, 32768)]


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear(sr, mu, m, n, k, group):
    g = mu.gen(m + n + k)
    x, w = mu.random_coded(g, m, k, group), mu.random_coded(g, n, k, group)
    w.step = None if group == 16 and m % 2 else w.step      # the step of 1
    y = _linear(sr, mu, x, w, pad=8)
    want, extra = mu.product(x.values(), w.values(), k)
    assert bool(((y[:, :n].double() - want).abs() <= mu.half_bound(want, extra)).all())
    assert bool((y[:, n:] == 9).all()) and sr.device_status() == 0


@pytest.mark.parametrize("m", [3, 40, 200])
def test_steps_with_groups_of_32_and_wide_scales(sr, mu, m):
    """Steps are taken with either group; scales from 2^-60 to 2^60 that meet in sums."""
    import torch
    g = mu.gen(m)
    x, w = mu.random_coded(g, m, 512, 32, 40), mu.random_coded(g, 136, 512, 32, 40)
    xs, ws = torch.rand(m, generator=g, device=mu.DEV) + 0.5, torch.rand(136, generator=g, device=mu.DEV) + 0.5
    y = torch.empty(m, 136, dtype=torch.float16, device=mu.DEV)
    sr.mx_linear(x.q, x.s, w.q, w.s, y, x_step=xs * 2.0 ** 10, w_step=ws)
    want, extra = mu.product(x.values() * (xs.double() * 2.0 ** 10)[:, None], w.values() * ws.double()[:, None], 512)
    assert bool(((y.double() - want).abs() <= mu.half_bound(want, extra)).all())


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m", [5, 100, 300])
def test_nan_scales_stay_in_their_rows_and_columns(sr, mu, m, group):
    import torch
    g = mu.gen(m)
    x, w = mu.random_coded(g, m, 384, group), mu.random_coded(g, 72, 384, group)
    x.s[mu.place(m, 384, group)[3, 5]] = 255 if group == 32 else 127
    w.s[mu.place(72, 384, group)[70, 1]] = 255 if group == 32 else 127
    y = _linear(sr, mu, x, w)
    bad = torch.zeros(m, 72, dtype=torch.bool, device=mu.DEV)
    bad[3], bad[:, 70] = True, True
    assert torch.equal(y.isnan(), bad)
    # infinite sums and zeros: an overflow of fp16 is an infinity, rows of zero codes give zeros
    x, w = mu.random_coded(g, m, 384, 32), mu.random_coded(g, 72, 384, 32)
    x.s[mu.place(m, 384, 32)[0]] = 200
    x.q[1] = 0
    y = _linear(sr, mu, x, w)
    assert bool((y[0].isinf() | (y[0] == 0)).all()) and bool((y[1] == 0).all()) and not bool(y[2:].isnan().any())


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (50, 1024, 4096), (600, 1032, 1024)])
def test_calls_repeated_side_by_side_and_replayed_give_the_same_bits(sr, mu, m, n, k):
    import torch
    g = mu.gen(k)
    x, w = mu.random_coded(g, m, k, 32), mu.random_coded(g, n, k, 32)
    want = _linear(sr, mu, x, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            got.append(_linear(sr, mu, x, w))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)
    graph, y = torch.cuda.CUDAGraph(), torch.empty(m, n, dtype=torch.float16, device=mu.DEV)
    with torch.cuda.graph(graph):
        for _ in range(3):
            sr.mx_linear(x.q, x.s, w.q, w.s, y)
    x.q ^= 0x88        # every sign turned: what is replayed reads the operands anew
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, -want)


GATED = [(1, 8, 128), (1, 14336, 4096), (3, 136, 384), (16, 64, 256), (17, 200, 1024), (40, 1000, 896), (64, 2816, 512), (100, 384, 4096), (128, 5632, 256),
         (129, 136, 384), (256, 128, 256), (333, 5632, 2048), (520, 1288, 640)]


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m,f,k", GATED)
def test_glu_values(sr, mu, m, f, k, group):
    import torch
    g = mu.gen(m + f)
    x, a, b = (mu.random_coded(g, r, k, group) for r in (m, f, f))
    scale = 2.0 / k ** 0.5 / (1 if group == 32 else 8)
    a.step = (torch.rand(f, generator=g, device=mu.DEV) + 0.1) * scale if group == 16 else torch.full((f,), scale, device=mu.DEV)
    h = torch.full((m, f + 16), 9.0, dtype=torch.float16, device=mu.DEV)
    walsh = 32 if f % 32 == 0 and m % 2 else 0
    sr.mx_glu(x.q, x.s, a.q, a.s, b.q, b.s, group=group, x_step=x.step, gate_step=a.step, up_step=b.step, h_out=h[:, 8:f + 8], walsh=walsh)
    gate = a.values() if group == 16 else a.values() * scale
    want, extra = mu.gated(x.values(), gate, b.values(), k)
    if walsh:
        extra = (extra + 7 * 2.0 ** -24 * want.abs()).reshape(m, -1, 32).sum(2).repeat_interleave(32, 1) / 32 ** 0.5
        want = mu.walsh(want, 32)
    ok = want.abs() < 60000
    assert bool(((h[:, 8:f + 8].double() - want).abs() <= mu.half_bound(want, extra))[ok].all())
    assert bool((h[:, :8] == 9).all()) and bool((h[:, f + 8:] == 9).all()) and sr.device_status() == 0


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("walsh", [0, 32])
@pytest.mark.parametrize("m,f,k", [(1, 128, 256), (1, 14336, 1024), (7, 384, 640), (30, 1280, 512), (61, 128, 4096), (128, 640, 384), (129, 256, 384), (400, 1024, 1024)])
def test_glu_codes(sr, mu, m, f, k, walsh, group):
    import torch
    g = mu.gen(m + f + walsh)
    x, a, b = (mu.random_coded(g, r, k, group) for r in (m, f, f))
    if group == 32:
        a.step = b.step = None
        a.s = (a.s.int() - 4).clamp(min=0).to(torch.uint8)
    c = mu.Coded(m, f, group)
    steps = torch.rand(m, generator=g, device=mu.DEV) + 0.25 if group == 16 else None
    sr.mx_glu(x.q, x.s, a.q, a.s, b.q, b.s, group=group, x_step=x.step, gate_step=a.step, up_step=b.step, q_out=c.q, scale_out=c.s, h_step=steps, walsh=walsh)
    want, extra = mu.gated(x.values(), a.values(), b.values(), k)
    if walsh:
        extra = (extra + 7 * 2.0 ** -24 * want.abs()).reshape(m, -1, 32).sum(2).repeat_interleave(32, 1) / 32 ** 0.5
        want = mu.walsh(want, 32)
    c.step = None
    mu.check_codes(c, want, extra, step=steps)
    rest = torch.ones(c.s.numel(), dtype=torch.bool, device=mu.DEV)
    rest[mu.place(m, f, group)] = False
    assert bool((c.s[rest] == (255 if group == 32 else 127)).all())


def test_large_gates(sr, mu):
    """exp(-gate) beyond fp32 gives 0 on one side and the gate itself on the other."""
    import torch
    x, w = mu.Coded(2, 128, 32), mu.Coded(16, 128, 32)
    for c in (x, w):
        c.q[:] = 0x22                                       # ones
        c.s[mu.place(c.m, 128, 32)] = 127
    w.q[8:] = 0xaa
    up = mu.Coded(16, 128, 32)
    up.q[:], up.s[mu.place(16, 128, 32)] = 0x22, 127
    h = torch.empty(2, 16, dtype=torch.float16, device=mu.DEV)
    for m in (2, 200):
        xx = mu.Coded(m, 128, 32)
        xx.q[:], xx.s[mu.place(m, 128, 32)] = 0x22, 127
        h = torch.empty(m, 16, dtype=torch.float16, device=mu.DEV)
        sr.mx_glu(xx.q, xx.s, w.q, w.s, up.q, up.s, h_out=h)
        assert bool((h[:, :8] == 128 * 128).all()) and bool((h[:, 8:] == 0).all())


def test_refusals_and_empty_calls(sr, mu):
    import torch
    g = mu.gen(0)
    x, w = mu.random_coded(g, 4, 256, 32), mu.random_coded(g, 128, 256, 32)
    y = torch.zeros(4, 128, dtype=torch.float16, device=mu.DEV)
    before = sr.launch_count()
    other = mu.random_coded(g, 128, 384, 32)
    c = mu.Coded(4, 128, 32)
    for bad in (lambda: sr.mx_linear(x.q, x.s, other.q, other.s, y), lambda: sr.mx_linear(x.q, x.s, w.q, w.s, y[:, :64]),
                lambda: sr.mx_linear(x.q, x.s[:100], w.q, w.s, y), lambda: sr.mx_linear(x.q, x.s, w.q, w.s, y, w_step=torch.ones(4, device=mu.DEV)),
                lambda: sr.mx_linear(x.q.T, x.s, w.q, w.s, y), lambda: sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s),
                lambda: sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s, h_out=y, q_out=c.q, scale_out=c.s),
                lambda: sr.mx_glu(x.q, x.s, w.q, w.s, w.q[:64], w.s, h_out=y), lambda: sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s, q_out=c.q),
                lambda: sr.mx_glu(x.q, x.s, w.q[:64], w.s, w.q[:64], w.s, q_out=c.q[:, :32], scale_out=c.s)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sr.mx_linear(x.q, x.s, w.q, w.s, y.float()), lambda: sr.mx_linear(x.q, x.s.int(), w.q, w.s, y)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sr.mx_linear(x.q, x.s, w.q[:12], w.s, y[:, :12]), lambda: sr.mx_glu(x.q, x.s, w.q, w.s, w.q, w.s, h_out=y, walsh=64)):
        with pytest.raises(sr.SmoothRotError):
            bad()
    sr.mx_linear(x.q[:0], x.s[:0], w.q, w.s, y[:0])
    sr.mx_linear(x.q, x.s, w.q[:0], w.s[:0], y[:, :0])
    sr.mx_glu(x.q[:0], x.s[:0], w.q, w.s, w.q, w.s, h_out=y[:0])
    assert sr.launch_count() == before and sr.device_status() == 0


def test_a_wait_that_runs_out_is_reported(sr, mu):
    import torch
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    sr.debug_set_wait_limit_ns(1_000_000)
    try:
        sr.debug_mx_wait_expiry()
        torch.cuda.synchronize()
        assert sr.device_status(clear=False) == 50 and sr.device_status() == 50 and sr.device_status() == 0
    finally:
        sr.debug_set_wait_limit_ns(0)
    g = mu.gen(0)
    x, w = mu.random_coded(g, 40, 256, 32), mu.random_coded(g, 128, 256, 32)
    want, extra = mu.product(x.values(), w.values(), 256)
    assert bool(((_linear(sr, mu, x, w).double() - want).abs() <= mu.half_bound(want, extra)).all())
