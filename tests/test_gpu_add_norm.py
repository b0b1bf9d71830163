"""add_norm against its 64-bit definition, its codes against the quantizers run on its own values, rows of all lengths, aliases,
refusals; and a run of the feed-forward half of a layer with the coded products."""
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


def _want(mu, y, h, post, post_w, gate, bs, rs, eps):
    """The stream in 64 bits and a bound for fp32 with every product and sum rounded, before the rounding to fp16."""
    import torch
    z = torch.zeros_like(h.double()) if y is None else y.double()
    if post:
        z = z * mu.rms(z, eps)
        if post_w is not None:
            z = z * post_w.double()
    if gate is not None:
        z = z * gate.double()
    z = z * bs
    r = 0 if h is None else h.double() * rs
    return z + r, 6 * 2.0 ** -24 * (z.abs() + (0 if h is None else r.abs()))


# rows that no, one or two chunks more than a warp, a CTA of 512, of 1024 threads take; few rows and pairs of them, odd numbers
SIZES = [(1, 8), (1, 4096), (3, 40), (7, 896), (2, 8200), (3, 16392), (2, 32768), (149, 2048), (700, 4096), (301, 5120), (1501, 896), (400, 8192), (901, 136),
         (1200, 16), (333, 12288), (160, 20480)]


@pytest.mark.parametrize("post,gated", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("m,k", SIZES)
def test_values(sr, mu, m, k, post, gated):
    import torch
    g = mu.gen(m + k)
    y, h = mu.rows(g, m, k, 2.0, pad=24, shift=8), mu.rows(g, m, k, pad=8)
    w = [1 + 0.3 * torch.randn(k, generator=g, device=mu.DEV) for _ in range(3)]
    if m > 2:
        y[1], h[1] = 0, 0
    eps, bs, rs = 1e-5, 0.37, 1.0 if m % 2 else 0.81
    ho = torch.full((m, k + 16), 9.0, dtype=torch.float16, device=mu.DEV)
    xo = torch.full((m, k + 8), 9.0, dtype=torch.float16, device=mu.DEV)
    sr.add_norm(y, h, w[0], h_out=ho[:, 8:k + 8], x_out=xo[:, :k], post_norm=post, post_weight=w[1] if post and gated else None,
                gate=w[2] if gated else None, block_scale=bs, residual_scale=rs, eps=eps)
    want, extra = _want(mu, y, h, post, w[1] if post and gated else None, w[2] if gated else None, bs, rs, eps)
    got = ho[:, 8:k + 8].double()
    assert bool(((got - want).abs() <= mu.half_bound(want, extra)).all())
    x = got * mu.rms(got, eps) * w[0].double()                  # of the stream as it is held
    assert bool(((xo[:, :k].double() - x).abs() <= mu.half_bound(x, 3 * 2.0 ** -24 * x.abs())).all())
    assert bool((ho[:, :8] == 9).all()) and bool((ho[:, k + 8:] == 9).all()) and bool((xo[:, k:] == 9).all())


@pytest.mark.parametrize("codes", ["int4", "mx16", "mx32"])
@pytest.mark.parametrize("m,k", [(1, 128), (3, 4096), (5, 14336), (700, 4096), (451, 5120), (1301, 896), (301, 8192), (3, 32768)])
def test_codes_are_the_quantizers_own(sr, mu, m, k, codes):
    import torch
    if codes == "int4" and k > 16384:
        k = 16384                                              # as far as quant_act_plain goes
    g = mu.gen(k)
    y, h = mu.rows(g, m, k), mu.rows(g, m, k)
    w = [1 + 0.3 * torch.randn(k, generator=g, device=mu.DEV) for _ in range(2)]
    if m > 2:
        y[2], h[2] = 0, 0
    group = 16 if codes == "mx16" else 32
    got, want = mu.Coded(m, k, group), mu.Coded(m, k, group)
    step = torch.full((m,), float("nan"), device=mu.DEV)
    x, ho = torch.empty(m, k, dtype=torch.float16, device=mu.DEV), torch.empty(m, k, dtype=torch.float16, device=mu.DEV)
    kw = dict(post_weight=w[1], block_scale=0.5, clip=0.8)
    sr.add_norm(y, h, w[0], h_out=ho, x_out=x, q_out=got.q, scale_out=None if codes == "int4" else got.s, step_out=None if codes == "mx32" else step,
                codes=codes, **kw)
    if codes == "int4":
        steps = torch.empty(m, device=mu.DEV)
        sr.quant_act_plain(x, None, 0.8, want.q, steps)
    else:
        sr.mx_quant(x, want.q, want.s, want.step, group=group)
        steps = want.step
    assert torch.equal(got.q, want.q) and torch.equal(got.s, want.s)
    assert codes == "mx32" or torch.equal(step, steps)
    # codes alone, without values, and the values without codes
    alone, x2 = mu.Coded(m, k, group), torch.empty_like(x)
    sr.add_norm(y, h, w[0], q_out=alone.q, scale_out=None if codes == "int4" else alone.s, step_out=None if codes == "mx32" else step, codes=codes, **kw)
    sr.add_norm(y, h, w[0], x_out=x2, **kw)
    assert torch.equal(alone.q, want.q) and torch.equal(alone.s, want.s) and torch.equal(x2, x)


@pytest.mark.parametrize("m,k", [(2, 1024), (600, 1024)])
def test_one_sided_and_in_place(sr, mu, m, k):
    import torch
    g = mu.gen(5)
    y, h = mu.rows(g, m, k), mu.rows(g, m, k)
    out = lambda: torch.empty(m, k, dtype=torch.float16, device=mu.DEV)  # noqa: E731
    ho, xo = out(), out()
    sr.add_norm(None, h, x_out=xo, residual_scale=0.25)
    r = (h.double() * 0.25).half().double()
    x = r * mu.rms(r, 1e-5)
    assert bool(((xo.double() - x).abs() <= mu.half_bound(x, 3 * 2.0 ** -24 * x.abs())).all())
    sr.add_norm(y, None, h_out=ho, post_norm=True, block_scale=-2.0)
    z = y.double() * mu.rms(y.double(), 1e-5) * -2
    assert bool(((ho.double() - z).abs() <= mu.half_bound(z, 4 * 2.0 ** -24 * z.abs())).all())
    sr.add_norm(y, h, h_out=ho, x_out=xo)
    a, b = y.clone(), h.clone()
    sr.add_norm(a, b, h_out=b, x_out=a)                        # the stream in its place, x in the block output's
    assert torch.equal(b, ho) and torch.equal(a, xo)
    a, b = y.clone(), h.clone()
    sr.add_norm(a, b, h_out=a, x_out=b)
    assert torch.equal(a, ho) and torch.equal(b, xo)


@pytest.mark.parametrize("m", [3, 700])
def test_infinities_and_nan_stay_in_their_rows(sr, mu, m):
    import torch
    g = mu.gen(6)
    y, h = mu.rows(g, m, 512), mu.rows(g, m, 512)
    h[1, 7], y[2, 9] = float("inf"), float("nan")
    xo, ho = (torch.empty(m, 512, dtype=torch.float16, device=mu.DEV) for _ in range(2))
    c = mu.Coded(m, 512, 32)
    sr.add_norm(y, h, h_out=ho, x_out=xo, q_out=c.q, scale_out=c.s, codes="mx32", post_norm=True)
    rows = xo.isnan().any(1)
    assert rows[:3].tolist() == [False, True, True] and not bool(rows[3:].any())
    assert c.values().isnan().any(1).tolist() == rows.tolist()
    assert bool(ho[1].isinf().any()) and bool(ho[2].isnan().all())


def test_streams_replays_and_refusals(sr, mu):
    import torch
    g = mu.gen(7)
    y, h = mu.rows(g, 40, 256), mu.rows(g, 40, 256)
    ho, xo = (torch.empty(40, 256, dtype=torch.float16, device=mu.DEV) for _ in range(2))
    sr.add_norm(y, h, h_out=ho, x_out=xo)
    a, b = torch.empty_like(ho), torch.empty_like(xo)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sr.add_norm(y, h, h_out=a, x_out=b)
    side.synchronize()
    assert torch.equal(a, ho) and torch.equal(b, xo)
    before = sr.launch_count()
    v = torch.ones(256, device=mu.DEV)
    for bad in (lambda: sr.add_norm(y, h[:39], h_out=ho), lambda: sr.add_norm(None, None, h_out=ho), lambda: sr.add_norm(y, h, v[:8], x_out=xo),
                lambda: sr.add_norm(y, h, x_out=xo[:, :128]), lambda: sr.add_norm(y, h, codes="mx32"), lambda: sr.add_norm(y, h, x_out=xo.T)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sr.add_norm(y.float(), h, h_out=ho), lambda: sr.add_norm(y, h, v.half(), x_out=xo), lambda: sr.add_norm(y, h, x_out=xo, eps="1")):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sr.add_norm(y, h, h_out=ho, x_out=ho), lambda: sr.add_norm(y, h), lambda: sr.add_norm(y, h, h_out=ho, eps=0.0),
                lambda: sr.add_norm(y, h, h_out=ho, post_norm=False, post_weight=v), lambda: sr.add_norm(None, h, h_out=ho, gate=v)):
        with pytest.raises(sr.SmoothRotError):
            bad()
    sr.add_norm(y[:0], h[:0], h_out=ho[:0])
    assert sr.launch_count() == before and sr.device_status() == 0


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m", [1, 61, 300])
def test_the_feed_forward_half_of_a_layer(sr, mu, m, group):
    """norm and codes, gated block into the down projection's codes, down projection, norm into the stream: captured, replayed on a
    second input, and each step equal to the 64-bit form of what it was given."""
    import torch
    d, f = 512, 1408
    g = mu.gen(m)
    W = lambda n, k: (torch.randn(n, k, generator=g, device=mu.DEV) / k ** 0.5).half()  # noqa: E731
    gate, up, down = (mu.Coded(n, k, group) for n, k in ((f, d), (f, d), (d, f)))
    sr.mx_quant(W(f, d), gate.q, gate.s, gate.step, group=group)
    sr.mx_quant(W(f, d), up.q, up.s, up.step, group=group)
    sr.mx_quant(W(d, f), down.q, down.s, down.step, group=group, walsh=32)
    w1, w2 = (1 + 0.1 * torch.randn(d, generator=g, device=mu.DEV) for _ in range(2))
    h, attn = mu.rows(g, m, d), mu.rows(g, m, d)
    h0 = h.clone()
    x, c = mu.Coded(m, d, group), mu.Coded(m, f, group)
    steps = torch.full((m,), 2.0 ** -7, device=mu.DEV) if group == 16 else None
    y, out, last = (torch.empty(m, d, dtype=torch.float16, device=mu.DEV) for _ in range(3))
    code = "mx%d" % group

    def block():
        sr.add_norm(attn, h, w1, h_out=h, q_out=x.q, scale_out=x.s, step_out=x.step, codes=code)
        sr.mx_glu(x.q, x.s, gate.q, gate.s, up.q, up.s, group=group, x_step=x.step, gate_step=gate.step, up_step=up.step, q_out=c.q, scale_out=c.s,
                  h_step=steps, walsh=32)
        sr.mx_linear(c.q, c.s, down.q, down.s, y, group=group, x_step=steps, w_step=down.step)
        sr.add_norm(y, h, w2, h_out=out, x_out=last)

    block()
    torch.cuda.synchronize()
    first = [t.clone() for t in (h, y, out, last)]
    c.step = steps
    want, extra = mu.product(c.values(), down.values(), f)
    assert bool(((y.double() - want).abs() <= mu.half_bound(want, extra)).all())
    v, dv = mu.gated(x.values(), gate.values(), up.values(), d)
    dv = (dv + 7 * 2.0 ** -24 * v.abs()).reshape(m, -1, 32).sum(2).repeat_interleave(32, 1) / 32 ** 0.5
    c.step = None
    mu.check_codes(c, mu.walsh(v, 32), dv, step=steps)
    stream = h0.double() + attn.double()
    assert bool(((h.double() - stream).abs() <= mu.half_bound(stream, 2.0 ** -24 * stream.abs())).all())
    normed = h.double() * mu.rms(h.double(), 1e-5) * w1.double()
    mu.check_codes(x, normed, mu.half_bound(normed, 3 * 2.0 ** -24 * normed.abs()))        # codes of the fp16 values
    stream = h.double() + y.double()
    assert bool(((out.double() - stream).abs() <= mu.half_bound(stream, 2.0 ** -24 * stream.abs())).all())
    normed = out.double() * mu.rms(out.double(), 1e-5) * w2.double()
    assert bool(((last.double() - normed).abs() <= mu.half_bound(normed, 3 * 2.0 ** -24 * normed.abs())).all())
    graph = torch.cuda.CUDAGraph()
    h.copy_(h0)
    with torch.cuda.graph(graph):
        block()
    h.copy_(h0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((h, y, out, last), first))
    assert sr.device_status() == 0
