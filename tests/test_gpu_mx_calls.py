"""The microscaled operators and norms called as programs call them: captured with branches that join, as the first call of a process,
from two threads, over tensors of more than 2^32 values, over themselves, and with arguments that do not go together."""
import subprocess
import sys
import threading

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


def _quant(sr, x, c):
    sr.mx_quant(x, c.q, c.s, c.step, group=c.group)


@pytest.mark.parametrize("m,n,k", [(1, 256, 1024), (300, 520, 4096)])
def test_branches_that_join_in_a_capture(sr, mu, m, n, k):
    """Copies, quantizers on two streams, the product of both: what follows a branch or a copy waits for it."""
    import torch
    g = mu.gen(n)
    x, w = torch.empty(m, k, dtype=torch.float16, device=mu.DEV), torch.empty(n, k, dtype=torch.float16, device=mu.DEV)
    source = [mu.rows(g, m, k), mu.rows(g, n, k)]
    cx, cw = mu.Coded(m, k, 16), mu.Coded(n, k, 16)
    y, back = torch.empty(m, n, dtype=torch.float16, device=mu.DEV), torch.empty(n, k, dtype=torch.float16, device=mu.DEV)
    _quant(sr, source[0], cx)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        x.copy_(source[0])
        _quant(sr, x, cx)
        with torch.cuda.stream(side):
            w.copy_(source[1])
            _quant(sr, w, cw)
            sr.mx_dequant(cw.q, cw.s, cw.step, back, group=16)
        main.wait_stream(side)
        sr.mx_linear(cx.q, cx.s, cw.q, cw.s, y, group=16, x_step=cx.step, w_step=cw.step)
        x.zero_()
    for seed in range(3):
        source[0].copy_(mu.rows(mu.gen(seed), m, k))
        source[1].copy_(mu.rows(mu.gen(seed + 7), n, k))
        graph.replay()
        torch.cuda.synchronize()
        a, b, want = mu.Coded(m, k, 16), mu.Coded(n, k, 16), torch.empty_like(y)
        _quant(sr, source[0], a)
        _quant(sr, source[1], b)
        sr.mx_linear(a.q, a.s, b.q, b.s, want, group=16, x_step=a.step, w_step=b.step)
        assert torch.equal(a.q, cx.q) and torch.equal(b.q, cw.q) and torch.equal(a.step, cx.step) and torch.equal(y, want)
        assert torch.equal(back, b.values().half()) and bool((x == 0).all())


FIRST = """
import torch
from paper_2506_05413_b200 import binding as sr
torch.manual_seed(0)
D = "cuda:0"
def go(m, c, y):
    sr.add_norm(None, x[:m], x_out=n[:m], q_out=c[0], scale_out=c[1], codes="mx32")
    sr.mx_linear(c[0], c[1], w, ws, y)
x = torch.randn(300, 4096, device=D).half()
n = torch.empty_like(x)
w = torch.randint(0, 256, (1024, 2048), device=D, dtype=torch.int32).to(torch.uint8)
ws = torch.full((1024 * 128,), 120, dtype=torch.uint8, device=D)
for m in (1, 300):
    c = torch.empty(m, 2048, dtype=torch.uint8, device=D), torch.empty(384 * 128, dtype=torch.uint8, device=D)
    y, again = torch.empty(m, 1024, dtype=torch.float16, device=D), torch.empty(m, 1024, dtype=torch.float16, device=D)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(m, c, y)
    graph.replay()
    go(m, c, again)
    torch.cuda.synchronize()
    assert torch.equal(y, again) and bool(y.isfinite().all())
print("same")
"""


def test_the_first_call_of_a_process_may_be_captured(sr):
    done = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "same" in done.stdout, done.stderr[-2000:]


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m,n,k", [(1, 5000, 1024), (2, 4360, 768), (16, 4360, 896), (31, 5120, 2048), (61, 5120, 640), (64, 5000, 896), (127, 4488, 768), (128, 5120, 1024),
                                   (150, 2600, 896)])
def test_k_in_three_parts(sr, mu, m, n, k, group):
    """Sizes whose tiles leave room for three parts of K, which divide neither the tokens of a tile nor the k-blocks."""
    import torch
    g = mu.gen(m + n)
    x, w = mu.random_coded(g, m, k, group), mu.random_coded(g, n, k, group)
    y = torch.full((m, n + 8), 9.0, dtype=torch.float16, device=mu.DEV)
    again = torch.empty(m, n, dtype=torch.float16, device=mu.DEV)
    for out in (y[:, :n], again):
        sr.mx_linear(x.q, x.s, w.q, w.s, out, group=group, x_step=x.step, w_step=w.step)
    want, extra = mu.product(x.values(), w.values(), k)
    assert bool(((again.double() - want).abs() <= mu.half_bound(want, extra)).all())
    assert torch.equal(y[:, :n], again) and bool((y[:, n:] == 9).all()) and sr.device_status() == 0


@pytest.mark.parametrize("m", [1, 15, 40, 100])
def test_gated_tiles_in_three_parts(sr, mu, m):
    import torch
    g = mu.gen(m)
    x, a, b = (mu.random_coded(g, r, 896, 32) for r in (m, 2536, 2536))
    step = torch.full((2536,), 2.0 / 30, device=mu.DEV)
    h = torch.full((m, 2536), 9.0, dtype=torch.float16, device=mu.DEV)
    sr.mx_glu(x.q, x.s, a.q, a.s, b.q, b.s, h_out=h, gate_step=step, up_step=step)
    want, extra = mu.gated(x.values(), a.values() * step.double()[:, None], b.values() * step.double()[:, None], 896)
    assert bool(((h.double() - want).abs() <= mu.half_bound(want, extra)).all()) and sr.device_status() == 0


def test_two_threads_with_a_stream_each(sr, mu):
    """Calls of both product kernels, the quantizer and the norm side by side."""
    import torch
    g = mu.gen(5)
    work = []
    for m in (4, 700):
        x, c, w = mu.rows(g, m, 2048), mu.Coded(m, 2048, 32), mu.random_coded(g, 2048, 2048, 32)
        h, y = torch.empty_like(x), torch.empty(m, 2048, dtype=torch.float16, device=mu.DEV)

        def go(x=x, c=c, w=w, h=h, y=y):
            sr.add_norm(x, x, h_out=h, q_out=c.q, scale_out=c.s, codes="mx32")
            sr.mx_linear(c.q, c.s, w.q, w.s, y)
            return torch.cat([h, y], 1)

        work.append((go, go()))
    torch.cuda.synchronize()
    bad = []

    def run(go, want):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(40):
                if not torch.equal(go(), want):
                    bad.append(want.shape)

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad and sr.device_status() == 0


def test_offsets_beyond_32_bits(sr, mu):
    """262,400 rows of 16384 values: the last rows are what they are alone."""
    import torch
    m, k, first = 262_400, 16384, 262_144
    tail = m - first
    x = torch.empty(m, k, dtype=torch.float16, device=mu.DEV)
    x.view(-1, 64, k)[:] = mu.rows(mu.gen(1), 64, k)
    x[first:] = mu.rows(mu.gen(2), tail, k)
    few = x[first:].clone()
    for group in (32, 16):
        c, t = mu.Coded(m, k, group), mu.Coded(tail, k, group)
        _quant(sr, x, c)
        _quant(sr, few, t)
        at = first * (k // group)
        assert torch.equal(c.q[first:], t.q) and torch.equal(c.s[at:], t.s) and (group == 32 or torch.equal(c.step[first:], t.step))
        y = torch.empty_like(x)
        sr.mx_dequant(c.q, c.s, c.step, y, group=group)
        assert torch.equal(y[first:], t.values().half())
    h, ht = torch.empty_like(x), torch.empty_like(few)
    sr.add_norm(x, y, h_out=h, x_out=y, q_out=c.q, scale_out=c.s, step_out=c.step, codes="mx16", post_norm=True)
    yt = t.values().half()
    sr.add_norm(few, yt, h_out=ht, x_out=yt, q_out=t.q, scale_out=t.s, step_out=t.step, codes="mx16", post_norm=True)
    assert torch.equal(h[first:], ht) and torch.equal(y[first:], yt) and torch.equal(c.q[first:], t.q) and torch.equal(c.step[first:], t.step)
    del x, few, c, t
    g = mu.gen(3)
    x, w, u = mu.random_coded(g, m, 256, 32), mu.random_coded(g, k, 256, 32), mu.random_coded(g, k, 256, 32)
    xs = mu.Coded(tail, 256, 32)
    xs.q, xs.s = x.q[first:].contiguous(), x.s[first * 8:].contiguous()
    sr.mx_linear(x.q, x.s, w.q, w.s, h)
    want, extra = mu.product(xs.values(), w.values(), 256)
    assert bool(((h[first:].double() - want).abs() <= mu.half_bound(want, extra)).all())
    step = torch.full((k,), 0.1, device=mu.DEV)
    sr.mx_glu(x.q, x.s, w.q, w.s, u.q, u.s, h_out=y, gate_step=step, up_step=step)
    sr.mx_glu(xs.q, xs.s, w.q, w.s, u.q, u.s, h_out=yt, gate_step=step, up_step=step)
    assert torch.equal(y[first:], yt)
    c, t = mu.Coded(m, k, 32), mu.Coded(tail, k, 32)
    sr.mx_glu(x.q, x.s, w.q, w.s, u.q, u.s, q_out=c.q, scale_out=c.s, gate_step=step, up_step=step, walsh=32)
    sr.mx_glu(xs.q, xs.s, w.q, w.s, u.q, u.s, q_out=t.q, scale_out=t.s, gate_step=step, up_step=step, walsh=32)
    assert torch.equal(c.q[first:], t.q) and torch.equal(c.s[first * (k // 32):], t.s) and sr.device_status() == 0


@pytest.mark.parametrize("m", [5, 700])
def test_integer_codes_of_rows_with_infinities_and_nan(sr, mu, m):
    """As the quantizer of integer codes makes them from the same values, but for rows with a NaN: their step is NaN."""
    import torch
    x = mu.rows(mu.gen(m), m, 1024)
    x[1, 7], x[2, 9], x[3, 11], x[4] = float("inf"), float("nan"), -float("inf"), 0
    h, n = torch.zeros_like(x), torch.empty_like(x)
    q, step = torch.empty(m, 512, dtype=torch.uint8, device=mu.DEV), torch.empty(m, device=mu.DEV)
    sr.add_norm(x, h, x_out=n, q_out=q, step_out=step, codes="int4", clip=0.9)
    want, ws = torch.empty_like(q), torch.empty_like(step)
    sr.quant_act_plain(n, None, 0.9, want, ws)
    # rows 1 to 3 hold a NaN (an infinity times a norm of 0), which the quantizer of integer codes passes over; here it stays in the step
    whole = ~n.isnan().any(1)
    assert whole[:5].tolist() == [True, False, False, False, True] and bool(whole[5:].all())
    assert torch.equal(q[whole], want[whole]) and torch.equal(step[whole], ws[whole]) and bool(step[~whole].isnan().all())


@pytest.mark.parametrize("group", [32, 16])
@pytest.mark.parametrize("m", [3, 40, 300])
def test_gated_values_that_leave_the_range(sr, mu, m, group):
    """Through a weight step: feature 5's sums are infinite, feature 70's NaN, feature 200's large, the rest ordinary.  Infinities and
    NaN make their group NaN; what is only too large for the row's step saturates."""
    import torch
    g = mu.gen(m)
    x, a, b = (mu.random_coded(g, r, 512, group) for r in (m, 256, 256))
    a.step = torch.full((256,), 2.0 ** -4, device=mu.DEV)
    b.step = a.step.clone()
    a.q[5], b.q[5], x.q[:] = 0x22, 0x22, x.q & 0x77        # sums of positive products
    a.step[5] = b.step[5] = 2.0 ** 100
    a.step[70] = float("nan")
    b.step[200] = 2.0 ** 60
    a.q[200], b.q[200] = 0x22, 0x22
    a.step[200] = 1.0
    c, h = mu.Coded(m, 256, group), torch.full((m,), 2.0 ** -6, device=mu.DEV)
    sr.mx_glu(x.q, x.s, a.q, a.s, b.q, b.s, group=group, x_step=x.step, gate_step=a.step, up_step=b.step, q_out=c.q, scale_out=c.s,
              h_step=h if group == 16 else None)
    c.step = h if group == 16 else None
    nan = c.units().isnan()
    want = torch.zeros(256 // group, dtype=torch.bool, device=mu.DEV)
    want[5 // group] = want[70 // group] = True
    assert bool((nan == want).all())
    far = c.values()[:, 200]
    assert bool((far == (2688.0 * 2.0 ** -6)).all()) if group == 16 else bool((far > 2.0 ** 55).all())


@pytest.mark.parametrize("which", ["x", "gate", "up", "x and up"])
@pytest.mark.parametrize("m", [20, 150, 600])
def test_steps_one_at_a_time(sr, mu, m, which):
    """The linear layer and the gated pair with some of their steps only, channels that end inside a tile, several tiles to a CTA."""
    import torch
    g = mu.gen(m)
    f, k = 2824 if m == 600 else 392, 384
    x, a, b = (mu.random_coded(g, r, k, 32) for r in (m, f, f))
    steps = {name: torch.rand(n, generator=g, device=mu.DEV) * 0.1 + 0.01 for name, n in (("x", m), ("gate", f), ("up", f))}
    given = {name: s if name in which else None for name, s in steps.items()}
    xs, gs, us = (x.values(), a.values(), b.values())
    xs, gs, us = (v if given[n] is None else v * given[n].double()[:, None] for n, v in (("x", xs), ("gate", gs), ("up", us)))
    y, h = (torch.empty(m, f, dtype=torch.float16, device=mu.DEV) for _ in range(2))
    sr.mx_linear(x.q, x.s, a.q, a.s, y, x_step=given["x"], w_step=given["gate"])
    want, extra = mu.product(xs, gs, k)
    assert bool(((y.double() - want).abs() <= mu.half_bound(want, extra)).all())
    sr.mx_glu(x.q, x.s, a.q, a.s, b.q, b.s, h_out=h, x_step=given["x"], gate_step=given["gate"], up_step=given["up"])
    want, extra = mu.gated(xs, gs, us, k)
    fine = (want.abs() + extra) < 65504          # beyond, fp16 is infinite
    assert bool((((h.double() - want).abs() <= mu.half_bound(want, extra)) | ~fine).all())


@pytest.mark.parametrize("power", [-60, -3, 0, 40])
def test_every_scale_at_the_borders_between_codes(sr, mu, power):
    """Groups of 16 whose largest value is 6 scales, for all scales but 0, with values on the borders: a border belongs to the even code."""
    import torch
    scale = torch.tensor([(1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) if b >> 3 else (b & 7) / 512 for b in range(1, 127)], device=mu.DEV)
    borders = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    grid = torch.tensor([6.0, 0.5] + borders + [-b for b in borders], device=mu.DEV)
    even = torch.tensor([7, 1, 0, 2, 2, 4, 4, 6, 6, 8, 10, 10, 12, 12, 14, 14], dtype=torch.uint8, device=mu.DEV)
    x = torch.zeros(3, 2048, device=mu.DEV)
    x[:, :126 * 16] = (scale[:, None] * grid).reshape(-1)
    x[1] *= 0.5
    x[2] *= 2.0 ** -3
    c = mu.Coded(3, 2048, 16)
    half = x.half()
    assert torch.equal(half.float(), x)      # the values are fp16
    sr.mx_quant(half, c.q, c.s, c.step, group=16, pre=torch.full((2048,), 2.0 ** power, device=mu.DEV))
    assert c.step.tolist() == [2.0 ** power, 2.0 ** (power - 1), 2.0 ** (power - 3)]
    codes = torch.stack([c.q & 15, c.q >> 4], -1).reshape(3, 128, 16)
    assert bool((codes[:, :126] == even).all()) and bool((codes[:, 126:] == 0).all())
    assert bool((c.s[mu.place(3, 2048, 16)][:, :126] == torch.arange(1, 127, device=mu.DEV)).all())


@pytest.mark.parametrize("codes", [None, "int4", "mx16", "mx32"])
@pytest.mark.parametrize("m,k,post", [(777, 4096, False), (2049, 4096, False), (3001, 4096, True), (1201, 2048, True), (1100, 896, True), (2300, 8192, True), (4099, 1152, False),
                                      (3700, 5120, True), (900, 384, True), (9001, 5632, False)])
def test_many_rows_are_normed_as_few(sr, mu, m, k, post, codes):
    """Calls of many rows, shared out in several ways, against calls of 70 rows of them: the same bits."""
    import torch
    g = mu.gen(m + k)
    y, h = mu.rows(g, m, k, pad=8), mu.rows(g, m, k)
    w = [torch.rand(k, generator=g, device=mu.DEV) + 0.5 for _ in range(3)]
    group = {"mx16": 16, "mx32": 32}.get(codes)

    def call(rows):
        n = rows.stop - rows.start
        out = dict(h_out=torch.empty(n, k, dtype=torch.float16, device=mu.DEV), x_out=torch.empty(n, k, dtype=torch.float16, device=mu.DEV))
        if codes is not None:
            c = mu.Coded(n, k, group or 16)
            out.update(q_out=c.q, scale_out=c.s if group else None, step_out=c.step if codes != "mx32" else None)
        sr.add_norm(y[rows], h[rows], w[0], codes=codes, post_weight=w[1] if post else None, gate=w[2], block_scale=0.5, **out)
        return out

    many = call(slice(0, m))
    for at in (0, 128 * (m // 256), m - 70):
        few = call(slice(at, at + 70))
        for name in ("h_out", "x_out", "q_out", "step_out"):
            if few.get(name) is not None:
                assert torch.equal(many[name][at:at + 70], few[name]), name
        if group:
            assert torch.equal(many["scale_out"][mu.place(m, k, group)[at:at + 70]], few["scale_out"][mu.place(70, k, group)])


def test_arguments_that_do_not_go_together(sr, mu):
    import torch
    x = torch.zeros(4, 256, dtype=torch.float16, device=mu.DEV)
    wide = torch.zeros(4, 512, dtype=torch.float16, device=mu.DEV)
    c, y = mu.Coded(4, 256, 16), torch.empty_like(x)
    before = sr.launch_count()
    for bad in (lambda: sr.add_norm(x, x, x_out=y, q_out=c.q), lambda: sr.add_norm(x, x, x_out=y, step_out=c.step),
                lambda: sr.add_norm(x, x, x_out=y, scale_out=c.s), lambda: sr.mx_quant(x, c.q, c.s, c.step, group=16, walsh=1 << 32),
                lambda: sr.add_norm(x, x, x_out=y, q_out=c.q, step_out=c.step, scale_out=c.s, codes="int4")):
        with pytest.raises(ValueError):
            bad()
    narrow = wide[:, :256]
    h = torch.as_strided(wide, (4, 256), (264, 1))
    for bad in (lambda: sr.add_norm(narrow, x, h_out=h), lambda: sr.add_norm(x, narrow, x_out=h)):
        with pytest.raises(sr.SmoothRotError):
            bad()
    sr.add_norm(narrow[:1], x[:1], h_out=h[:1])
    assert sr.launch_count() == before + 1
