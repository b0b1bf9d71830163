"""Plain 64-bit forms of the microscaled operators and of the norms around a block, and inputs for their tests."""
import math

import torch

DEV = "cuda:0"
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rows(g, m, k, spread=1.0, pad=0, shift=0):
    """fp16 rows, some channels standing out; with `pad` a slice of wider rows, `shift` values into them."""
    x = torch.randn(m, k + pad, generator=g, device=DEV) * spread
    x[:, 5::max(7, k // 6)] *= 10
    return x.half()[:, shift:shift + k]


def place(m, k, group):
    """Offsets of the scales of m rows, [m, k / group], by the formula of the header."""
    r = torch.arange(m, device=DEV)[:, None]
    c = torch.arange(k // group, device=DEV)[None, :]
    return (r // 128 * (k // group // 4) + c // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + c % 4


class Coded:
    """Buffers for coded rows; the scale bytes behind the rows are NaN, which nothing may depend on."""

    def __init__(self, m, k, group):
        self.m, self.k, self.group = m, k, group
        self.q = torch.full((m, k // 2), 0x5a, dtype=torch.uint8, device=DEV)
        bytes_ = (m + 127) // 128 * 128 * (k // group)
        self.s = torch.full((bytes_,), 255 if group == 32 else 127, dtype=torch.uint8, device=DEV)
        self.step = torch.full((m,), float("nan"), device=DEV) if group == 16 else None

    def codes(self):
        """The codes' values in 64 bits, [m, k]."""
        grid = torch.tensor(GRID + [-x for x in GRID], dtype=torch.float64, device=DEV)
        return grid[torch.stack([self.q & 15, self.q >> 4], -1).reshape(self.m, self.k).long()]

    def units(self):
        """What a code of 1 stands for, per group, in 64 bits, [m, k / group]."""
        b = self.s[place(self.m, self.k, self.group)].long()
        if self.group == 32:
            u = torch.exp2(b.double() - 127)
            return torch.where(b == 255, torch.full_like(u, math.nan), u)
        e, f = b >> 3, (b & 7).double()
        u = torch.where(e == 0, f / 512, torch.exp2(e.double() - 7) * (1 + f / 8))
        u = torch.where(b == 127, torch.full_like(u, math.nan), u)
        return u if self.step is None else u * self.step.double()[:, None]

    def values(self):
        return self.codes() * self.units().repeat_interleave(self.group, 1)


def random_coded(g, m, k, group, spread=6):
    """Codes of all kinds under scales over 2^spread and steps of no particular form."""
    c = Coded(m, k, group)
    c.q = torch.randint(0, 256, (m, k // 2), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    low = 127 - spread if group == 32 else 8 * (7 - spread // 2)
    high = 127 if group == 32 else 8 * (7 + spread // 2)
    c.s[place(m, k, group)] = torch.randint(low, high, (m, k // group), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    if group == 16:
        c.step = torch.rand(m, generator=g, device=DEV) + 0.01
    return c


def scale_32(top):
    """2^E with the least E such that top <= 7 * 2^E; 1 for 0."""
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 7))
    e = e + (top > 7 * torch.exp2(e)) - (top <= 7 * torch.exp2(e - 1)).double()
    return torch.where(top == 0, torch.ones_like(top), torch.exp2(e.clamp(min=-127)))


def step_16(top):
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 2688))
    e = e + (top > 2688 * torch.exp2(e)) - (top <= 2688 * torch.exp2(e - 1)).double()
    return torch.where(top == 0, torch.ones_like(top), torch.exp2(e.clamp(min=-100)))


def e4m3(t):
    """The nearest value of 8 bits (1 + 4 + 3), ties to even, at most 448."""
    t = t.clamp(max=448)
    grain = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)
    return torch.round(t / grain) * grain


def nearest(v, unit):
    """The values of codes under `unit` next to v, ties to the even code; 0 where the unit is 0."""
    q = torch.where(unit == 0, torch.zeros_like(v), v / torch.where(unit == 0, torch.ones_like(unit), unit)).abs()
    r = torch.where(q < 2, torch.round(q * 2) / 2, torch.where(q < 4, torch.round(q), torch.round(q / 2) * 2)).clamp(max=6)
    return torch.sign(v) * r * unit


def check_codes(got, v, delta, step=None):
    """Asserts that `got` (a Coded) is what some values within `delta` of v are coded to, v and delta [m, k] in 64 bits.
    `step`: steps that were given ([m] fp32), otherwise those of groups of 16 are checked too."""
    m, k, group = got.m, got.k, got.group
    g = v.reshape(m, -1, group).abs()
    d = delta.reshape(m, -1, group)
    low, high = (g - d).clamp(min=0).amax(2), (g + d).amax(2)
    if group == 32:
        assert bool(((got.units() >= scale_32(low)) | (low == 0)).all()) and bool((got.units() <= scale_32(high)).all() or (high == 0).any())
        bad = (got.units() > scale_32(high)) & (high > 0)
        assert not bool(bad.any())
    else:
        if step is None:
            assert bool((got.step.double() >= step_16(low.amax(1))).all()) and bool((got.step.double() <= step_16(high.amax(1))).all())
        s = got.step.double()[:, None] if step is None else step.double()[:, None]
        scale = got.units() / s if step is None else got.units()
        # the quotient by 6 steps is rounded twice on its way
        assert bool((scale >= e4m3(low / (6 * s) * (1 - 2.0 ** -22))).all()) and bool((scale <= e4m3(high / (6 * s) * (1 + 2.0 ** -22))).all())
    unit = got.units()
    if group == 16 and step is not None:
        unit = unit * step.double()[:, None]
    unit = unit.repeat_interleave(group, 1)
    value = got.codes() * unit
    best = nearest(v, unit)
    off = (value - v).abs() - (best - v).abs()
    assert bool((off <= 2 * delta + 2.0 ** -22 * unit).all()), float((off - 2 * delta).max())


def walsh(x, n):
    """Blocks of n values times the Walsh matrix over sqrt(n)."""
    if not n:
        return x
    i = torch.arange(n, device=DEV)
    bits = i[:, None] & i[None, :]
    sign = torch.ones(n, n, dtype=torch.float64, device=DEV)
    for b in range(n.bit_length()):
        sign = torch.where((bits >> b) & 1 == 1, -sign, sign)
    return (x.reshape(-1, n) @ sign / math.sqrt(n)).reshape(x.shape)


def product(x, w, k):
    """x w^T in 64 bits and a bound on how far fp32 sums of it may be off: an instruction adds 64 products to what it has, each
    such addition, and the few of partial sums, keeps 23 bits of what all magnitudes together come to."""
    return x @ w.T, (k / 64 + 16) * 2.0 ** -23 * (x.abs() @ w.abs().T)


def half_bound(y, extra):
    """Half a step of fp16 at y, and `extra` before the rounding."""
    return 2.0 ** -11 * (y.abs() + extra) + 2.0 ** -25 + extra


def gated(x, gate, up, k):
    """SiLU(x gate^T) * (x up^T) and a bound for fp32: the sums', the exponential's and quotient's few units, and the product's."""
    g, dg = product(x, gate, k)
    u, du = product(x, up, k)
    s = g * torch.sigmoid(g)
    h = s * u
    return h, 1.1 * dg * (u.abs() + du) + s.abs() * du + (8 + 2 * g.abs()) * 2.0 ** -23 * h.abs() + 2.0 ** -120


def rms(x, eps):
    return 1 / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + eps)
