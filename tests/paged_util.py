"""Plain 64-bit forms of the cache and attention operators, and inputs for their tests (torch tensors on the GPU)."""
import math

import torch

DEV = "cuda:0"
GROUP = 128


def rows(gen, n, width, spread=1.0, pad=0, outliers=None):
    """n rows of fp16 values; with `pad` they are a slice of wider rows.  `outliers`: these columns of every 64 stand out."""
    x = torch.randn(n, width + pad, generator=gen, device=DEV) * spread
    if outliers:
        for c in outliers:
            x[:, c::64] *= 7
    return x.half()[:, pad // 16 * 8:][:, :width]


def rotary_table(n, D, base=10000.0):
    a = torch.arange(n, device=DEV).double()[:, None] * base ** (-torch.arange(0, D, 2, device=DEV).double() / D)
    return torch.cat([a.cos(), a.sin()], 1).float()


def turn(x, D, positions, table, interleaved, walsh):
    """[T, heads * D] -> rotated, in 64 bits, with the table's own fp32 angles."""
    T = x.shape[0]
    x = x.double().reshape(T, -1, D)
    t = table.double()[positions.long()][:, None, :]
    c, s = t[..., :D // 2], t[..., D // 2:]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        x = torch.stack([a * c - b * s, b * c + a * s], -1).reshape(x.shape)
    else:
        a, b = x[..., :D // 2], x[..., D // 2:]
        x = torch.cat([a * c - b * s, b * c + a * s], -1)
    if walsh:
        i = torch.arange(D, device=DEV)
        bits = (i[:, None] & i[None, :])
        sign = torch.ones(D, D, dtype=torch.float64, device=DEV)
        for b in range(D.bit_length()):
            sign = torch.where((bits >> b) & 1 == 1, -sign, sign)
        x = x @ sign / math.sqrt(D)
    return x.reshape(T, -1)


def encode(x, clip):
    """[T, C] in 64 bits -> codes, step, zero by Eq. 1's asymmetric form (steps in fp32, as the cache holds them)."""
    g = x.reshape(x.shape[0], -1, GROUP)
    clip = float(torch.tensor(clip, dtype=torch.float32))
    hi, lo = clip * g.amax(2), clip * g.amin(2)
    step = torch.where(hi == lo, torch.ones_like(hi), (hi - lo) / 15)
    zero = -torch.round(lo / step)
    code = (torch.round(g / step[..., None]) + zero[..., None]).clamp(0, 15)
    return code.reshape(x.shape), step, zero


class Cache:
    """A paged cache and its plain reading."""

    def __init__(self, pages, page, kv, D, bits, fill=None):
        self.page, self.kv, self.D, self.bits = page, kv, D, bits
        shape = (pages, kv, page, D if bits == 16 else D // 2)
        self.k = torch.zeros(shape, dtype=torch.float16 if bits == 16 else torch.uint8, device=DEV)
        self.v = torch.zeros_like(self.k)
        self.kp = self.vp = None
        if bits == 4:
            self.kp = torch.zeros(pages, kv * D // GROUP, page, 2, device=DEV)
            self.vp = torch.zeros_like(self.kp)
        if fill is not None:
            for t in (self.k, self.v, self.kp, self.vp):
                if t is not None:
                    t.fill_(fill if t.is_floating_point() else 255)

    def tensors(self):
        return self.k, self.v, self.kp, self.vp

    def put(self, slots, k, v, clip=0.95):
        """Rows [T, kv * D] (any float type), coded on the way with 4 bits."""
        page, off = slots // self.page, slots % self.page
        for x, cache, params in ((k, self.k, self.kp), (v, self.v, self.vp)):
            T = x.shape[0]
            if self.bits == 16:
                cache[page, :, off] = x.half().reshape(T, self.kv, self.D)
            else:
                code, step, zero = encode(x.double(), clip)
                code = code.to(torch.uint8)
                cache[page, :, off] = (code[:, 0::2] | (code[:, 1::2] << 4)).reshape(T, self.kv, self.D // 2)
                params[page, :, off] = torch.stack([step, zero], -1).float()

    def codes(self, slots):
        page, off = slots // self.page, slots % self.page
        out = []
        for cache in (self.k, self.v):
            b = cache[page, :, off].flatten(1)
            out.append(torch.stack([b & 15, b >> 4], -1).flatten(1).to(torch.int32))
        return out

    def get(self, slots):
        """Rows at these slots in 64 bits."""
        page, off = slots // self.page, slots % self.page
        out = []
        if self.bits == 16:
            return [c[page, :, off].double().flatten(1) for c in (self.k, self.v)]
        for code, params in zip(self.codes(slots), (self.kp, self.vp)):
            p = params[page, :, off].double()
            g = code.double().reshape(len(slots), self.kv * self.D // GROUP, GROUP)
            out.append(((g - p[..., 1:]) * p[..., :1]).flatten(1))
        return out


def attend(q, k, v, D, kv, scale, seen):
    """One sequence in 64 bits: q [m, H * D], k, v [n, kv * D], seen [m, n] -> (y, bound): softmax attention over what is
    seen, 0 where nothing is, and how far a kernel may be that rounds each weight and the result to fp16 and sums in fp32.

    The bound, per value: 2^-11 |y| for the result, 2 * 2^-11 A for the weights (A = sum p |v| / sum p; the rounding of a weight
    does not enter the sum of the weights, so numerator and denominator each move), n 2^-24 max|v| for
    weights below fp16's normal range, and A times twice the error of a score, which is an fp32 sum of D products:
    2^-20 scale sum |q||k| with the tensor cores' wider alignment counted."""
    m, n = q.shape[0], k.shape[0]
    H = q.shape[1] // D
    y = torch.zeros(m, H * D, dtype=torch.float64, device=DEV)
    bound = torch.full_like(y, 2.0 ** -24)
    if n == 0 or m == 0:
        return y, bound
    some = seen.any(1)
    for h in range(H):
        c = slice((h // (H // kv)) * D, (h // (H // kv) + 1) * D)
        hs = slice(h * D, (h + 1) * D)
        qh, kh, vh = q[:, hs].double(), k[:, c].double(), v[:, c].double()
        s = (qh @ kh.T * scale).masked_fill(~seen, -math.inf)
        p = torch.softmax(s, 1)
        p = torch.where(some[:, None], p, torch.zeros_like(p))
        y[:, hs] = p @ vh
        A = p @ vh.abs()
        ds = 2.0 ** -20 * scale * ((qh.abs() @ kh.abs().T) * seen).amax(1, keepdim=True)
        bound[:, hs] += 2.0 ** -11 * y[:, hs].abs() + 2.0 ** -10 * A + n * 2.0 ** -24 * vh.abs().max() + 2 * ds * A
    return y, bound
