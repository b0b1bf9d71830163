"""What the edge tests of the cache and attention calls share: paged caches, one call of attn_decode, and a bound on the
attention's error that does not grow with the number of keys."""
import math

import torch

import paged_util as pu

DEV, GROUP = pu.DEV, pu.GROUP


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def paged(gen, lengths, kv, D, page, bits, keys=None, values=None, clip=0.95, fill=None):
    """A cache that holds these sequences on shuffled pages -> (cache, table, slots of every sequence).  `keys` and `values`:
    functions of a length that give its rows [n, kv * D]; normal values if None.  Entries of the table past a sequence's pages
    point outside the cache."""
    keys = keys or (lambda n: pu.rows(gen, n, kv * D, outliers=(5, 40)))
    values = values or (lambda n: pu.rows(gen, n, kv * D, 0.7))
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 2
    order = torch.randperm(pages, generator=gen, device=DEV)
    cache = pu.Cache(pages, page, kv, D, bits, fill)
    table = torch.full((len(lengths), max(max(need), 1)), 1 << 30, dtype=torch.int32, device=DEV)
    used, slots = 0, []
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[used:used + need[b]].int()
        used += need[b]
        at = torch.arange(n, device=DEV)
        slots.append(table[b].long()[at // page] * page + at % page)
        if n:
            k, v = keys(n), values(n)
            for part in at.split(1 << 15):
                cache.put(slots[b][part], k[part], v[part], clip)
    return cache, table, slots


def workspace(sr, B, H, kv, D, fill=0):
    return torch.full((max(sr.attn_decode_workspace_bytes(B, H, kv, D), 16),), fill, dtype=torch.uint8, device=DEV)


def decode(sr, q, cache, table, lengths, scale=None, ws=None):
    B, H = q.shape[0], q.shape[1] // cache.D
    y = torch.full((B, H * cache.D), float("nan"), dtype=torch.float16, device=DEV)
    ws = workspace(sr, B, H, cache.kv, cache.D, 255) if ws is None else ws
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    sr.attn_decode(q, cache.k, cache.v, table, n, y, cache.kp, cache.vp, scale=scale, workspace=ws)
    torch.cuda.synchronize()
    return y


def attend(q, k, v, D, kv, scale, seen=None, key_step=None, step=None):
    """One sequence in 64 bits: q [m, H * D], k, v [n, kv * D], seen [m, n] -> (y, bound).  `key_step`, `step` [n, kv]: the 4-bit
    steps of the keys and values.

    The bound, per value, with p the weights relative to the row's largest and A = sum p |v| / sum p:
      2^-11 |y| + 2^-25    the result's rounding to fp16
      2^-11 A              the weights' rounding to fp16: 11 bits of each weight that is normal in fp16.  (With 4-bit values the
                           kernel rounds the weight times the value's step, which is as good.)
      sum min(2^-32, w) |v| / s / sum p     over weights w = p s / max(p s) below fp16's normal range, s the step (1 without steps):
                           the kernels keep the largest w at 2^7 or above, so normal means w >= 2^-21 and the subnormals' last place
                           is 2^-31
      2 ds A               a score is an fp32 sum of D products with the tensor cores' wider alignment: ds = 2^-20 scale sum |q||k|,
                           with 4-bit keys of |q| times what is multiplied, a code with up to 72 added, times the step
      2^-18 A              exponentials and sums in fp32, over at most some thousand terms a lane
    Not counted: with 4-bit values the kernel sums codes less 8, so an output near 0 also carries the last fp32 place of some 8 steps.
    """
    m, n = q.shape[0], k.shape[0]
    H = q.shape[1] // D
    y = torch.zeros(m, H * D, dtype=torch.float64, device=DEV)
    bound = torch.full_like(y, 2.0 ** -25)
    if n == 0 or m == 0:
        return y, bound
    seen = torch.ones(m, n, dtype=torch.bool, device=DEV) if seen is None else seen
    for h in range(H):
        g = h // (H // kv)
        c, hs = slice(g * D, (g + 1) * D), slice(h * D, (h + 1) * D)
        qh, kh, vh = q[:, hs].double(), k[:, c].double(), v[:, c].double()
        s = (qh @ kh.T * scale).masked_fill(~seen, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = p.sum(1, keepdim=True)
        total = torch.where(total == 0, torch.ones_like(total), total)
        y[:, hs] = p @ vh / total
        A = p @ vh.abs() / total
        size = torch.ones(n, dtype=torch.float64, device=DEV) if step is None else step[:, g].double()
        w = p * size
        w = w / w.amax(1, keepdim=True).clamp_min(1e-300)
        # a weight's absolute error, back in units of p: times the largest p s, over s
        small = torch.where(w < 2.0 ** -21, w.clamp_max(2.0 ** -32), torch.zeros_like(w))
        lost = small * (p * size).amax(1, keepdim=True) @ (vh.abs() / size[:, None]) / total
        size_k = qh.abs() @ kh.abs().T
        if key_step is not None:
            size_k = size_k + 72 * qh.abs().sum(1, keepdim=True) * key_step[:, g].double()
        ds = 2.0 ** -20 * abs(scale) * (size_k * seen).amax(1, keepdim=True)
        bound[:, hs] += 2.0 ** -11 * y[:, hs].abs() + (2.0 ** -11 + 2 * ds + 2.0 ** -18) * A + lost
    return y, bound


def off(y, want):
    """How far, relative in the 2-norm."""
    return float((y.double() - want).norm() / want.norm())


def steps(cache, slots):
    """The 4-bit steps of keys and values at these slots, [n, kv]; None with fp16."""
    if cache.bits == 16:
        return None, None
    page, at = slots // cache.page, slots % cache.page
    per = GROUP // cache.D
    return [p[page, :, at, 0].repeat_interleave(per, 1) for p in (cache.kp, cache.vp)]


def check(y, q, cache, slots, scale=None, close=None):
    """Every sequence of a decode call against `attend`; `close`: also in the 2-norm, relative."""
    scale = 1 / math.sqrt(cache.D) if scale is None else scale
    for b, at in enumerate(slots):
        k, v = cache.get(at)
        want, bound = attend(q[b:b + 1], k, v, cache.D, cache.kv, scale, None, *steps(cache, at))
        bad = (y[b:b + 1].double() - want).abs() - bound
        assert bool((bad <= 0).all()), (b, len(at), float(bad.max()), float(want.abs().max()))
        if close is not None and len(at):
            assert off(y[b:b + 1], want) <= close, (b, len(at), off(y[b:b + 1], want))
