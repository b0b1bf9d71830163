"""Cases of the paged key-value cache and of the attention operators, with the operators' plain forms.

Four operators of one decoder layer between its fused QKV projection and its output projection:

  append   position rotation of queries and keys (and, where `walsh` is set, the Walsh rotation of every head),
           keys and values written to a paged cache, then read back at the same slots
  gather   rows of a paged cache read back as contiguous fp16 keys and values
  decode   attention of one new token per sequence over the paged cache
  prefill  attention over packed prompts, with a prefix of earlier keys where `prefix` is not zero

A cache holds fp16 values (`bits` 16) or asymmetric 4-bit codes in groups of 128 values of a token's row with a step
and a zero point each (`bits` 4).  Cache tensors are [pages, kv heads, page size, head dim (or half of it, two codes
per byte)], step and zero point [pages, groups, page size, 2].  A slot is page * page size + offset.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
GROUP = 128
CLIP = 0.95

# (heads, kv heads, head dim): grouped heads of an 8B decoder layer, its 7B ungrouped form, and other groups and widths
HEADS = [(32, 8, 128), (32, 32, 128), (8, 8, 128), (28, 4, 128), (12, 4, 64), (16, 2, 64), (64, 8, 128)]


def listed():
    return [
        # one new token of one sequence: the smallest call of a decode step
        dict(name="append_token_int4", op="append", heads=32, kv_heads=8, dim=128, bits=4, page=16, tokens=1, walsh=True, pairs=False),
        # one new token of each of 61 sequences, 4-bit keys after the Walsh rotation
        dict(name="append_step61_int4", op="append", heads=32, kv_heads=8, dim=128, bits=4, page=16, tokens=61, walsh=True, pairs=False),
        # a prompt of 2048 tokens into the 4-bit cache
        dict(name="append_prompt2048_int4", op="append", heads=32, kv_heads=8, dim=128, bits=4, page=64, tokens=2048, walsh=False, pairs=False),
        # prompts of 8192 tokens in all, ungrouped heads, fp16 cache, interleaved pairs
        dict(name="append_prompt8192_f16", op="append", heads=32, kv_heads=32, dim=128, bits=16, page=16, tokens=8192, walsh=False, pairs=True),
        # a short prefix with heads of 64, read back for the next chunk of a prompt
        dict(name="gather_777_f16_d64", op="gather", heads=12, kv_heads=4, dim=64, bits=16, page=16, tokens=777),
        # a long 4-bit prefix, read back for the next chunk of a prompt
        dict(name="gather_16384_int4", op="gather", heads=32, kv_heads=8, dim=128, bits=4, page=64, tokens=16384),
        # one sequence in the middle of a short answer: latency
        dict(name="decode_b1_301_int4", op="decode", heads=32, kv_heads=8, dim=128, bits=4, page=16, batch=1, longest=301),
        # a serving batch of very different lengths
        dict(name="decode_b64_4001_int4", op="decode", heads=32, kv_heads=8, dim=128, bits=4, page=16, batch=64, longest=4001),
        # one very long sequence: the length has to be split
        dict(name="decode_b1_131072_int4", op="decode", heads=32, kv_heads=8, dim=128, bits=4, page=64, batch=1, longest=131072),
        # ungrouped heads with an fp16 cache
        dict(name="decode_b16_2048_mha_f16", op="decode", heads=32, kv_heads=32, dim=128, bits=16, page=32, batch=16, longest=2048),
        # short prompts of different lengths in one call, some with an earlier prefix
        dict(name="prefill_b9_2048_prefix", op="prefill", heads=32, kv_heads=8, dim=128, batch=9, tokens=2048, prefix=300, causal=True),
        # one long prompt
        dict(name="prefill_b1_8192", op="prefill", heads=32, kv_heads=8, dim=128, batch=1, tokens=8192, prefix=0, causal=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["append", "gather", "decode", "prefill"])
    h, kv, d = rng.choice(HEADS)
    c = dict(op=op, heads=h, kv_heads=kv, dim=d)
    if op != "prefill":
        c.update(bits=rng.choice([4, 16]), page=rng.choice([8, 16, 32, 64, 128]))
    if op == "append":
        c.update(tokens=_spread(rng, 1, 8192 * 96 // max(96, h + 2 * kv)), walsh=rng.random() < 0.5, pairs=rng.random() < 0.3)
    elif op == "gather":
        c.update(tokens=_spread(rng, 1, 16384 * 8 * 128 // max(8 * 128, kv * d)))
    elif op == "decode":
        c["batch"] = _spread(rng, 1, 128)
        row = 2 * kv * (2 * d if c["bits"] == 16 else d // 2 + d // 16)
        most = min(131072, int(3e8 / row / c["batch"]))
        c["longest"] = _spread(rng, 1, max(2, most))
    else:
        c["batch"] = _spread(rng, 1, 24)
        most = int(8192 * math.sqrt(32 * 128 / max(32 * 128, h * d)))
        c["tokens"] = _spread(rng, c["batch"], most)
        c["prefix"] = 0 if rng.random() < 0.6 else _spread(rng, 1, max(1, (8192 - c["tokens"]) // c["batch"] // 2 + 1))
        c["causal"] = rng.random() < 0.85
        if not c["causal"]:
            c["tokens"] = max(c["batch"], c["tokens"] // 2)
    return c


# ---- the lengths of a case: the same for every seed ----

def _lengths(case):
    """decode: the sequences' lengths, the first the longest, the last 0 in larger batches.
    prefill: (new tokens, earlier keys) of every sequence."""
    rng = random.Random("%s %s %s" % (case["op"], case["batch"], case.get("longest", case.get("tokens"))))
    b = case["batch"]
    if case["op"] == "decode":
        n = [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(b - 1)]
        if b >= 8:
            n[-1], n[-2] = 0, 1
        return n
    cuts = sorted(rng.sample(range(1, case["tokens"]), b - 1)) if b > 1 else []
    news = [y - x for x, y in zip([0] + cuts, cuts + [case["tokens"]])]
    return news, [rng.randint(0, case["prefix"]) if case["prefix"] else 0 for _ in news]


def _visible(case):
    """Pairs of a query and a key that a prefill case looks at, per head."""
    pairs = 0
    for n, p in zip(*_lengths(case)):
        pairs += n * p + (n * (n + 1) // 2 if case["causal"] else n * n)
    return pairs


def work(case):
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "prefill":
        news, olds = _lengths(case)
        keys = sum(news) + sum(olds)
        return {"bytes": 2 * d * (2 * h * sum(news) + 2 * kv * keys), "flops": 4 * d * h * _visible(case)}
    row = 2 * kv * d * 2 if case["bits"] == 16 else 2 * kv * (d // 2) + 2 * (kv * d // GROUP) * 8
    if case["op"] == "decode":
        n = sum(_lengths(case))
        return {"bytes": n * row + 2 * case["batch"] * h * d * 2, "flops": 4 * n * h * d}
    t = case["tokens"]
    if case["op"] == "gather":
        return {"bytes": t * (row + 2 * kv * d * 2 + 8), "flops": t * 2 * kv * d * 2}
    flops = t * (h + kv) * d * (3 + (d.bit_length() if case["walsh"] else 0)) + (t * 2 * kv * d * 8 if case["bits"] == 4 else 0)
    # q, k, v in; q and the cache's rows out; the rows in again and their values out; angles, positions, slots
    return {"bytes": t * (2 * d * (h + 2 * kv) + 2 * d * h + 2 * row + 2 * kv * d * 2 + 4 * d + 20), "flops": flops}


# ---- inputs ----

def _rows(gen, n, heads, d, spread=1.0, outliers=False):
    """n rows of heads * d values; keys have two channels of every head that stand out, as trained keys do."""
    x = torch.randn(n, heads, d, generator=gen, device=DEVICE) * spread
    if outliers:
        x[:, :, 5] *= 8
        x[:, :, d // 2 + 9] *= 6
    return x.reshape(n, heads * d).half()


def _encode(x, clip=CLIP):
    """[n, C] in 32 bits -> codes [n, C] uint8, step and zero point [n, C / 128]."""
    g = x.reshape(x.shape[0], -1, GROUP)
    hi, lo = g.amax(2) * clip, g.amin(2) * clip
    step = torch.where(hi == lo, torch.ones_like(hi), (hi - lo) / torch.full_like(hi, 15))
    zero = -torch.round(lo / step)
    inverse = 1 / step
    code = (torch.round(g * inverse[:, :, None]) + zero[:, :, None]).clamp(0, 15)
    return code.reshape(x.shape).to(torch.uint8), step, zero


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpack(byte):
    return torch.stack([byte & 15, byte >> 4], -1).flatten(-2)


def _store(s, slots, k, v):
    """Rows of keys and values in 32 bits into the cache."""
    page, offset = slots // s["page"], slots % s["page"]
    for x, cache, params in ((k, s["k_cache"], s["k_params"]), (v, s["v_cache"], s["v_params"])):
        shape = (x.shape[0], s["kv_heads"], -1)
        if s["bits"] == 16:
            cache[page, :, offset] = x.reshape(shape).half()
        else:
            code, step, zero = _encode(x)
            cache[page, :, offset] = _pack(code).reshape(shape)
            params[page, :, offset] = torch.stack([step, zero], -1)


def _load(s, slots):
    """Rows of keys and values of the cache in 32 bits, [n, kv heads * dim]."""
    page, offset = slots // s["page"], slots % s["page"]
    got = []
    for cache, params in ((s["k_cache"], s["k_params"]), (s["v_cache"], s["v_params"])):
        x = cache[page, :, offset]
        if s["bits"] == 16:
            got.append(x.float().reshape(x.shape[0], -1))
        else:
            sz = params[page, :, offset]
            g = _unpack(x).float().reshape(x.shape[0], -1, GROUP)
            got.append(((g - sz[:, :, 1:]) * sz[:, :, :1]).reshape(x.shape[0], -1))
    return got


def _empty_cache(s, pages):
    kv, d, page = s["kv_heads"], s["dim"], s["page"]
    shape = (pages, kv, page, d if s["bits"] == 16 else d // 2)
    kind = torch.float16 if s["bits"] == 16 else torch.uint8
    for name in ("k", "v"):
        s[name + "_cache"] = torch.zeros(shape, dtype=kind, device=DEVICE)
        s[name + "_params"] = torch.ones(pages, kv * d // GROUP, page, 2, device=DEVICE) if s["bits"] == 4 else None


def _fill(s, gen, slots):
    for at in slots.split(1 << 15):
        k = _rows(gen, len(at), s["kv_heads"], s["dim"], 1.0, True).float()
        v = _rows(gen, len(at), s["kv_heads"], s["dim"], 0.5).float()
        _store(s, at, k, v)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = {k: v for k, v in case.items() if k != "name"}
    h, kv, d = s["heads"], s["kv_heads"], s["dim"]
    half = dict(dtype=torch.float16, device=DEVICE)
    if s["op"] == "prefill":
        news, olds = _lengths(case)
        ends = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=DEVICE)  # noqa: E731
        keys = sum(news) + sum(olds)
        s["cu_q"], s["cu_k"] = ends(news), ends([n + p for n, p in zip(news, olds)])
        s["q"] = _rows(gen, sum(news), h, d)
        # keys and values lie side by side, as the projection leaves them
        kv_rows = torch.cat([_rows(gen, keys, kv, d, 1.0, True), _rows(gen, keys, kv, d, 0.5)], 1)
        s["k"], s["v"] = kv_rows[:, :kv * d], kv_rows[:, kv * d:]
        s["y"] = torch.empty(sum(news), h * d, **half)
        return s
    if s["op"] == "decode":
        lengths, page = _lengths(case), s["page"]
        wide = -(-max(lengths) // page)
        pages = sum(-(-n // page) for n in lengths) + 3
        order = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32)
        _empty_cache(s, pages)
        table = torch.zeros(len(lengths), wide, dtype=torch.int32, device=DEVICE)
        used, slots = 0, []
        for b, n in enumerate(lengths):
            m = -(-n // page)
            table[b, :m] = order[used:used + m]
            used += m
            at = torch.arange(n, device=DEVICE)
            slots.append(table[b].long()[at // page] * page + at % page)
        _fill(s, gen, torch.cat(slots))
        s["table"] = table
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)
        # queries after the position rotation, row by row; the scratch is the caller's, used again from call to call
        s["q"] = _rows(gen, len(lengths), h, d)
        s["y"] = torch.empty(len(lengths), h * d, **half)
        s["scratch"] = torch.empty(16 << 20, dtype=torch.uint8, device=DEVICE)
        return s
    t, page = s["tokens"], s["page"]
    pages = -(-t // page) + 5
    _empty_cache(s, pages)
    order = torch.randperm(pages, generator=gen, device=DEVICE)
    at = torch.arange(t, device=DEVICE)
    s["slots"] = order[at // page] * page + at % page
    if s["op"] == "append" and t <= 256:  # a decode step: each token goes to a page of another sequence
        s["slots"] = torch.randperm(pages * page, generator=gen, device=DEVICE)[:t]
    s["k_back"], s["v_back"] = torch.empty(t, kv * d, **half), torch.empty(t, kv * d, **half)
    if s["op"] == "gather":
        _fill(s, gen, s["slots"])
        return s
    # one fused projection's output; the queries, keys and values are slices of its rows
    qkv = torch.cat([_rows(gen, t, h, d), _rows(gen, t, kv, d, 1.0, True), _rows(gen, t, kv, d, 0.5)], 1)
    s["q"], s["k"], s["v"] = qkv[:, :h * d], qkv[:, h * d:(h + kv) * d], qkv[:, (h + kv) * d:]
    s["q_out"] = torch.empty(t, h * d, **half)
    rows = max(t, 4096)
    s["positions"] = (at if t > 256 else torch.randint(0, rows, (t,), generator=gen, device=DEVICE)).to(torch.int32)
    angle = torch.arange(rows, device=DEVICE).double()[:, None] * 500000.0 ** (-torch.arange(0, d, 2, device=DEVICE).double() / d)
    s["rotary"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    return s


# ---- the plain forms ----

def _turn(x, s, heads):
    """Position rotation of [t, heads * dim] in 32 bits, then the Walsh rotation of each head where the case asks for it."""
    t, d = x.shape[0], s["dim"]
    table = s["rotary"][s["positions"].long()][:, None, :]
    c, w = table[..., :d // 2], table[..., d // 2:]
    x = x.reshape(t, heads, d)
    if s["pairs"]:
        a, b = x[..., 0::2], x[..., 1::2]
        x = torch.stack([a * c - b * w, b * c + a * w], -1).flatten(-2)
    else:
        a, b = x[..., :d // 2], x[..., d // 2:]
        x = torch.cat([a * c - b * w, b * c + a * w], -1)
    if s["walsh"]:
        stride = 1
        while stride < d:  # log2(dim) butterflies
            p = x.reshape(t, heads, d // (2 * stride), 2, stride)
            x = torch.stack([p[..., 0, :] + p[..., 1, :], p[..., 0, :] - p[..., 1, :]], -2).reshape(t, heads, d)
            stride *= 2
        x = x * (1.0 / math.sqrt(d))
    return x.reshape(t, heads * d)


def _attend(q, k, v, seen, d):
    """q [.., g, m, d], k and v [.., n, d] in 32 bits, seen [.., m, n]: softmax(q k / sqrt(d)) v over what is seen; nothing seen: zero."""
    m = q.shape[-2]
    score = torch.matmul(q.flatten(-3, -2), k.transpose(-1, -2)).unflatten(-2, (-1, m)).mul_(1.0 / math.sqrt(d))
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = score.sum(-1, keepdim=True)
    y = torch.matmul(score.flatten(-3, -2), v).unflatten(-2, (-1, m))
    return torch.where(total > 0, y / total, torch.zeros_like(y))


def _plain(s):
    h, kv, d = s["heads"], s["kv_heads"], s["dim"]
    if s["op"] == "append":
        q, k = _turn(s["q"].float(), s, h), _turn(s["k"].float(), s, kv)
        _store(s, s["slots"], k, s["v"].float())
        k, v = _load(s, s["slots"])
        return {"q": q.half(), "k": k.half(), "v": v.half()}
    if s["op"] == "gather":
        k, v = _load(s, s["slots"])
        return {"k": k.half(), "v": v.half()}
    if s["op"] == "decode":
        b, wide = s["table"].shape
        at = torch.arange(wide * s["page"], device=DEVICE)
        slots = s["table"].long()[:, at // s["page"]] * s["page"] + at % s["page"]
        seen = at < s["lengths"][:, None]
        k, v = (x.reshape(b, -1, kv, d).transpose(1, 2) for x in _load(s, slots.reshape(-1)))
        # places past a sequence's end hold another sequence's rows: they take no part
        v = v.masked_fill(~seen[:, None, :, None], 0)
        q = s["q"].float().reshape(b, kv, h // kv, 1, d)
        return _attend(q, k, v, seen[:, None, None, None, :], d).reshape(b, h * d).half()
    t, n = s["q"].shape[0], s["k"].shape[0]
    i, j = torch.arange(t, device=DEVICE), torch.arange(n, device=DEVICE)
    si, sj = torch.bucketize(i, s["cu_q"][1:], right=True), torch.bucketize(j, s["cu_k"][1:], right=True)
    seen = si[:, None] == sj
    if s["causal"]:
        seen &= (j - s["cu_k"][1:][sj]) <= (i - s["cu_q"][1:][si])[:, None]
    q = s["q"].float().reshape(t, kv, h // kv, d).permute(1, 2, 0, 3)
    k, v = (s[x].float().reshape(n, kv, d).transpose(0, 1) for x in ("k", "v"))
    return _attend(q, k, v, seen, d).permute(2, 0, 1, 3).reshape(t, h * d).half()


# ---- the framework's operators ----

def _own(s):
    from paper_2506_05413_b200 import binding as sr
    if s["op"] == "append":
        sr.kv_append(s["q"], s["k"], s["v"], s["positions"], s["rotary"], s["slots"], s["k_cache"], s["v_cache"],
                     s["k_params"], s["v_params"], q_out=s["q_out"], clip=CLIP, walsh=s["walsh"], interleaved=s["pairs"])
        sr.kv_gather(s["slots"], s["k_cache"], s["v_cache"], s["k_back"], s["v_back"], s["k_params"], s["v_params"])
        return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}
    if s["op"] == "gather":
        sr.kv_gather(s["slots"], s["k_cache"], s["v_cache"], s["k_back"], s["v_back"], s["k_params"], s["v_params"])
        return {"k": s["k_back"], "v": s["v_back"]}
    if s["op"] == "decode":
        sr.attn_decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["y"], s["k_params"], s["v_params"],
                       workspace=s["scratch"])
        return s["y"]
    sr.attn_prefill(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["y"], head_dim=s["dim"], causal=s["causal"])
    return s["y"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits ----

def _exact_code(x):
    """Rows in 64 bits -> the values that 4-bit codes of them stand for."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[1], GROUP):
        g = x[:, a:a + GROUP]
        hi, lo = CLIP * g.max(1, keepdim=True).values, CLIP * g.min(1, keepdim=True).values
        step = (hi - lo) / 15
        step[step == 0] = 1
        zero = -(lo / step).round()
        out[:, a:a + GROUP] = (((g / step).round() + zero).clamp(0, 15) - zero) * step
    return out


def _exact_turn(x, s, heads):
    d = s["dim"]
    place = s["positions"].double()
    freq = 500000.0 ** (-torch.arange(0, d, 2, device=DEVICE).double() / d)
    spin = torch.polar(torch.ones(1, dtype=torch.float64, device=DEVICE), place[:, None] * freq)[:, None, :]
    x = x.double().reshape(-1, heads, d)
    z = torch.complex(x[..., 0::2], x[..., 1::2]) if s["pairs"] else torch.complex(x[..., :d // 2], x[..., d // 2:])
    z = z * spin
    x = torch.view_as_real(z).flatten(-2) if s["pairs"] else torch.cat([z.real, z.imag], -1)
    if s["walsh"]:
        w = torch.ones(1, 1, dtype=torch.float64, device=DEVICE)
        two = torch.tensor([[1.0, 1.0], [1.0, -1.0]], dtype=torch.float64, device=DEVICE)
        while w.shape[0] < d:
            w = torch.kron(w, two)
        x = x @ w / math.sqrt(d)
    return x.reshape(-1, heads * d)


def _exact_rows(s, slots):
    """The cache's rows at these slots, in 64 bits."""
    got = []
    for name in ("k", "v"):
        cache = s[name + "_cache"].transpose(1, 2).reshape(-1, s["kv_heads"], s[name + "_cache"].shape[-1])[slots]
        if s["bits"] == 16:
            got.append(cache.double().flatten(1))
            continue
        byte = cache.flatten(1).to(torch.int32)
        code = torch.empty(len(slots), 2 * byte.shape[1], dtype=torch.float64, device=DEVICE)
        code[:, 0::2], code[:, 1::2] = (byte % 16).double(), (byte // 16).double()
        params = s[name + "_params"].transpose(1, 2).reshape(-1, s[name + "_params"].shape[1], 2)[slots].double()
        step, zero = params[..., 0].repeat_interleave(GROUP, 1), params[..., 1].repeat_interleave(GROUP, 1)
        got.append((code - zero) * step)
    return got


def _exact_heads(q, k, v, s, y, seen=None):
    """Attention of one sequence in 64 bits, one key-value head after another, into y."""
    h, kv, d = s["heads"], s["kv_heads"], s["dim"]
    if not len(q) or not len(k):
        return
    g = h // kv
    for a in range(h):
        c = a // g
        p = (q[:, a * d:(a + 1) * d].double() @ k[:, c * d:(c + 1) * d].double().T) / math.sqrt(d)
        if seen is not None:
            p = p.masked_fill(~seen, -math.inf)
        y[:, a * d:(a + 1) * d] = torch.softmax(p, 1) @ v[:, c * d:(c + 1) * d].double()


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "append":
        k, v = _exact_turn(s["k"], s, s["kv_heads"]), s["v"].double()
        if s["bits"] == 4:
            k, v = _exact_code(k), _exact_code(v)
        return {"q": _exact_turn(s["q"], s, s["heads"]), "k": k, "v": v}
    if s["op"] == "gather":
        k, v = _exact_rows(s, s["slots"])
        return {"k": k, "v": v}
    y = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    if s["op"] == "decode":
        for b, n in enumerate(s["lengths"].tolist()):
            at = torch.arange(n, device=DEVICE)
            k, v = _exact_rows(s, s["table"][b].long()[at // s["page"]] * s["page"] + at % s["page"])
            _exact_heads(s["q"][b:b + 1], k, v, s, y[b:b + 1])
        return y
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(len(cq) - 1):
        nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        seen = torch.ones(nq, nk, dtype=torch.bool, device=DEVICE)
        if s["causal"]:
            seen = seen.tril(nk - nq)
        _exact_heads(s["q"][cq[b]:cq[b + 1]], s["k"][ck[b]:ck[b + 1]], s["v"][ck[b]:ck[b + 1]], s, y[cq[b]:cq[b + 1]], seen)
    return y
