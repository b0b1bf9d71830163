"""Cases of the microscaled 4-bit floating-point operators and of the norms around a block, with their plain forms.

Operators of the feed-forward half of one decoder layer:

  quant   rows of fp16 values into 4-bit floating-point codes with a scale per group of 32 (a power of two) or of 16 (an
          8-bit float, over a power of two per row), where `walsh` is set after a Walsh rotation in blocks, then read back
  linear  the product of coded tokens and coded weights
  norm    residual stream plus gated, scaled (and where `post` is set, normalised) block output, then the norm of the sum
          as fp16 values or as codes that are read back
  glu     both projections of a gated feed-forward block, its activation and product, fp16 output
  ffn     quant, then both projections, activation and product into codes, then the down projection

A code is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign in bit 3, two to a byte along the row, the even one in the low
half.  Scales of 128 rows and 4 groups lie in 512 bytes: row r and group g at (r % 32) * 16 + (r % 128 // 32) * 4 + g % 4.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5

# (width, inner width) of feed-forward blocks: an 8B layer's, smaller and odd ones
BLOCKS = [(4096, 14336), (4096, 11008), (2048, 5632), (2048, 8192), (1024, 2816), (5120, 13824), (896, 4864)]
# output channels of projections: fused query-key-value, output, grouped keys and values, odd multiples of 8
CHANNELS = [6144, 4096, 1024, 512, 5120, 2056, 1288, 14336]


def listed():
    return [
        # one new token before a rotated projection: latency
        dict(name="quant_token_g32", op="quant", rows=1, width=4096, group=32, walsh=32, pre=False),
        # a ragged prompt at the down projection's width, smoothed and rotated
        dict(name="quant_611x14336_g32_w128", op="quant", rows=611, width=14336, group=32, walsh=128, pre=True),
        # prompts of 8192 tokens in all
        dict(name="quant_8192x4096_g16", op="quant", rows=8192, width=4096, group=16, walsh=0, pre=False),
        # output projection of one new token
        dict(name="linear_token_g32", op="linear", rows=1, channels=4096, width=4096, group=32),
        # fused query-key-value projection of a serving batch
        dict(name="linear_61x6144_g16", op="linear", rows=61, channels=6144, width=4096, group=16),
        # down projection of a prompt
        dict(name="linear_2048_down_g32", op="linear", rows=2048, channels=4096, width=14336, group=32),
        # one new token between two blocks, into codes
        dict(name="norm_token_g32", op="norm", rows=1, width=4096, post=False, gate=False, out=32),
        # prompts of 8192 tokens, norms before and after the block, a gate per channel
        dict(name="norm_8192_sandwich_g32", op="norm", rows=8192, width=4096, post=True, gate=True, out=32),
        # a ragged prompt through a small block's projections
        dict(name="glu_333x5632_g16", op="glu", rows=333, width=2048, inner=5632, group=16),
        # a prompt of 2048 tokens, values kept in fp16
        dict(name="glu_2048x14336_g32", op="glu", rows=2048, width=4096, inner=14336, group=32),
        # the whole block for one new token
        dict(name="ffn_token_g32", op="ffn", rows=1, width=4096, inner=14336, group=32, walsh=32),
        # the whole block for prompts of 8192 tokens
        dict(name="ffn_8192_g32", op="ffn", rows=8192, width=4096, inner=14336, group=32, walsh=32),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["quant", "linear", "norm", "glu", "ffn"])
    width, inner = rng.choice(BLOCKS)
    if op == "quant":
        width = rng.choice([width, inner])
        return dict(op=op, rows=_spread(rng, 1, 8192 * 4096 // max(width, 4096)), width=width, group=rng.choice([16, 32]), walsh=rng.choice([0, 32, 64, 128]),
                    pre=rng.random() < 0.4)
    if op == "norm":
        return dict(op=op, rows=_spread(rng, 1, 8192 * 4096 // max(width, 4096)), width=width, post=rng.random() < 0.5, gate=rng.random() < 0.5,
                    out=rng.choice([0, 16, 32]))
    rows = _spread(rng, 1, 8192 * 4096 // max(width, 4096))
    if op == "linear":
        channels = rng.choice(CHANNELS)
        if rng.random() < 0.3:  # a down projection
            width, channels = inner, width
        return dict(op=op, rows=rows, channels=channels, width=width, group=rng.choice([16, 32]))
    c = dict(op=op, rows=rows, width=width, inner=inner, group=rng.choice([16, 32]))
    if op == "ffn":
        c["walsh"] = rng.choice([0, 32])
    return c


def _coded(rows, width, group):
    """Bytes of coded rows: codes, scales and, with groups of 16, steps."""
    return rows * (width // 2 + width // group + (4 if group == 16 else 0))


def work(case):
    m, k = case["rows"], case["width"]
    if case["op"] == "quant":
        g = case["group"]
        flops = m * k * (4 + (case["walsh"].bit_length() if case["walsh"] else 0))
        return {"bytes": 2 * m * k + 2 * _coded(m, k, g) + 2 * m * k + (4 * k if case["pre"] else 0), "flops": flops}
    if case["op"] == "norm":
        g = case["out"]
        weights = 4 * k * (1 + case["post"] + case["gate"])
        return {"bytes": 6 * m * k + (2 * m * k if not g else 2 * _coded(m, k, g) + 2 * m * k) + weights, "flops": m * k * (12 if case["post"] else 8)}
    g = case["group"]
    if case["op"] == "linear":
        n = case["channels"]
        return {"bytes": _coded(m + n, k, g) + 2 * m * n, "flops": 2 * m * n * k}
    f = case["inner"]
    if case["op"] == "glu":
        return {"bytes": _coded(m + 2 * f, k, g) + 2 * m * f, "flops": 4 * m * f * k}
    return {"bytes": 2 * m * k + 2 * _coded(m, k, g) + _coded(2 * f, k, g) + 2 * _coded(m, f, g) + _coded(k, f, g) + 2 * m * k, "flops": 6 * m * f * k}


# ---- codes ----

def _round(q):
    """The nearest of the values of a code, ties to the even code, at most 6."""
    a = q.abs()
    r = torch.where(a < 2, torch.round(a * 2) * 0.5, torch.where(a < 4, torch.round(a), torch.round(a * 0.5) * 2))
    return torch.copysign(r.clamp(max=6.0), q)


def _scales(v, group, step=None):
    """[m, k] in 32 bits -> scales [m, k / group, 1] (32: a power of two; 16: of 8 bits, over the row's step), steps [m, 1]."""
    g = v.reshape(v.shape[0], -1, group)
    top = g.abs().amax(2, keepdim=True)
    if group == 32:
        part, e = torch.frexp(top)  # part in [0.5, 1)
        e = (e - 3 + (part > 0.875)).clamp(-127, 127)
        return torch.where(top == 0, torch.ones_like(top), torch.ldexp(torch.ones_like(top), e)), None
    if step is None:
        part, e = torch.frexp(top.amax(1))
        e = (e - 12 + (part > 0.65625)).clamp(min=-100)  # 2688 is 0.65625 * 2^12
        step = torch.where(part == 0, torch.ones_like(part), torch.ldexp(torch.ones_like(part), e))
    unit = step[:, :, None] * 6
    return (top / unit).clamp(max=448).to(torch.float8_e4m3fn).float(), step


def _encode(v, group, step=None):
    """[m, k] in 32 bits -> the codes' values [m, k / group, group], scales [m, k / group, 1], steps [m, 1] or None."""
    g = v.reshape(v.shape[0], -1, group)
    scale, step = _scales(v, group, step)
    unit = scale if step is None else scale * step[:, :, None]
    return _round(torch.where(unit == 0, torch.zeros_like(g), g / unit)), scale, step


def _values(code, scale, step):
    """What codes stand for, in 32 bits, [m, k]."""
    return (code * (scale if step is None else scale * step[:, :, None])).flatten(1)


def _place(m, groups):
    """Where the scales of m rows lie, [m, groups]."""
    r, g = torch.arange(m, device=DEVICE)[:, None], torch.arange(groups, device=DEVICE)
    return (r // 128 * (groups // 4) + g // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + g % 4


def _pack(x, group):
    """Values in 32 bits -> bytes of codes, bytes of scales as they lie, steps."""
    code, scale, step = _encode(x, group)
    m, groups = code.shape[:2]
    order = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEVICE)
    nibble = torch.bucketize(code.abs(), order) | (torch.signbit(code).long() << 3)
    nibble = nibble.to(torch.uint8).flatten(1)
    s = torch.zeros((m + 127) // 128 * 128 * groups, dtype=torch.uint8, device=DEVICE)
    byte = (torch.log2(scale) + 127).to(torch.uint8) if group == 32 else scale.to(torch.float8_e4m3fn).view(torch.uint8)
    s[_place(m, groups)] = byte[:, :, 0]
    return dict(q=nibble[:, 0::2] | (nibble[:, 1::2] << 4), s=s, step=None if step is None else step[:, 0].contiguous(), group=group)


def _unpack(t):
    """Coded rows -> values in 32 bits, [m, k]."""
    q, group = t["q"], t["group"]
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEVICE)
    code = value[torch.stack([q & 15, q >> 4], -1).flatten(1).int()].reshape(q.shape[0], -1, group)
    byte = t["s"][_place(q.shape[0], code.shape[1])]
    scale = torch.ldexp(torch.ones(byte.shape, device=DEVICE), byte.int() - 127) if group == 32 else byte.view(torch.float8_e4m3fn).float()
    return _values(code, scale[:, :, None], None if t["step"] is None else t["step"][:, None])


def _walsh(x, n):
    """Blocks of n values times the Walsh matrix over sqrt(n), in 32 bits."""
    if not n:
        return x
    stride = 1
    while stride < n:
        p = x.reshape(x.shape[0], -1, 2, stride)
        x = torch.stack([p[:, :, 0] + p[:, :, 1], p[:, :, 0] - p[:, :, 1]], 2).reshape(x.shape)
        stride *= 2
    return x * torch.tensor(1.0 / math.sqrt(n), device=DEVICE)


# ---- inputs ----

def _tokens(gen, m, k):
    """Hidden states: a few channels stand out."""
    x = torch.randn(m, k, generator=gen, device=DEVICE)
    x[:, 7::max(8, k // 5)] *= 12
    return x.half()


def _weights(gen, n, k, group):
    return _pack((torch.randn(n, k, generator=gen, device=DEVICE) * (1.0 / math.sqrt(k))).half().float(), group)


def _room(m, k, group):
    """Memory for coded rows."""
    s = torch.zeros((m + 127) // 128 * 128 * (k // group), dtype=torch.uint8, device=DEVICE)
    return dict(q=torch.empty(m, k // 2, dtype=torch.uint8, device=DEVICE), s=s, step=torch.empty(m, device=DEVICE) if group == 16 else None, group=group)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = {k: v for k, v in case.items() if k != "name"}
    m, k = s["rows"], s["width"]
    half = dict(dtype=torch.float16, device=DEVICE)
    if s["op"] == "quant":
        s["x"] = _tokens(gen, m, k)
        s["pre"] = torch.exp(torch.randn(k, generator=gen, device=DEVICE) * 0.5) if s["pre"] else None
        s["codes"], s["back"] = _room(m, k, s["group"]), torch.empty(m, k, **half)
        return s
    if s["op"] == "norm":
        s["h"] = _tokens(gen, m, k)
        s["y"] = torch.randn(m, k, generator=gen, device=DEVICE).half()
        for name, on in (("w_post", s["post"]), ("gates", s["gate"]), ("w_pre", True)):
            s[name] = 1 + 0.2 * torch.randn(k, generator=gen, device=DEVICE) if on else None
        s["h_out"], s["x"] = torch.empty(m, k, **half), torch.empty(m, k, **half)
        s["codes"] = _room(m, k, s["out"]) if s["out"] else None
        return s
    g = s["group"]
    if s["op"] == "linear":
        s["x"], s["w"] = _pack(_tokens(gen, m, k).float(), g), _weights(gen, s["channels"], k, g)
        s["out"] = torch.empty(m, s["channels"], **half)
    else:
        f = s["inner"]
        s["gate"], s["up"] = _weights(gen, f, k, g), _weights(gen, f, k, g)
        if s["op"] == "glu":
            s["x"], s["out"] = _pack(_tokens(gen, m, k).float(), g), torch.empty(m, f, **half)
        else:
            s["x"], s["down"], s["out"] = _tokens(gen, m, k), _weights(gen, k, f, g), torch.empty(m, k, **half)
            s["codes"], s["inner_codes"] = _room(m, k, g), _room(m, f, g)
            if g == 16:  # the steps of the inner values are calibrated beforehand
                s["inner_codes"]["step"].fill_(2.0 ** -6)
    return s


# ---- the plain forms ----

def _product(x, w):
    return torch.matmul(x, w.T)


def _gated(x, s):
    a = _product(x, _unpack(s["gate"]))
    return a / (1 + torch.exp(-a)) * _product(x, _unpack(s["up"]))


def _rms(x):
    """1 / root of the mean square, the sum in 64 bits, rounded to 32."""
    return (x.double().square().mean(1, keepdim=True) + EPS).rsqrt().float()


def _plain(s):
    if s["op"] == "quant":
        v = s["x"].float()
        v = _walsh(v if s["pre"] is None else v * s["pre"], s["walsh"])
        return _values(*_encode(v, s["group"])).half()
    if s["op"] == "norm":
        y = s["y"].float()
        if s["w_post"] is not None:
            y = y * _rms(y) * s["w_post"]
        if s["gates"] is not None:
            y = y * s["gates"]
        h = (s["h"].float() + y * 0.5).half()
        x = (h.float() * _rms(h.float()) * s["w_pre"]).half()
        if s["codes"] is not None:
            x = _values(*_encode(x.float(), s["out"])).half()
        return {"h": h, "x": x}
    if s["op"] == "linear":
        return _product(_unpack(s["x"]), _unpack(s["w"])).half()
    if s["op"] == "glu":
        return _gated(_unpack(s["x"]), s).half()
    h = _walsh(_gated(_values(*_encode(s["x"].float(), s["group"])), s), s["walsh"])
    step = s["inner_codes"]["step"]
    h = _values(*_encode(h, s["group"], None if step is None else step[:, None]))
    return _product(h, _unpack(s["down"])).half()


# ---- the framework's operators ----

def _own(s):
    from paper_2506_05413_b200 import binding as sr
    if s["op"] == "quant":
        c = s["codes"]
        sr.mx_quant(s["x"], c["q"], c["s"], c["step"], group=s["group"], pre=s["pre"], walsh=s["walsh"])
        sr.mx_dequant(c["q"], c["s"], c["step"], s["back"], group=s["group"])
        return s["back"]
    if s["op"] == "norm":
        c = s["codes"]
        if c is None:
            sr.add_norm(s["y"], s["h"], s["w_pre"], h_out=s["h_out"], x_out=s["x"], post_weight=s["w_post"], gate=s["gates"], block_scale=0.5, eps=EPS)
        else:
            sr.add_norm(s["y"], s["h"], s["w_pre"], h_out=s["h_out"], q_out=c["q"], scale_out=c["s"], step_out=c["step"], codes="mx%d" % s["out"],
                        post_weight=s["w_post"], gate=s["gates"], block_scale=0.5, eps=EPS)
            sr.mx_dequant(c["q"], c["s"], c["step"], s["x"], group=s["out"])
        return {"h": s["h_out"], "x": s["x"]}
    if s["op"] == "linear":
        x, w = s["x"], s["w"]
        sr.mx_linear(x["q"], x["s"], w["q"], w["s"], s["out"], group=s["group"], x_step=x["step"], w_step=w["step"])
        return s["out"]
    a, b = s["gate"], s["up"]
    if s["op"] == "glu":
        x = s["x"]
        sr.mx_glu(x["q"], x["s"], a["q"], a["s"], b["q"], b["s"], group=s["group"], x_step=x["step"], gate_step=a["step"], up_step=b["step"],
                  h_out=s["out"])
        return s["out"]
    c, h, w = s["codes"], s["inner_codes"], s["down"]
    sr.mx_quant(s["x"], c["q"], c["s"], c["step"], group=s["group"])
    sr.mx_glu(c["q"], c["s"], a["q"], a["s"], b["q"], b["s"], group=s["group"], x_step=c["step"], gate_step=a["step"], up_step=b["step"],
              q_out=h["q"], scale_out=h["s"], h_step=h["step"], walsh=s["walsh"])
    sr.mx_linear(h["q"], h["s"], w["q"], w["s"], s["out"], group=s["group"], x_step=h["step"], w_step=w["step"])
    return s["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits ----

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_nearest(q):
    """|q| in 64 bits -> the nearest value of a code, by the borders between them; a border belongs to the even code."""
    out = torch.zeros_like(q)
    for i in range(1, 8):
        border = (GRID[i - 1] + GRID[i]) / 2
        out = torch.where(q >= border if i % 2 == 0 else q > border, torch.full_like(q, GRID[i]), out)
    return out


def _exact_coded(x, group, step=None):
    """Rows in 64 bits -> the values that their codes stand for."""
    out = torch.empty_like(x)
    if group == 16 and step is None:
        most = x.abs().amax(1, keepdim=True)
        step = torch.where(most == 0, torch.ones_like(most), torch.exp2(torch.ceil(torch.log2((most / 2688).clamp(min=2.0 ** -100)))))
    for a in range(0, x.shape[1], group):
        v = x[:, a:a + group]
        most = v.abs().amax(1, keepdim=True)
        if group == 32:
            unit = torch.exp2(torch.ceil(torch.log2((most / 7).clamp(min=2.0 ** -120))))
        else:
            t = (most / (6 * step)).clamp(max=448)
            # 8 bits: steps of 1/8 of the power of two below, of 2^-9 at the least
            grain = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)
            unit = torch.round(t / grain) * grain * step
        safe = torch.where(unit == 0, torch.ones_like(unit), unit)
        out[:, a:a + group] = torch.sign(v) * _exact_nearest(v.abs() / safe) * unit
    return out


def _exact_values(t):
    """Coded rows in 64 bits, byte by byte from their places."""
    q, group = t["q"].long(), t["group"]
    m, k = q.shape[0], 2 * q.shape[1]
    code = torch.empty(m, k, dtype=torch.float64, device=DEVICE)
    for half in (0, 1):
        n = q // 16 if half else q % 16
        e, f = n // 2 % 4, n % 2
        code[:, half::2] = torch.where(e == 0, 0.5 * f, torch.exp2(e.double() - 1) * (1 + 0.5 * f)) * (1 - 2 * (n // 8))
    tiles = t["s"].reshape(-1, k // group // 4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, k // group)[:m].long()
    if group == 32:
        scale = torch.exp2(tiles.double() - 127)
    else:
        e, f = tiles // 8, (tiles % 8).double()
        scale = torch.where(e == 0, f / 512, torch.exp2(e.double() - 7) * (1 + f / 8)) * t["step"].double()[:, None]
    return code * scale.repeat_interleave(group, 1)


def _exact_walsh(x, n):
    if not n:
        return x
    w = torch.ones(1, 1, dtype=torch.float64, device=DEVICE)
    two = torch.tensor([[1.0, 1.0], [1.0, -1.0]], dtype=torch.float64, device=DEVICE)
    while w.shape[0] < n:
        w = torch.kron(w, two)
    return (x.reshape(-1, n) @ w).reshape(x.shape) / math.sqrt(n)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "quant":
        x = s["x"].double()
        return _exact_coded(_exact_walsh(x if s["pre"] is None else x * s["pre"].double(), s["walsh"]), s["group"])
    if s["op"] == "norm":
        y = s["y"].double()
        if s["w_post"] is not None:
            y = y / torch.sqrt((y * y).sum(1, keepdim=True) / y.shape[1] + EPS) * s["w_post"].double()
        if s["gates"] is not None:
            y = y * s["gates"].double()
        h = s["h"].double() + 0.5 * y
        kept = h.half().double()  # the norm is that of the stream as it is held
        x = kept / torch.sqrt((kept * kept).sum(1, keepdim=True) / kept.shape[1] + EPS) * s["w_pre"].double()
        return {"h": h, "x": x if s["codes"] is None else _exact_coded(x.half().double(), s["out"])}
    if s["op"] == "linear":
        return _exact_values(s["x"]) @ _exact_values(s["w"]).T
    x = _exact_values(s["x"]) if s["op"] == "glu" else _exact_coded(s["x"].double(), s["group"])
    a = x @ _exact_values(s["gate"]).T
    h = a * torch.sigmoid(a) * (x @ _exact_values(s["up"]).T)
    if s["op"] == "glu":
        return h
    step = s["inner_codes"]["step"]
    h = _exact_coded(_exact_walsh(h, s["walsh"]), s["group"], None if step is None else step.double()[:, None])
    return h @ _exact_values(s["down"]).T
