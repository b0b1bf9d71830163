"""The attention block of examples/attention_layer.py: prompts, chunks of prompts and single steps agree."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")


@pytest.fixture(scope="module")
def mod():
    from paper_2506_05413_b200 import build
    build.build()
    spec = importlib.util.spec_from_file_location("attention_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _x(mod, n, seed=3):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return torch.randn(n, mod.HIDDEN, generator=g, device="cuda:0").half()


def _rel(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def test_steps_and_chunks_equal_the_whole_prompt(mod):
    """Every path attends to the same cached 4-bit keys and values.  Between the paths the attention outputs differ by fp16
    roundings (2^-10) and so, after the 4-bit quantizer, by single codes at rounding boundaries: a value moves by a step, 0.3 of the
    spread, for 2^-10 / 0.3 of the values, sqrt(0.003) * 0.3 = 0.02 of the norm; the QKV codes of the fused decode call may move the
    same way."""
    import torch
    n, x = 130, _x(mod, 130)
    whole = mod.AttentionLayer(1, 200)
    want = whole.prompt(x, [n])
    chunks = mod.AttentionLayer(1, 200)
    got = torch.cat([chunks.prompt(x[:50], [50]), chunks.prompt(x[50:120], [70]),
                     *(chunks.step(x[i:i + 1]) for i in range(120, n))])
    torch.cuda.synchronize()
    assert mod.sr.device_status() == 0
    assert int(chunks.lengths[0]) == n and torch.equal(whole.table, chunks.table)
    assert _rel(got[:120], want[:120]) <= 0.05 and _rel(got[120:], want[120:]) <= 0.05


def test_sequences_do_not_touch_each_other(mod):
    import torch
    x = _x(mod, 90)
    both = mod.AttentionLayer(2, 100)
    y = both.prompt(x, [40, 50])
    steps = both.step(x[:2])
    alone = mod.AttentionLayer(2, 100)
    y1 = alone.prompt(x[40:], [0, 50])
    torch.cuda.synchronize()
    assert torch.equal(y[40:], y1)
    assert bool(torch.isfinite(steps).all())


def test_the_block_equals_its_plain_form(mod):
    """The whole block in 64 bits, quantizers and all.  The bound is that of the test above: the 4-bit quantizers on the way turn
    roundings into single codes at rounding boundaries."""
    import math

    import paged_util as pu
    import torch
    n, x = 200, _x(mod, 200)
    layer = mod.AttentionLayer(1, 256)
    got = layer.prompt(x, [n])

    def act(t):                                            # per token, symmetric, clip ratio 0.9
        step = 0.9 * t.abs().amax(1, keepdim=True) / 7
        return (t / step).round().clamp(-8, 7) * step

    def weights(packed):
        codes, step = packed
        c = torch.stack([codes & 15, codes >> 4], -1).flatten(1).double()
        return torch.where(c > 7, c - 16, c) * step.double()[:, None]

    def cached(t):
        code, step, zero = pu.encode(t, mod.CLIP_KV)
        return ((code.reshape(n, -1, 128) - zero[..., None]) * step[..., None]).flatten(1)

    H, kv, D = mod.HEADS, mod.KV_HEADS, mod.DIM
    # what the calls hand to each other is fp16
    qkv = (act(x.double() @ mod.walsh(mod.HIDDEN, x.device).double()) @ weights(layer.qkv).T).half()
    pos = torch.arange(n, device=x.device)
    q = pu.turn(qkv[:, :H * D], D, pos, layer.rotary, False, True).half()
    k = cached(pu.turn(qkv[:, H * D:(H + kv) * D], D, pos, layer.rotary, False, True))
    v = cached(qkv[:, (H + kv) * D:].double())
    y, _ = pu.attend(q, k.half(), v.half(), D, kv, 1 / math.sqrt(D), torch.ones(n, n, dtype=torch.bool, device=x.device).tril())
    y = torch.einsum("nhd,hg->ngd", y.half().double().reshape(n, H, D), mod.walsh(H, x.device).double()).reshape(n, -1)
    want = act(y) @ weights(layer.out).T
    assert _rel(got, want) <= 0.05
