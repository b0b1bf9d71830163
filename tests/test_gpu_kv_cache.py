"""kv_append and kv_gather against plain 64-bit forms: rotations, cache layout, codes, odd sizes, refusals."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    from paper_2506_05413_b200 import build, binding
    build.build()
    binding.load()
    return binding


@pytest.fixture(scope="module")
def pu():
    import paged_util
    return paged_util


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return g


# T, heads, kv heads, D, page size, bits, walsh, interleaved
CASES = [
    (1, 32, 8, 128, 16, 4, False, False),
    (1, 32, 8, 128, 1, 16, True, False),
    (5, 8, 8, 128, 8, 4, True, True),
    (37, 28, 4, 128, 64, 4, False, True),
    (37, 12, 4, 64, 16, 4, False, False),
    (65, 16, 2, 64, 128, 4, True, False),
    (3, 5, 1, 64, 4, 16, True, True),          # odd numbers of heads of 64: the last unit is half full
    (130, 7, 7, 64, 32, 16, False, False),
    (611, 32, 32, 128, 16, 16, True, False),
    (1300, 4, 2, 128, 1024, 4, False, False),  # more tokens than one block each keeps resident
    (9, 0, 8, 128, 16, 4, False, False),       # keys and values alone
]


@pytest.mark.parametrize("T,H,kv,D,page,bits,walsh,inter", CASES)
def test_append_matches_the_plain_form(sr, pu, T, H, kv, D, page, bits, walsh, inter):
    import torch
    gen = _gen(T + D)
    q = pu.rows(gen, T, H * D, pad=64) if H else None
    k = pu.rows(gen, T, kv * D, pad=32, outliers=(5, 40))
    v = pu.rows(gen, T, kv * D, 0.5, pad=128)
    pages = -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=gen, device=pu.DEV)[:T]
    positions = torch.randint(0, 5000, (T,), generator=gen, device=pu.DEV, dtype=torch.int32)
    table = pu.rotary_table(5000, D)
    cache = pu.Cache(pages, page, kv, D, bits)
    before = [None if t is None else t.clone() for t in cache.tensors()]
    q_out = torch.full((T, H * D + 16), float("nan"), dtype=torch.float16, device=pu.DEV)[:, 8:8 + H * D] if H else None
    k_out = torch.full((T, kv * D), float("nan"), dtype=torch.float16, device=pu.DEV)
    sr.kv_append(q, k, v, positions, table, slots, *cache.tensors(), q_out=q_out, k_out=k_out, clip=0.95, walsh=walsh,
                 interleaved=inter)
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    want_k = pu.turn(k, D, positions, table, inter, walsh)
    # fp16 rounding of the result (2^-11 relative, 2^-24 at the smallest); in fp32 before it three roundings of the
    # pair, and with the Walsh rotation one more per stage and the norm, each relative to the head's largest sum
    for got, x in ((q_out, q), (k_out, k)):
        if got is None:
            continue
        want = pu.turn(x, D, positions, table, inter, walsh)
        size = x.double().reshape(T, -1, D).abs().sum(2).repeat_interleave(D, 1)
        bound = 2.0 ** -11 * want.abs() + 2.0 ** -24 + 12 * 2.0 ** -24 * size
        assert bool(((got.double() - want).abs() <= bound).all())
    if bits == 16:
        kc, vc = cache.get(slots)
        assert torch.equal(kc, k_out.double()) and torch.equal(vc, v.double())
    else:
        # values: the very codes, steps and zero points of the row quantizer
        qv = torch.empty(T, kv * D // 2, dtype=torch.uint8, device=pu.DEV)
        st, ze = (torch.empty(T, kv * D // 128, device=pu.DEV) for _ in range(2))
        sr.kv_quant(v.contiguous(), 0.95, qv, st, ze)
        p, o = slots // page, slots % page
        assert torch.equal(cache.v[p, :, o].flatten(1), qv)
        assert torch.equal(cache.vp[p, :, o][..., 0], st) and torch.equal(cache.vp[p, :, o][..., 1], ze)
        # keys: coded from the fp32 values after the rotation; a code may move by one at a rounding boundary
        code, step, zero = pu.encode(want_k, 0.95)
        got = cache.codes(slots)[0].double()
        params = cache.kp[p, :, o].double()
        assert float(((params[..., 0] - step).abs() / step).max()) <= 4e-6
        dz = (params[..., 1] - zero).abs()
        assert float(dz.max()) <= 1 and float((dz != 0).double().mean()) <= max(1e-3, 1.5 / dz.numel())
        diff = (got - code).abs().reshape(T, -1, 128)[dz == 0]
        assert float(diff.max()) <= 1 and float((diff != 0).double().mean()) <= max(1e-4, 1.5 / diff.numel())
    # nothing else of the cache is touched
    rest = torch.ones(pages * page, dtype=torch.bool, device=pu.DEV)
    rest[slots] = False
    rest = rest.nonzero()[:, 0]
    for t, b in zip(cache.tensors(), before):
        if t is not None:
            assert torch.equal(t[rest // page, :, rest % page], b[rest // page, :, rest % page])


@pytest.mark.parametrize("T,H,kv,D,page,bits,walsh,inter", [c for c in CASES if c[0] > 1 and c[1]][:6])
def test_append_in_place_equals_append_into_other_buffers(sr, pu, T, H, kv, D, page, bits, walsh, inter):
    import torch
    gen = _gen(3)
    q, k, v = pu.rows(gen, T, H * D), pu.rows(gen, T, kv * D), pu.rows(gen, T, kv * D)
    slots = torch.arange(T, device=pu.DEV)
    pos = torch.arange(T, dtype=torch.int32, device=pu.DEV)
    table = pu.rotary_table(T, D)
    a, b = (pu.Cache(-(-T // page), page, kv, D, bits) for _ in range(2))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    sr.kv_append(q, k, v, pos, table, slots, *a.tensors(), q_out=qo, k_out=ko, walsh=walsh, interleaved=inter)
    sr.kv_append(q, k, v, pos, table, slots, *b.tensors(), q_out=q, k_out=k, walsh=walsh, interleaved=inter)
    torch.cuda.synchronize()
    assert torch.equal(q, qo) and torch.equal(k, ko)
    for x, y in zip(a.tensors(), b.tensors()):
        assert x is None or torch.equal(x, y)


@pytest.mark.parametrize("T,kv,D,page,bits", [(1, 8, 128, 16, 4), (77, 8, 128, 16, 16), (130, 4, 64, 8, 4), (33, 5, 64, 1, 16),
                                              (4099, 2, 128, 256, 4), (4099, 32, 128, 64, 16)])
def test_gather_matches_the_plain_form(sr, pu, T, kv, D, page, bits):
    import torch
    gen = _gen(T)
    pages = -(-T // page) + 1
    cache = pu.Cache(pages, page, kv, D, bits)
    slots = torch.randperm(pages * page, generator=gen, device=pu.DEV)[:T]
    cache.put(slots, pu.rows(gen, T, kv * D, 2.0), pu.rows(gen, T, kv * D) + 3)
    if T > 3:
        slots[2] = -1
    out = torch.full((T, 2 * kv * D + 24), float("nan"), dtype=torch.float16, device=pu.DEV)
    ko, vo = out[:, :kv * D], out[:, kv * D + 8:2 * kv * D + 8]
    sr.kv_gather(slots, cache.k, cache.v, ko, vo, cache.kp, cache.vp)
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    for got, want in zip((ko, vo), cache.get(slots.clamp_min(0))):
        want[slots < 0] = 0
        # (code - zero) is a whole number below 2^24, exact; one rounding in fp32, one to fp16
        assert bool(((got.double() - want).abs() <= (2.0 ** -11 + 2.0 ** -23) * want.abs() + 2.0 ** -24).all())
    assert torch.isnan(out[:, kv * D:kv * D + 8]).all() and torch.isnan(out[:, 2 * kv * D + 8:]).all()


@pytest.mark.parametrize("D,kv,inter", [(128, 8, False), (128, 8, True), (64, 16, False)])
def test_append_rounds_every_product(sr, pu, D, kv, inter):
    """Enough values that some lie at rounding boundaries: the rotation equals separate fp32 operations bit for bit, and the
    codes those of the row quantizer."""
    import torch
    T = 4096
    gen = _gen(6)
    q, k, v = pu.rows(gen, T, 8 * D), pu.rows(gen, T, kv * D, outliers=(5, 40)), pu.rows(gen, T, kv * D, 0.5)
    pos = torch.arange(T, dtype=torch.int32, device=pu.DEV)
    table = pu.rotary_table(T, D)
    slots = torch.randperm(T, generator=gen, device=pu.DEV)
    cache = pu.Cache(T // 64, 64, kv, D, 4)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    sr.kv_append(q, k, v, pos, table, slots, *cache.tensors(), q_out=qo, k_out=ko, interleaved=inter)
    torch.cuda.synchronize()
    c, s = table[:, None, :D // 2], table[:, None, D // 2:]
    for got, x in ((qo, q), (ko, k)):
        x = x.float().reshape(T, -1, D)
        a, b = (x[..., 0::2], x[..., 1::2]) if inter else (x[..., :D // 2], x[..., D // 2:])
        ac, bs, bc, as_ = a * c, b * s, b * c, a * s          # each rounded by itself
        one, two = ac - bs, bc + as_
        want = torch.stack([one, two], -1).flatten(-2) if inter else torch.cat([one, two], -1)
        assert torch.equal(got, want.reshape(T, -1).half())
    qv = torch.empty(T, kv * D // 2, dtype=torch.uint8, device=pu.DEV)
    st, ze = (torch.empty(T, kv * D // 128, device=pu.DEV) for _ in range(2))
    sr.kv_quant(v, 0.95, qv, st, ze)
    p, o = slots // 64, slots % 64
    assert torch.equal(cache.v[p, :, o].flatten(1), qv)
    assert torch.equal(cache.vp[p, :, o][..., 0], st) and torch.equal(cache.vp[p, :, o][..., 1], ze)


def test_constant_and_far_off_groups(sr, pu):
    """Groups whose values are all equal, and groups far from zero (a zero point far outside 0..15)."""
    import torch
    T, kv, D = 3, 2, 128
    k = torch.zeros(T, kv * D, dtype=torch.float16, device=pu.DEV)
    v = torch.zeros_like(k)
    v[0] = 3.0
    v[1, :D] = 1000 + torch.arange(D, device=pu.DEV).half() * 0.5
    v[2, D:] = -500 + (torch.arange(D, device=pu.DEV) % 3).half()
    cache = pu.Cache(1, 16, kv, D, 4)
    slots = torch.arange(T, device=pu.DEV)
    pos = torch.zeros(T, dtype=torch.int32, device=pu.DEV)
    sr.kv_append(None, k, v, pos, pu.rotary_table(1, D), slots, *cache.tensors(), clip=1.0)
    qv = torch.empty(T, kv * D // 2, dtype=torch.uint8, device=pu.DEV)
    st, ze = (torch.empty(T, kv, device=pu.DEV) for _ in range(2))
    sr.kv_quant(v, 1.0, qv, st, ze)
    torch.cuda.synchronize()
    assert torch.equal(cache.v[0, :, :T].transpose(0, 1).flatten(1), qv)
    assert torch.equal(cache.vp[0, :, :T, 0].T, st) and torch.equal(cache.vp[0, :, :T, 1].T, ze)
    assert float(ze[1, 0]) < -100
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    sr.kv_gather(slots, cache.k, cache.v, ko, vo, cache.kp, cache.vp)
    torch.cuda.synchronize()
    assert torch.equal(ko, k) and torch.equal(vo[0], v[0])


def test_slots_and_positions_out_of_range_are_left_out_and_reported(sr, pu):
    import torch
    T, kv, D, page, pages = 6, 2, 128, 16, 2
    gen = _gen(1)
    q, k, v = pu.rows(gen, T, 4 * D), pu.rows(gen, T, kv * D), pu.rows(gen, T, kv * D)
    cache = pu.Cache(pages, page, kv, D, 16, fill=7.0)
    slots = torch.tensor([0, pages * page, -1, 3, 4, 1 << 40], device=pu.DEV)
    pos = torch.tensor([1, 1, 1, -1, 9, 2], dtype=torch.int32, device=pu.DEV)
    qo = torch.full_like(q, 5.0)
    sr.device_status()
    sr.kv_append(q, k, v, pos, pu.rotary_table(9, D), slots, *cache.tensors(), q_out=qo)
    torch.cuda.synchronize()
    assert sr.device_status() == 32 and sr.device_status() == 0
    written = [bool((qo[i] != 5.0).any()) for i in range(T)]
    assert written == [True, False, True, False, False, False]      # a negative slot is rotated, not cached
    touched = (cache.k != 7.0).any(3).any(1).flatten().nonzero()[:, 0].tolist()
    assert touched == [0]
    ko, vo = torch.full_like(k, 5.0), torch.full_like(v, 5.0)
    sr.kv_gather(slots, cache.k, cache.v, ko, vo)
    torch.cuda.synchronize()
    assert sr.device_status() == 33
    assert torch.equal(vo[0], v[0]) and float(ko[[1, 2, 5]].abs().max()) == 0.0 and float(ko[3].float().mean()) == 7.0


def test_offsets_beyond_32_bits(sr, pu):
    """A cache of more than 2^31 values (and 2^32 bytes) per tensor: its last slots."""
    import torch
    kv, D, page = 8, 128, 64
    pages = (1 << 31) // (kv * D * page) + 2
    cache = pu.Cache(pages, page, kv, D, 16)
    T = 5
    gen = _gen(2)
    k, v = pu.rows(gen, T, kv * D), pu.rows(gen, T, kv * D)
    slots = torch.tensor([0, pages * page - 1, pages * page - 2, (pages - 1) * page, 77], device=pu.DEV)
    pos = torch.zeros(T, dtype=torch.int32, device=pu.DEV)
    ko, vo, kr = torch.empty_like(k), torch.empty_like(v), torch.empty_like(k)
    sr.kv_append(None, k, v, pos, pu.rotary_table(1, D), slots, *cache.tensors(), k_out=kr)
    sr.kv_gather(slots, cache.k, cache.v, ko, vo)
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    assert torch.equal(vo, v) and torch.equal(ko, kr)
    assert torch.equal(cache.v[-1, :, -1].flatten(), v[1]) and int((cache.v != 0).any(3).any(1).sum()) == T


def test_another_stream(sr, pu):
    import torch
    T, kv, D = 64, 8, 128
    gen = _gen(4)
    k, v = pu.rows(gen, T, kv * D), pu.rows(gen, T, kv * D)
    cache = pu.Cache(4, 16, kv, D, 16)
    slots = torch.arange(T, device=pu.DEV)
    pos = torch.arange(T, dtype=torch.int32, device=pu.DEV)
    table = pu.rotary_table(T, D)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sr.kv_append(None, k, v, pos, table, slots, *cache.tensors())
        sr.kv_gather(slots, cache.k, cache.v, ko, vo)
    side.synchronize()
    assert torch.equal(vo, v)


def test_empty_calls_launch_nothing(sr, pu):
    import torch
    kv, D = 2, 128
    cache = pu.Cache(1, 16, kv, D, 4)
    none = torch.empty(0, kv * D, dtype=torch.float16, device=pu.DEV)
    n = sr.launch_count()
    sr.kv_append(None, none, none, torch.empty(0, dtype=torch.int32, device=pu.DEV), pu.rotary_table(1, D),
                 torch.empty(0, dtype=torch.int64, device=pu.DEV), *cache.tensors())
    sr.kv_gather(torch.empty(0, dtype=torch.int64, device=pu.DEV), cache.k, cache.v, none, none, cache.kp, cache.vp)
    assert sr.launch_count() == n


def test_refusals_of_the_binding(sr, pu):
    import torch
    T, kv, D = 2, 2, 128
    gen = _gen(5)
    k, v = pu.rows(gen, T, kv * D), pu.rows(gen, T, kv * D)
    cache = pu.Cache(1, 16, kv, D, 4)
    slots = torch.arange(T, device=pu.DEV)
    pos = torch.zeros(T, dtype=torch.int32, device=pu.DEV)
    table = pu.rotary_table(4, D)
    bad = [
        (ValueError, dict(k=k[:, :128])),                       # half the heads
        (TypeError, dict(k=k.float())),
        (ValueError, dict(k=k.T.contiguous().T)),               # columns contiguous
        (ValueError, dict(v=v[:1])),
        (TypeError, dict(slots=slots.int())),
        (TypeError, dict(positions=pos.long())),
        (ValueError, dict(rotary=table[:, :64])),
        (ValueError, dict(k_params=None)),
        (ValueError, dict(v_params=cache.vp[..., :1])),
        (ValueError, dict(q=k, q_out=None)),
        (ValueError, dict(v_cache=cache.v[:, :1])),
        (TypeError, dict(k=k.cpu())),
        (sr.SmoothRotError, dict(clip=0.0)),
        (sr.SmoothRotError, dict(clip=1.5)),
    ]
    base = dict(q=None, k=k, v=v, positions=pos, rotary=table, slots=slots, k_cache=cache.k, v_cache=cache.v,
                k_params=cache.kp, v_params=cache.vp)
    n = sr.launch_count()
    for kind, change in bad:
        with pytest.raises(kind):
            sr.kv_append(**{**base, **change})
    odd = torch.empty(2 * kv * D + 1, dtype=torch.float16, device=pu.DEV)[1:].reshape(2, kv * D)
    with pytest.raises(sr.SmoothRotError) as err:
        sr.kv_append(**{**base, "k": odd})
    assert err.value.status == -3
    wide = pu.Cache(1, 12, kv, D, 4)                            # pages of 12
    with pytest.raises(sr.SmoothRotError) as err:
        sr.kv_gather(slots, wide.k, wide.v, k, v, wide.kp, wide.vp)
    assert err.value.status == -1
    assert sr.launch_count() == n
