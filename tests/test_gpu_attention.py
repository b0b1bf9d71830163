"""attn_decode and attn_prefill against plain 64-bit attention: lengths from 0, pages that end anywhere, grouped heads,
both caches, masks that leave rows empty, what lies in masked places, strides, streams, refusals."""
import math

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


def _paged(pu, gen, lengths, kv, D, page, bits, spread=1.0, shift=0.0, fill=None):
    """A cache with these sequences on shuffled pages; the table's unused entries point outside the cache."""
    import torch
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 2
    order = torch.randperm(pages, generator=gen, device=pu.DEV)
    cache = pu.Cache(pages, page, kv, D, bits, fill)
    table = torch.full((len(lengths), max(max(need), 1)), 1 << 30, dtype=torch.int32, device=pu.DEV)
    used, slots = 0, []
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[used:used + need[b]].int()
        used += need[b]
        at = torch.arange(n, device=pu.DEV)
        slots.append(table[b].long()[at // page] * page + at % page)
        if n:
            cache.put(slots[b], pu.rows(gen, n, kv * D, spread, outliers=(5, 40)), pu.rows(gen, n, kv * D, 0.7) + shift)
    return cache, table, slots


def _decode(sr, pu, q, cache, table, lengths, H, scale=None):
    import torch
    B = len(lengths)
    y = torch.full((B, H * cache.D + 8), float("nan"), dtype=torch.float16, device=pu.DEV)[:, :H * cache.D]
    ws = torch.full((max(sr.attn_decode_workspace_bytes(B, H, cache.kv, cache.D), 16),), 255, dtype=torch.uint8, device=pu.DEV)
    sr.attn_decode(q, cache.k, cache.v, table, torch.tensor(lengths, dtype=torch.int32, device=pu.DEV), y, cache.kp, cache.vp,
                   scale=scale, workspace=ws)
    torch.cuda.synchronize()
    return y


def _check_decode(pu, y, q, cache, slots, lengths, scale):
    import torch
    for b, n in enumerate(lengths):
        k, v = cache.get(slots[b])
        want, bound = pu.attend(q[b:b + 1], k, v, cache.D, cache.kv, scale, torch.ones(1, n, dtype=torch.bool, device=pu.DEV))
        bad = (y[b:b + 1].double() - want).abs() - bound
        assert bool((bad <= 0).all()), (b, n, float(bad.max()), float(want.abs().max()))


DECODE = [
    # lengths, H, kv, D, page, bits
    ([1], 32, 8, 128, 16, 4),
    ([1], 32, 8, 128, 16, 16),
    ([0], 4, 2, 128, 16, 4),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], 8, 2, 128, 16, 4),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], 8, 2, 128, 16, 16),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], 8, 4, 64, 8, 4),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], 9, 3, 64, 8, 16),
    ([301], 32, 8, 128, 16, 4),
    ([9001], 32, 8, 128, 64, 4),
    ([9001, 3], 8, 8, 128, 64, 16),
    ([20000], 4, 1, 128, 256, 4),
    ([700, 0, 5, 2500, 1, 999], 32, 32, 128, 32, 16),
    ([700, 0, 5, 2500, 1, 999], 28, 4, 128, 128, 4),      # groups of 7
    ([77, 513], 12, 1, 64, 1, 16),                       # pages of one token, a group of 12
    ([77, 513], 40, 2, 128, 1024, 4),                    # a group of 20
    ([77, 513, 40], 71, 1, 64, 16, 16),                  # one key head for 71
    ([300 + 7 * i for i in range(67)], 16, 2, 64, 16, 4),
    ([64] * 300, 8, 8, 128, 16, 4),
    ([3000] + [0] * 200 + [4000], 8, 2, 128, 16, 4),
]


@pytest.mark.parametrize("lengths,H,kv,D,page,bits", DECODE)
def test_decode_matches_the_plain_form(sr, pu, lengths, H, kv, D, page, bits):
    gen = _gen(len(lengths) + H)
    cache, table, slots = _paged(pu, gen, lengths, kv, D, page, bits)
    q = pu.rows(gen, len(lengths), H * D, pad=64)
    y = _decode(sr, pu, q, cache, table, lengths, H)
    assert sr.device_status() == 0
    _check_decode(pu, y, q, cache, slots, lengths, 1 / math.sqrt(D))
    again = _decode(sr, pu, q, cache, table, lengths, H)
    import torch
    assert torch.equal(y, again)                         # a fixed order of sums


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("spread,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.1), (4.0, 1.5)])
def test_decode_scores_of_any_size(sr, pu, bits, spread, scale):
    gen = _gen(8)
    lengths = [1500, 40]
    cache, table, slots = _paged(pu, gen, lengths, 2, 128, 16, bits, spread)
    q = pu.rows(gen, 2, 8 * 128)
    y = _decode(sr, pu, q, cache, table, lengths, 8, scale)
    _check_decode(pu, y, q, cache, slots, lengths, 1 / math.sqrt(128) if scale is None else scale)


@pytest.mark.parametrize("size", [3e-5, 1e-3, 2000.0])
def test_decode_of_small_and_large_values(sr, pu, size):
    """4-bit steps from below 1e-5 to some hundreds, and zero points far from 0..15."""
    import torch
    gen = _gen(9)
    lengths = [333]
    cache, table, slots = _paged(pu, gen, lengths, 2, 128, 16, 4)
    at = slots[0]
    cache.put(at, pu.rows(gen, 333, 256), pu.rows(gen, 333, 256).float() * size + size * 20)
    q = pu.rows(gen, 1, 8 * 128)
    y = _decode(sr, pu, q, cache, table, lengths, 8)
    _check_decode(pu, y, q, cache, slots, lengths, 1 / math.sqrt(128))


@pytest.mark.parametrize("bits", [4, 16])
def test_decode_ignores_what_lies_past_a_sequence(sr, pu, bits):
    """Unused places of the pages hold NaN (values, steps and zero points), unused table entries are out of range."""
    import torch
    gen = _gen(10)
    lengths = [1, 7, 16, 50, 129, 0]
    cache, table, slots = _paged(pu, gen, lengths, 2, 128, 64, bits, fill=float("nan"))
    q = pu.rows(gen, len(lengths), 8 * 128)
    y = _decode(sr, pu, q, cache, table, lengths, 8)
    assert sr.device_status() == 0 and bool(torch.isfinite(y).all())
    _check_decode(pu, y, q, cache, slots, lengths, 1 / math.sqrt(128))


def test_decode_values_that_are_not_finite_reach_their_own_sequence_only(sr, pu):
    import torch
    gen = _gen(11)
    lengths = [40, 40, 40]
    cache, table, slots = _paged(pu, gen, lengths, 2, 128, 16, 16)
    s = int(slots[1][7])
    cache.v[s // 16, 0, s % 16, 3] = float("inf")
    q = pu.rows(gen, 3, 4 * 128)
    y = _decode(sr, pu, q, cache, table, lengths, 4)
    bad = ~torch.isfinite(y)
    assert bad.nonzero().tolist() == [[1, 3], [1, 131]]   # both query heads of key head 0, value 3
    assert float(y[1, 3]) == math.inf


def test_decode_lengths_and_pages_out_of_range_are_reported(sr, pu):
    import torch
    gen = _gen(12)
    cache, table, slots = _paged(pu, gen, [64, 64], 2, 128, 16, 16)
    q = pu.rows(gen, 2, 4 * 128)
    whole = _decode(sr, pu, q, cache, table, [64, 64], 4)
    sr.device_status()
    y = _decode(sr, pu, q, cache, table, [1000, -5], 4)   # clamped to the table's width, and to nothing
    assert sr.device_status() == 34
    assert torch.equal(y[0], whole[0]) and float(y[1].abs().max()) == 0.0
    table[0, 1] = -1                                      # tokens 16..31 are left out
    table[1, 3] = cache.k.shape[0]
    y = _decode(sr, pu, q, cache, table, [64, 64], 4)
    assert sr.device_status() == 34
    for b, gone in ((0, range(16, 32)), (1, range(48, 64))):
        k, v = cache.get(torch.stack([slots[b][j] for j in range(64) if j not in gone]))
        want, bound = pu.attend(q[b:b + 1], k, v, 128, 2, 1 / math.sqrt(128), torch.ones(1, 48, dtype=torch.bool, device=pu.DEV))
        assert bool(((y[b:b + 1].double() - want).abs() <= bound).all())


def test_decode_far_end_of_a_cache_beyond_32_bits(sr, pu):
    import torch
    kv, D, page = 8, 128, 64
    pages = (1 << 31) // (kv * D * page) + 2
    cache = pu.Cache(pages, page, kv, D, 16)
    n = 2 * page - 3
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device=pu.DEV)
    gen = _gen(13)
    at = torch.arange(n, device=pu.DEV)
    slots = table[0].long()[at // page] * page + at % page
    cache.put(slots, pu.rows(gen, n, kv * D), pu.rows(gen, n, kv * D))
    q = pu.rows(gen, 1, kv * D)
    y = _decode(sr, pu, q, cache, table, [n], kv)
    assert sr.device_status() == 0
    _check_decode(pu, y, q, cache, [slots], [n], 1 / math.sqrt(D))


def test_decode_on_another_stream_and_in_a_graph(sr, pu):
    import torch
    gen = _gen(14)
    lengths = [5000, 17]
    cache, table, slots = _paged(pu, gen, lengths, 2, 128, 16, 4)
    q = pu.rows(gen, 2, 8 * 128)
    want = _decode(sr, pu, q, cache, table, lengths, 8)
    n = torch.tensor(lengths, dtype=torch.int32, device=pu.DEV)
    y = torch.zeros(2, 8 * 128, dtype=torch.float16, device=pu.DEV)
    ws = torch.empty(max(sr.attn_decode_workspace_bytes(2, 8, 2, 128), 16), dtype=torch.uint8, device=pu.DEV)
    call = lambda: sr.attn_decode(q, cache.k, cache.v, table, n, y, cache.kp, cache.vp, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        y.zero_()
        ws.fill_(171)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    n.copy_(torch.tensor([900, 0], dtype=torch.int32))     # the same graph with other lengths
    graph.replay()
    torch.cuda.synchronize()
    _check_decode(pu, y, q, cache, [slots[0][:900], slots[1][:0]], [900, 0], 1 / math.sqrt(128))


def test_decode_refusals(sr, pu):
    import torch
    gen = _gen(15)
    cache, table, _ = _paged(pu, gen, [20, 30], 2, 128, 16, 4)
    q = pu.rows(gen, 2, 4 * 128)
    y = torch.empty(2, 4 * 128, dtype=torch.float16, device=pu.DEV)
    n = torch.tensor([20, 30], dtype=torch.int32, device=pu.DEV)
    need = sr.attn_decode_workspace_bytes(2, 4, 2, 128)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=pu.DEV)
    base = dict(q=q, k_cache=cache.k, v_cache=cache.v, block_table=table, lengths=n, Y=y, k_params=cache.kp,
                v_params=cache.vp, workspace=ws)
    before = sr.launch_count()
    bad = [
        (TypeError, dict(q=q.float())), (TypeError, dict(lengths=n.long())), (TypeError, dict(block_table=table.long())),
        (ValueError, dict(lengths=n[:1])), (ValueError, dict(block_table=table[:1])), (ValueError, dict(Y=y[:, :256])),
        (ValueError, dict(q=q[:, :200], Y=y[:, :200])), (ValueError, dict(k_params=None)),
        (TypeError, dict(k_cache=cache.k.float(), v_cache=cache.v.float())),
        (sr.SmoothRotError, dict(scale=float("nan"))),
        (sr.SmoothRotError, dict(q=pu.rows(gen, 2, 3 * 128), Y=torch.empty(2, 3 * 128, dtype=torch.float16, device=pu.DEV))),
    ]
    for kind, change in bad:
        with pytest.raises(kind):
            sr.attn_decode(**{**base, **change})
    if need:
        with pytest.raises(sr.SmoothRotError) as err:
            sr.attn_decode(**{**base, "workspace": ws[:need - 1]})
        assert err.value.status == -4
    assert sr.launch_count() == before
    sr.attn_decode(q[:0], cache.k, cache.v, table[:0], n[:0], y[:0], cache.kp, cache.vp)
    assert sr.launch_count() == before


# ---- prompts ----

PREFILL = [
    # (new tokens, earlier keys) per sequence, H, kv, D, causal
    ([(1, 0)], 32, 8, 128, True),
    ([(1, 0), (2, 0), (3, 0)], 4, 4, 64, True),
    ([(127, 0), (128, 0), (129, 0), (1, 0), (0, 0), (63, 0), (64, 0), (65, 0)], 8, 2, 128, True),
    ([(127, 0), (128, 0), (129, 0), (1, 0), (0, 0), (63, 0), (64, 0), (65, 0)], 8, 8, 64, True),
    ([(300, 0), (17, 0)], 8, 2, 128, False),
    ([(300, 0), (17, 0)], 6, 2, 64, False),
    ([(1, 500), (33, 400), (200, 1), (5, 128)], 8, 2, 128, True),
    ([(1, 500), (33, 400), (200, 1), (5, 128)], 8, 1, 64, True),
    ([(700, 0)], 28, 4, 128, True),                    # groups of 7
    ([(257, 30)], 12, 4, 64, True),                    # groups of 3
    ([(260, 3), (40, 0)], 5, 5, 128, True),
    ([(70, 3), (9, 0)], 71, 1, 64, True),              # one key head for 71
    ([(70, 3), (9, 100)], 130, 1, 64, True),           # more heads in a group than a tile has rows
    ([(1500, 0), (600, 900)], 32, 8, 128, True),
    ([(1025, 0)], 8, 8, 128, True),
    ([(1025, 0)], 8, 8, 64, False),
    ([(40, -25), (10, -10), (200, -150), (1, -1), (30, 0)], 8, 2, 128, True),   # more queries than keys: rows that see nothing
    ([(40, -25), (10, -10), (200, -150), (1, -1), (30, 0)], 4, 2, 64, True),
    ([(3, -3), (20, 5)], 4, 2, 64, False),             # no keys at all
    ([(i, 0) for i in range(1, 60)], 4, 2, 128, True),
]


def _packed(pu, gen, seqs, H, kv, D, pad=64):
    import torch
    nq = [a for a, _ in seqs]
    nk = [a + p for a, p in seqs]
    ends = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=pu.DEV)  # noqa: E731
    q = pu.rows(gen, sum(nq), H * D, pad=pad)
    k = pu.rows(gen, sum(nk), kv * D, pad=pad, outliers=(5, 40))
    v = pu.rows(gen, sum(nk), kv * D, 0.7, pad=pad)
    return q, k, v, ends(nq), ends(nk), nq, nk


def _prefill(sr, pu, q, k, v, cq, ck, D, causal, scale=None):
    import torch
    y = torch.full((q.shape[0], q.shape[1] + 8), float("nan"), dtype=torch.float16, device=pu.DEV)[:, :q.shape[1]]
    sr.attn_prefill(q, k, v, cq, ck, y, head_dim=D, causal=causal, scale=scale)
    torch.cuda.synchronize()
    return y


def _seen(pu, a, n, causal):
    import torch
    s = torch.ones(a, n, dtype=torch.bool, device=pu.DEV)
    return s.tril(n - a) if causal else s


def _check_prefill(pu, y, q, k, v, nq, nk, D, kv, causal, scale):
    iq = ik = 0
    for b, (a, n) in enumerate(zip(nq, nk)):
        want, bound = pu.attend(q[iq:iq + a], k[ik:ik + n], v[ik:ik + n], D, kv, scale, _seen(pu, a, n, causal))
        if a:
            bad = (y[iq:iq + a].double() - want).abs() - bound
            assert bool((bad <= 0).all()), (b, a, n, float(bad.max()), (bad > 0).nonzero()[:5].tolist())
        iq, ik = iq + a, ik + n


@pytest.mark.parametrize("seqs,H,kv,D,causal", PREFILL)
def test_prefill_matches_the_plain_form(sr, pu, seqs, H, kv, D, causal):
    import torch
    gen = _gen(len(seqs) + H)
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, seqs, H, kv, D)
    y = _prefill(sr, pu, q, k, v, cq, ck, D, causal)
    assert sr.device_status() == 0
    _check_prefill(pu, y, q, k, v, nq, nk, D, kv, causal, 1 / math.sqrt(D))
    assert torch.equal(y, _prefill(sr, pu, q, k, v, cq, ck, D, causal))


@pytest.mark.parametrize("H,kv,D,seqs", [(32, 8, 128, [(64, -44), (60, -40), (63, -33), (128, -100)]), (8, 8, 64, [(256, -140), (200, -130)])])
def test_prefill_a_tile_without_keys_beside_one_with_keys(sr, pu, H, kv, D, seqs):
    """The first tile of a pair sees no key and answers at once, while its queries are still being loaded."""
    gen = _gen(27)
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, seqs, H, kv, D)
    for _ in range(20):
        y = _prefill(sr, pu, q, k, v, cq, ck, D, True)
        _check_prefill(pu, y, q, k, v, nq, nk, D, kv, True, 1 / math.sqrt(D))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.1), (4.0, 1.5)])
def test_prefill_scores_of_any_size(sr, pu, D, spread, scale):
    gen = _gen(21)
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, [(300, 0), (100, 90)], 4, 2, D)
    k = (k.float() * spread).half()
    y = _prefill(sr, pu, q, k, v, cq, ck, D, True, scale)
    _check_prefill(pu, y, q, k, v, nq, nk, D, 2, True, 1 / math.sqrt(D) if scale is None else scale)


@pytest.mark.parametrize("D,H,kv", [(128, 8, 2), (64, 4, 4)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf"), 65504.0])
def test_prefill_masked_places_have_no_part(sr, pu, D, H, kv, what):
    """Keys and values of later tokens and of other sequences that are not finite (or as large as the type allows)
    change nothing for a query that does not see them, bit for bit."""
    import torch
    gen = _gen(22)
    seqs = [(200, 0), (150, 20), (90, 0)]
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, seqs, H, kv, D)
    clean = _prefill(sr, pu, q, k, v, cq, ck, D, True)
    at = sum(nk[:1]) + 20 + 77                           # token 77 of the second sequence
    for x in (k, v):
        x[at, 1::3] = what
    y = _prefill(sr, pu, q, k, v, cq, ck, D, True)
    first, last = sum(nq[:1]) + 77, sum(nq[:2])
    assert torch.equal(y[:first], clean[:first]) and torch.equal(y[last:], clean[last:])
    if not math.isfinite(what):
        assert not bool(torch.isfinite(y[first:last]).all())


@pytest.mark.parametrize("D,H,kv", [(128, 8, 2), (64, 4, 4)])
def test_prefill_values_that_are_not_finite_show_where_they_are_seen(sr, pu, D, H, kv):
    import torch
    gen = _gen(23)
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, [(300, 0)], H, kv, D)
    clean = _prefill(sr, pu, q, k, v, cq, ck, D, True)
    v[140, 9] = float("inf")
    v[30, 11] = float("nan")
    y = _prefill(sr, pu, q, k, v, cq, ck, D, True)
    g = H // kv
    want = clean.clone()
    for h in range(g):                                   # key head 0
        want[140:, h * D + 9] = float("inf")
        want[30:, h * D + 11] = float("nan")
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.isinf(y), torch.isinf(want))
    ok = torch.isfinite(want)
    assert torch.equal(y[ok], want[ok])


def test_prefill_sequences_that_leave_the_buffers_are_left_out(sr, pu):
    import torch
    gen = _gen(24)
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, [(40, 0), (50, 0)], 4, 2, 128)
    clean = _prefill(sr, pu, q, k, v, cq, ck, 128, True)
    sr.device_status()
    bad = ck.clone()
    bad[2] = 1000
    y = _prefill(sr, pu, q, k, v, cq, bad, 128, True)
    assert sr.device_status() == 35
    assert torch.equal(y[:40], clean[:40]) and bool(torch.isnan(y[40:]).all())
    short = cq.clone()
    short[2] = 70                                        # rows 70.. belong to no sequence
    y = _prefill(sr, pu, q, k, v, short, ck, 128, True)
    assert sr.device_status() == 0 and bool(torch.isnan(y[70:]).all()) and bool(torch.isfinite(y[:70]).all())


def test_prefill_slices_of_a_fused_projection_and_another_stream(sr, pu):
    import torch
    gen = _gen(25)
    H, kv, D, T = 8, 2, 128, 333
    qkv = pu.rows(gen, T, (H + 2 * kv) * D)
    q, k, v = qkv[:, :H * D], qkv[:, H * D:(H + kv) * D], qkv[:, (H + kv) * D:]
    c = torch.tensor([0, 100, T], dtype=torch.int32, device=pu.DEV)
    y = torch.empty(T, H * D, dtype=torch.float16, device=pu.DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sr.attn_prefill(q, k, v, c, c, y, head_dim=D)
    side.synchronize()
    _check_prefill(pu, y, q, k, v, [100, 233], [100, 233], D, kv, True, 1 / math.sqrt(D))
    assert torch.equal(y, _prefill(sr, pu, q.contiguous(), k.contiguous(), v.contiguous(), c, c, D, True))


def test_prefill_agrees_with_decode(sr, pu):
    """The last query of a causal prompt and a new token over a cache with the same keys."""
    import torch
    gen = _gen(26)
    n, H, kv, D = 1000, 8, 2, 128
    cache, table, slots = _paged(pu, gen, [n], kv, D, 16, 16)
    k, v = (x.half() for x in cache.get(slots[0]))
    q = pu.rows(gen, n, H * D)
    c = torch.tensor([0, n], dtype=torch.int32, device=pu.DEV)
    y = _prefill(sr, pu, q, k, v, c, c, D, True)
    one = _decode(sr, pu, q[-1:].contiguous(), cache, table, [n], H)
    want, bound = pu.attend(q[-1:], k, v, D, kv, 1 / math.sqrt(D), torch.ones(1, n, dtype=torch.bool, device=pu.DEV))
    assert bool(((y[-1:].double() - one.double()).abs() <= 2 * bound).all())


def test_prefill_refusals(sr, pu):
    import torch
    gen = _gen(27)
    q, k, v, cq, ck, nq, nk = _packed(pu, gen, [(20, 0)], 4, 2, 128)
    y = torch.empty(20, 512, dtype=torch.float16, device=pu.DEV)
    base = dict(q=q, k=k, v=v, cu_q=cq, cu_k=ck, Y=y)
    before = sr.launch_count()
    bad = [
        (TypeError, dict(q=q.float())), (TypeError, dict(cu_q=cq.long(), cu_k=ck.long())), (ValueError, dict(cu_k=ck[:1])),
        (ValueError, dict(v=v[:, :128])), (ValueError, dict(Y=y[:10])), (ValueError, dict(head_dim=96)),
        (sr.SmoothRotError, dict(head_dim=32)), (sr.SmoothRotError, dict(scale=float("nan"))),
        (sr.SmoothRotError, dict(q=pu.rows(gen, 20, 3 * 128), Y=torch.empty(20, 384, dtype=torch.float16, device=pu.DEV))),
        (TypeError, dict(k=k.cpu())),
    ]
    for kind, change in bad:
        with pytest.raises(kind):
            sr.attn_prefill(**{**base, **change})
    odd = torch.empty(20 * 512 + 1, dtype=torch.float16, device=pu.DEV)[1:].reshape(20, 512)
    with pytest.raises(sr.SmoothRotError) as err:
        sr.attn_prefill(**{**base, "q": odd})
    assert err.value.status == -3
    assert sr.launch_count() == before
    sr.attn_prefill(q[:0], k, v, cq[:1] * 0, ck[:1] * 0, y[:0])
    assert sr.launch_count() == before
