"""The bounded waits of the attention kernels: one that nobody satisfies runs out, its code is reported, the kernel winds down and the
next calls are right.  Nothing here hangs or faults: the probes wait on a barrier nobody arrives on, and with a limit below a
microsecond the kernels take a wait as run out before any copy (attn_prefill) or drain their copies (attn_decode)."""
import math
import time

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    from paper_2506_05413_b200 import build, binding
    build.build()
    binding.load()
    return binding


@pytest.fixture(scope="module")
def au():
    import attention_util
    return attention_util


@pytest.mark.parametrize("code", [36, 37, 38, 39, 40, 41])
def test_each_wait_that_runs_out_reports_its_code(sr, code):
    import torch
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    sr.debug_set_wait_limit_ns(1_000_000)
    try:
        t0 = time.perf_counter()
        sr.debug_attn_wait_expiry(code)
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 1.0
        assert sr.device_status(clear=False) == code
        assert sr.device_status() == code and sr.device_status() == 0
    finally:
        sr.debug_set_wait_limit_ns(0)


def test_codes_without_a_wait_are_refused(sr):
    before = sr.launch_count()
    for code in (0, 7, 35, 42):
        with pytest.raises(sr.SmoothRotError) as err:
            sr.debug_attn_wait_expiry(code)
        assert err.value.status == -1
    assert sr.launch_count() == before


@pytest.mark.parametrize("D,causal", [(128, True), (64, False)])
def test_prefill_winds_down_and_the_next_call_is_right(sr, au, D, causal):
    import torch
    gen = au.generator(D)
    H, kv, n = 8, 2, 1500
    q, k, v = (au.pu.rows(gen, n, w * D) for w in (H, kv, kv))
    ends = torch.tensor([0, 500, n], dtype=torch.int32, device=au.DEV)
    y = torch.empty(n, H * D, dtype=torch.float16, device=au.DEV)
    call = lambda: sr.attn_prefill(q, k, v, ends, ends, y, head_dim=D, causal=causal)  # noqa: E731
    try:
        sr.debug_set_wait_limit_ns(1)
        for _ in range(2):
            call()
            torch.cuda.synchronize()
            assert sr.device_status() == 36
    finally:
        sr.debug_set_wait_limit_ns(0)
    for _ in range(2):
        y.fill_(float("nan"))
        call()
        torch.cuda.synchronize()
        assert sr.device_status() == 0
        for a, b in ((0, 500), (500, n)):
            seen = torch.ones(b - a, b - a, dtype=torch.bool, device=au.DEV)
            want, bound = au.attend(q[a:b], k[a:b], v[a:b], D, kv, 1 / math.sqrt(D), seen.tril() if causal else seen)
            assert bool(((y[a:b].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("lengths", [[5], [250, 3], [6000, 40]])
def test_decode_winds_down_and_the_next_call_is_as_before(sr, au, lengths, bits):
    import torch
    gen = au.generator(bits)
    cache, table, slots = au.paged(gen, lengths, 2, 128, 16, bits)
    q = au.pu.rows(gen, len(lengths), 8 * 128)
    before = au.decode(sr, q, cache, table, lengths)
    ws = au.workspace(sr, len(lengths), 8, 2, 128, 171)
    try:
        sr.debug_set_wait_limit_ns(1)
        au.decode(sr, q, cache, table, lengths, ws=ws)
        assert sr.device_status() == 41
    finally:
        sr.debug_set_wait_limit_ns(0)
    y = au.decode(sr, q, cache, table, lengths, ws=ws)
    assert sr.device_status() == 0 and bool(torch.isfinite(before).all())
    assert torch.equal(y, before)
