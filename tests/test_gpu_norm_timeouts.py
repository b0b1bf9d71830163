"""add_norm's bounded wait for rows, made to run out with a short limit: its code, how its team leaves, and the calls after it."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    from paper_2506_05413_b200 import build, binding
    build.build()
    binding.load()
    return binding


def test_a_wait_for_rows_that_runs_out_is_reported(sr):
    import torch
    import mx_util as mu
    g = mu.gen(1)
    y, h = mu.rows(g, 3000, 4096), mu.rows(g, 3000, 4096)          # so many rows that they go through the teams that wait
    out, want = torch.empty_like(y), torch.empty_like(y)
    sr.add_norm(y, h, h_out=want, post_norm=True)
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    sr.debug_set_wait_limit_ns(1_000_000)
    try:
        for _ in range(2):
            sr.debug_norm_wait_expiry()
            torch.cuda.synchronize()
            assert sr.device_status(clear=False) == 51 and sr.device_status() == 51 and sr.device_status() == 0
        sr.debug_mx_wait_expiry()                                  # of two codes one is reported, and both are cleared
        sr.debug_norm_wait_expiry()
        torch.cuda.synchronize()
        assert sr.device_status() in (50, 51) and sr.device_status() == 0
    finally:
        sr.debug_set_wait_limit_ns(0)
    sr.add_norm(y, h, h_out=out, post_norm=True)
    assert torch.equal(out, want) and sr.device_status() == 0
    z = y.double()
    stream = h.double() + z * mu.rms(z, 1e-5)
    assert bool(((out.double() - stream).abs() <= mu.half_bound(stream, 6 * 2.0 ** -24 * (h.double().abs() + (z * mu.rms(z, 1e-5)).abs()))).all())


def test_the_limit_is_the_waits_own(sr):
    """The probe takes as long as the limit says: the limit that is set reaches this kernel's wait."""
    import time
    import torch
    took = []
    for ms in (2, 60):
        sr.debug_set_wait_limit_ns(ms * 1_000_000)
        try:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            sr.debug_norm_wait_expiry()
            torch.cuda.synchronize()
            took.append(time.perf_counter() - t0)
        finally:
            sr.debug_set_wait_limit_ns(0)
        assert sr.device_status() == 51
    assert took[0] >= 0.002 and took[1] >= 0.06 and took[1] < 1.5
