"""attn_decode in a graph whose segments reach over several CTAs, replayed on one workspace: other queries and other lengths give
their own results, and every launch takes down the flags that its CTAs meet by, also one whose waits run out."""
import pytest

pytestmark = pytest.mark.gpu

H, KV, D = 8, 2, 128


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


class Replay:
    """A captured call over [5000, 17] tokens: 40 CTAs, 20 and more of them at one segment."""

    def __init__(self, sr, au, bits, lengths=(5000, 17)):
        import torch
        gen = au.generator(bits)
        self.sr, self.au, self.lengths = sr, au, list(lengths)
        self.cache, self.table, self.slots = au.paged(gen, self.lengths, KV, D, 16, bits)
        self.gen = gen
        self.q = au.pu.rows(gen, len(lengths), H * D)
        self.n = torch.tensor(self.lengths, dtype=torch.int32, device=au.DEV)
        self.y = torch.zeros(len(lengths), H * D, dtype=torch.float16, device=au.DEV)
        self.ws = au.workspace(sr, len(lengths), H, KV, D)
        call = lambda: sr.attn_decode(self.q, self.cache.k, self.cache.v, self.table, self.n, self.y, self.cache.kp,  # noqa: E731
                                      self.cache.vp, workspace=self.ws)
        call()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            call()

    def new_queries(self):
        self.q.copy_(self.au.pu.rows(self.gen, self.q.shape[0], H * D))

    def run(self):
        import torch
        self.y.fill_(float("nan"))
        self.graph.replay()
        torch.cuda.synchronize()

    def flags_up(self):
        """Flags (the workspace's first 16 bytes a CTA) that are not down."""
        import torch
        ctas = 2 * torch.cuda.get_device_properties(0).multi_processor_count
        return int((self.ws[:16 * ctas].view(torch.int64) != 0).sum())

    def check(self, lengths=None):
        self.au.check(self.y, self.q, self.cache, [s[:n] for s, n in zip(self.slots, lengths or self.lengths)])


@pytest.mark.parametrize("bits", [4, 16])
def test_replays_with_other_queries_on_the_same_workspace(sr, au, bits):
    r = Replay(sr, au, bits)
    for _ in range(4):
        r.new_queries()
        r.run()
        assert sr.device_status() == 0
        r.check()
        assert r.flags_up() == 0


@pytest.mark.parametrize("bits", [4, 16])
def test_replays_with_other_lengths_on_the_same_workspace(sr, au, bits):
    import torch
    r = Replay(sr, au, bits, (9000, 3000, 700))
    for lengths in ([9000, 3000, 700], [4000, 1, 0], [30, 2999, 650], [9000, 0, 1], [8999, 3000, 700]):
        r.new_queries()
        r.n.copy_(torch.tensor(lengths, dtype=torch.int32))
        r.run()
        assert sr.device_status() == 0
        r.check(lengths)
        assert r.flags_up() == 0


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("lengths", [(5000, 17), (9000, 3000, 700), (3, 20000), tuple(range(200, 500))])
def test_a_launch_whose_waits_run_out_leaves_no_flag_for_the_next(sr, au, bits, lengths):
    """With a limit below a microsecond every warp takes its first wait as run out; the launch drains its copies, reports code 41
    and ends.  A replay, whose tag is the same, must not find pieces of it."""
    r = Replay(sr, au, bits, lengths)
    r.run()
    r.check()
    try:
        sr.debug_set_wait_limit_ns(1)
        for _ in range(3):
            r.new_queries()
            r.run()
            assert sr.device_status() == 41
            assert r.flags_up() == 0
    finally:
        sr.debug_set_wait_limit_ns(0)
    for _ in range(2):
        r.new_queries()
        r.run()
        assert sr.device_status() == 0
        r.check()
        assert r.flags_up() == 0
