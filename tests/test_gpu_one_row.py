"""One row whose values do not lie next to each other (a column of a wider tensor, every second value, one value expanded): the
calls read and write a row's values as neighbours, so such a row is refused, as two of them are."""
import pytest

pytestmark = pytest.mark.gpu

H, KV, D = 4, 2, 128


@pytest.fixture(scope="module")
def sr():
    from paper_2506_05413_b200 import build, binding
    build.build()
    binding.load()
    return binding


def _row(width):
    import torch
    return torch.zeros(1, width, dtype=torch.float16, device="cuda:0")


def _spread(kind, width):
    import torch
    if kind == "column":
        return torch.zeros(width, 2, dtype=torch.float16, device="cuda:0")[:, :1].T
    if kind == "second":
        return torch.zeros(1, 2 * width, dtype=torch.float16, device="cuda:0")[:, ::2]
    return torch.zeros(1, 1, dtype=torch.float16, device="cuda:0").expand(1, width)


def _calls(sr):
    """Every call with one row: (function, arguments, the row arguments and their widths)."""
    import torch
    one = lambda t: torch.zeros(1, dtype=t, device="cuda:0")  # noqa: E731
    cache = lambda: torch.zeros(1, KV, 16, D, dtype=torch.float16, device="cuda:0")  # noqa: E731
    ends = torch.tensor([0, 1], dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(sr.attn_decode_workspace_bytes(1, H, KV, D), dtype=torch.uint8, device="cuda:0")
    hd, kd = H * D, KV * D
    return {
        "append": (sr.kv_append, dict(q=_row(hd), k=_row(kd), v=_row(kd), positions=one(torch.int32), rotary=torch.zeros(1, D, device="cuda:0"),
                                      slots=one(torch.int64), k_cache=cache(), v_cache=cache(), q_out=_row(hd), k_out=_row(kd)),
                   dict(q=hd, k=kd, v=kd, q_out=hd, k_out=kd)),
        "gather": (sr.kv_gather, dict(slots=one(torch.int64), k_cache=cache(), v_cache=cache(), k_out=_row(kd), v_out=_row(kd)),
                   dict(k_out=kd, v_out=kd)),
        "decode": (sr.attn_decode, dict(q=_row(hd), k_cache=cache(), v_cache=cache(), block_table=torch.zeros(1, 1, dtype=torch.int32, device="cuda:0"),
                                        lengths=torch.ones(1, dtype=torch.int32, device="cuda:0"), Y=_row(hd), workspace=ws), dict(q=hd, Y=hd)),
        "prefill": (sr.attn_prefill, dict(q=_row(hd), k=_row(kd), v=_row(kd), cu_q=ends, cu_k=ends, Y=_row(hd)),
                    dict(q=hd, k=kd, v=kd, Y=hd)),
        "kv_quant": (sr.kv_quant, dict(X=_row(128), clip=0.9, q_out=torch.zeros(1, 64, dtype=torch.uint8, device="cuda:0"),
                                       step_out=torch.zeros(1, 1, device="cuda:0"), zero_out=torch.zeros(1, 1, device="cuda:0")), dict(X=128)),
    }


@pytest.mark.parametrize("kind", ["column", "second", "expanded"])
@pytest.mark.parametrize("name", ["append", "gather", "decode", "prefill", "kv_quant"])
def test_a_row_that_is_not_contiguous_is_refused(sr, name, kind):
    call, args, rows = _calls(sr)[name]
    before = sr.launch_count()
    for arg, width in rows.items():
        with pytest.raises(ValueError):
            call(**{**args, arg: _spread(kind, width)})
    assert sr.launch_count() == before


@pytest.mark.parametrize("name", ["append", "gather", "decode", "prefill", "kv_quant"])
def test_one_row_of_a_wider_tensor_is_taken(sr, name):
    import torch
    call, args, rows = _calls(sr)[name]
    for arg, width in rows.items():
        call(**{**args, arg: torch.zeros(3, width + 64, dtype=torch.float16, device="cuda:0")[1:2, :width]})
    torch.cuda.synchronize()
    assert sr.device_status() == 0
