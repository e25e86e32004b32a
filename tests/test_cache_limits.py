"""What the cache and 4-bit calls refuse at their largest sizes, and the workspaces that they ask for, through the C ABI (CPU: no
pointer is read)."""
import pytest

from tests.test_abi import pace
from tests.test_cache_refusals import BIG, ODD, P, append, attend, cache, w4


@pytest.mark.parametrize("call,kw", [
    (append, dict(c=cache(page=16, heads=8), ks=1024, vs=1024, B=1 << 12, n_src=1 << 14, n_new=1 << 14, max_new=1 << 14, max_pages=1 << 11)),
    (append, dict(c=cache(heads=BIG), ks=1 << 40, vs=1 << 40, B=BIG, n_src=64, n_new=64, max_new=1)),
    (append, dict(c=cache(bits=16), B=1 << 22, n_src=64, n_new=64, max_new=64)),
    (attend, dict(c=cache(heads=8), Hq=8, B=1 << 21, n_q=1 << 21, max_q=1)),
    (attend, dict(c=cache(heads=8), Hq=8, B=1 << 20, n_q=1 << 20, max_q=200)),
])
def test_launches_of_too_many_threads_are_refused(call, kw):
    """2^32 threads or more of padded batches: an error of these calls, before any launch."""
    st, msg = call(**kw)
    assert st == 1 and "too many" in msg, msg


def test_weights_whose_last_tile_of_columns_passes_two_gib():
    st, msg = w4(M=1, N=(1 << 27) - 8, K=32, group=32)
    assert st == 1 and "2 GiB" in msg
    assert pace.lib().pace_gemm_w4_workspace_size(1, (1 << 27) - 8, 32) == 0


def test_sizes_of_calls_that_are_refused_are_zero():
    size = pace.lib().pace_cache_attention_workspace_size
    for B, n, hq, heads in ((BIG, 1, 4, 4), (1, BIG, 4, 4), (1, 1 << 30, 1 << 20, 1 << 10), (1 << 16, 1 << 16, 1 << 30, 1), (BIG, BIG, BIG, 1), (1, 1, BIG, BIG)):
        assert size(n, hq, heads, 128, 16, B, n, 4096, 0, 0) == 0


@pytest.mark.parametrize("args,parts", [
    # n_q, Hq, heads, bits, B, max_q, max_len, window, sinks: the most parts that a length up to max_len is split into
    ((1, 28, 4, 8, 1, 1, 131072, 0, 0), 128), ((1, 28, 4, 16, 1, 1, 131072, 0, 0), 128), ((1, 28, 4, 16, 1, 1, 1183, 0, 0), 10),
    ((48, 28, 4, 8, 48, 1, 16384, 0, 0), 5), ((1024, 28, 4, 16, 1, 1024, 10677, 0, 0), 2), ((64, 28, 4, 16, 64, 1, 300, 0, 0), 3),
    ((1, 28, 4, 16, 1, 1, 128, 0, 0), 1), ((256, 28, 4, 8, 256, 1, 131072, 0, 0), 1), ((24, 28, 4, 8, 24, 1, 32768, 4096, 64), 5)])
def test_attention_asks_for_its_parts_and_refuses_less(args, parts):
    n, hq, heads, bits, B, max_q, max_len, window, sinks = args
    need = pace.lib().pace_cache_attention_workspace_size(n, hq, heads, 128, bits, B, max_q, max_len, window, sinks)
    assert need == (parts * n * hq * (128 + 4) * 4 if parts > 1 else 0)
    if parts > 1:
        kw = dict(c=cache(heads=heads, bits=bits), Hq=hq, n_q=n, B=B, max_q=max_q, max_len=max_len, max_pages=2048, window=window, sinks=sinks)
        for ws, wsb, st, word in ((None, 0, 3, "workspace"), (P, need - 1, 3, "workspace"), (ODD, need, 1, "aligned")):
            got, msg = attend(ws=ws, wsb=wsb, **kw)
            assert got == st and word in msg
