"""Every output of the 8-bit operators is written: the norm's rows past 4 GiB in both widths, and codes with their scales in replayed graphs and on
two streams, over NaN."""
import numpy as np
import pytest

from oracle import fp8 as o8
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, host
from tests.test_gpu_cache import f64
from tests.test_gpu_fp8 import check_norm, rows_of
from tests.test_gpu_fp8_run import calls, outputs, run, same   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 16])
def test_norm_of_rows_past_four_gib(bits):
    """300,000 rows of 16,384: 9.8 GB of bf16, 4.9 GB of codes."""
    import torch
    from paper_2608_27206_amd import pace
    M, K = 300_000, 16_384
    x = torch.randint(-3, 4, (M, K), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    gamma = 1 + 0.1 * torch.randn(K, device="cuda")
    y, s, h = pace.rmsnorm(x, gamma, residual=x, bits=bits)
    torch.cuda.synchronize()
    for a in (0, 131_072 - 8, 262_144 - 8, M - 16):
        rows = slice(a, a + 16)
        X = f64(x[rows])
        H, Y, tol = o8.norm(X, X, host(gamma).astype(np.float64), float(np.float32(1e-6)))
        check_norm(y[rows], None if s is None else s[:, rows], h[rows], H, Y, tol, True, bits)


def poison(some):
    import torch
    for c in some:
        for t in (c[4]["out"], c[4].get("out_scale")):
            if t is not None:
                t.view(torch.uint8).fill_(0xFF)


def expected(all_calls, workspace):
    import torch
    for c in all_calls:
        run(c, workspace)
    torch.cuda.synchronize()
    return [outputs(c) for c in all_calls]


def test_replays_write_codes_and_scales(calls):   # noqa: F811
    import torch
    ws = torch.empty(max(c[5] for c in calls), dtype=torch.uint8, device="cuda")
    want = expected(calls, ws)
    graphs = []
    for half in (calls[0::2], calls[1::2]):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for c in half:
                run(c, ws)
        graphs.append((graph, half))
    for _ in range(3):
        for graph, half in graphs:
            poison(half)
            ws.fill_(0xFF)
            graph.replay()
        assert all(same(outputs(c), w) for c, w in zip(calls, want))


def test_streams_write_codes_and_scales(calls):   # noqa: F811
    import torch
    ws = [torch.empty(max(c[5] for c in calls), dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = expected(calls, ws[0])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        poison(calls)
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for c in calls[i::2]:
                    run(c, ws[i])
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert all(same(outputs(c), w) for c, w in zip(calls, want))


@pytest.mark.parametrize("M,K,residual,bits", [(1023, 1024, True, 8), (1024, 1024, True, 8), (1024, 1008, False, 16), (1024, 1040, True, 16), (4095, 1536, False, 8), (4096, 1536, False, 8),
                                               (4097, 1040, False, 16), (4096, 1552, False, 16), (19_999, 1280, True, 8), (20_001, 1280, True, 8), (20_000, 1072, True, 8),
                                               (20_000, 1280, True, 16), (20_000, 1296, True, 8)])
def test_norm_on_both_sides_of_its_rule(M, K, residual, bits):
    """Rows that a wave holds, and those that 256 threads hold."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + K)
    x, r, gamma = rows_of(rs, M, K), rows_of(rs, M, K), (1 + 0.1 * rs.standard_normal(K)).astype(np.float32)
    y, s, h = pace.rmsnorm(dev_bf16(x), dev_f32(gamma), dev_bf16(r) if residual else None, bits=bits)
    torch.cuda.synchronize()
    m = np.unique(np.concatenate([np.arange(0, M, 61), np.arange(M - 8, M)]))
    at = torch.from_numpy(m).cuda()
    H, Y, tol = o8.norm(wl.bf16_bits_to_f64(x[m]), wl.bf16_bits_to_f64(r[m]) if residual else None, gamma.astype(np.float64), float(np.float32(1e-6)))
    y = y[at] if bits == 16 else y.view(torch.uint8)[at].view(torch.float8_e4m3fn)
    check_norm(y, None if s is None else s[:, at], None if h is None else h[at], H, Y, tol, residual, bits)
