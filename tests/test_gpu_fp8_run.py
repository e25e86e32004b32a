"""The 8-bit operators as a program runs them: a layer over a selection's kept rows and its decode steps, in two graphs that
share a workspace, on two streams, over operands past 4 GiB.  Every step against the oracle on the inputs that it got."""
import numpy as np
import pytest

from oracle import fp8 as o8
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, host, say
from tests.test_gpu_cache import f64
from tests.test_gpu_fp8 import bits_of, check_norm, check_product, code_values

pytestmark = pytest.mark.gpu


class Weights:
    """Weights laid out once: bf16 rows to codes with a scale for each 128 x 128."""

    def __init__(self, rs, n, k):
        from paper_2608_27206_amd import pace
        self.w, self.s = pace.quantize_fp8(dev_bf16(bits_of(rs.standard_normal((n, k)) / np.sqrt(k))), rows=128)
        self.W, self.S = code_values(self.w), host(self.s).astype(np.float64)


def product(x, xs, m, bits=16, **kw):
    """gemm_fp8 on the codes x, checked."""
    import torch
    from paper_2608_27206_amd import pace
    y, s = pace.gemm_fp8(x, xs, m.w, m.s, bits=bits, **kw)
    torch.cuda.synchronize()
    res = kw.get("residual")
    ref = o8.product(code_values(x), host(xs).astype(np.float64), m.W, m.S, None if kw.get("bias") is None else host(kw["bias"]),
                     None if res is None else f64(res), kw.get("epilogue", 0), bits == 8)
    check_product(y, s, ref, bits)
    return y, s


def normed(x, gamma, residual):
    import torch
    from paper_2608_27206_amd import pace
    y, s, h = pace.rmsnorm(x, gamma, residual=residual, bits=8)
    torch.cuda.synchronize()
    H, Y, tol = o8.norm(f64(x), None if residual is None else f64(residual), host(gamma).astype(np.float64), float(np.float32(1e-6)))
    check_norm(y, s, h, H, Y, tol, residual is not None, 8)
    return y, s, h


def quantized(x):
    import torch
    from paper_2608_27206_amd import pace
    q, s = pace.quantize_fp8(x)
    torch.cuda.synchronize()
    X, S = f64(x), host(s).astype(np.float64)
    assert o8.codes_ok(code_values(q), X, S, 1, 0.0).all() and np.all(np.abs(S - o8.scales(X, 1)) <= 2.0 ** -23 * S)
    return q, s


def test_layer_over_kept_rows_and_decode_steps():
    """A selection keeps rows of the context; a layer runs over them (norm, fused projection, append, attention, output
    projection with the residual, norm, gate and up, down with the residual), then over single tokens of two sequences."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(7)
    hq, hkv, d, page, hidden, ffn, nv, text = 8, 2, 128, 32, 272, 400, 150, 12
    qkv, out, gu, down = (Weights(rs, n, k) for n, k in (((hq + 2 * hkv) * d, hidden), (hidden, hq * d), (2 * ffn, hidden), (hidden, ffn)))
    bias, g1, g2 = dev_f32(0.1 * rs.standard_normal((hq + 2 * hkv) * d)), dev_f32(1 + 0.1 * rs.standard_normal(hidden)), dev_f32(np.ones(hidden))
    idx, _ = pace.topk_gather(dev_f32(rs.random(nv)), 61)
    rows = torch.cat([idx, torch.arange(nv, nv + text, dtype=torch.int32, device="cuda")])
    stream = pace.gather_rows(dev_bf16(bits_of(rs.standard_normal((nv + text, hidden)))), rows)
    cache = pace.KvCache.empty(9, hkv, page, d)
    table = dev_i32([[5, 0, 8, 3], [1, 2, 4, 6]])
    freq = dev_f32(1e6 ** (-np.arange(d // 2) * 2 / d))

    def layer(x, add, cu, ctx, lens, longest):
        """x: what the layer before adds to the stream `add` (None: x is the stream)."""
        n = x.shape[0]
        say(f"layer over {n} rows")
        a, a_s, h = normed(x, g1, add)
        h = x if h is None else h
        p, _ = product(a, a_s, qkv, bias=bias)
        q, k, v = (p[:, i * d:j * d].view(n, j - i, d) for i, j in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
        pos = dev_i32(np.concatenate([np.arange(c, c + b - a) for a, b, c in zip(cu, cu[1:], ctx)]))
        q = pace.cache_append(q, k, v, cache, dev_i32(cu), dev_i32(ctx), table[:len(ctx)].contiguous(), longest, positions=pos, inv_freq=freq)
        o, _ = pace.cache_attention(q, cache, dev_i32(cu), dev_i32(lens), table[:len(ctx)].contiguous(), longest, 128)
        b, b_s = quantized(o.view(n, hq * d))
        r, _ = product(b, b_s, out, epilogue=1, residual=h)
        c, c_s, _ = normed(r, g2, None)
        f, f_s = product(c, c_s, gu, bits=8, epilogue=2)
        y, _ = product(f, f_s, down)
        return y, r

    n = int(rows.numel())
    y, r = layer(stream, None, [0, n, n + 0], [0, 0], [n, 0], n)
    y, r = layer(y, r, [0, n, n], [0, 0], [n, 0], n)               # a second layer: its norm adds what the first one gave
    one = dev_bf16(bits_of(rs.standard_normal((2, hidden))))
    for step in range(3):
        y, r = layer(one, one, [0, 1, 2], [n + step, step], [n + step + 1, step + 1], 1)
        one = y


@pytest.fixture(scope="module")
def calls():
    """Calls of every kind of plan (few rows, tiles, parts of K and their join, two launches, several tiles to a workgroup) on fixed
    inputs, each with a workspace and outputs of its own."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(3)
    made = []
    for M, N, K, epilogue, bits, sums in ((1, 640, 3584, 0, 16, 0), (9, 1024, 1040, 2, 8, 0), (48, 384, 4112, 1, 16, 0), (300, 1056, 1552, 2, 8, 1), (300, 520, 656, 1, 16, 0),
                                          (700, 3616, 272, 2, 8, 0), (2700, 6700, 1040, 1, 16, 0), (5300, 5136, 528, 0, 16, 0), (3000, 6144, 528, 2, 8, 0)):
        x, xs = pace.quantize_fp8(dev_bf16(bits_of(rs.standard_normal((M, K)))))
        w, ws = pace.quantize_fp8(dev_bf16(bits_of(rs.standard_normal((N, K)))), rows=128)
        cols = N // 2 if epilogue == 2 else N
        kw = dict(epilogue=epilogue, bits=bits, sums=sums)
        if epilogue == 1:
            kw["residual"] = dev_bf16(bits_of(rs.standard_normal((M, N))))
        kw["out"] = torch.empty((M, cols), dtype=torch.float8_e4m3fn if bits == 8 else torch.bfloat16, device="cuda")
        if bits == 8:
            kw["out_scale"] = torch.empty(((cols + 127) // 128, M), device="cuda")
        need = pace.lib().pace_gemm_fp8_workspace_size(M, N, K, bits, sums)
        made.append((x, xs, w, ws, kw, need))
    return made


def outputs(call):
    kw = call[4]
    return [t.view(torch_u8()).clone() for t in (kw["out"], kw.get("out_scale")) if t is not None]


def torch_u8():
    import torch
    return torch.uint8


def run(call, workspace):
    from paper_2608_27206_amd import pace
    x, xs, w, ws, kw, need = call
    pace.gemm_fp8(x, xs, w, ws, workspace=workspace if need else None, **kw)


def same(a, b):
    import torch
    return len(a) == len(b) and all(torch.equal(u, v) for u, v in zip(a, b))


def test_equal_calls_give_equal_bits(calls):
    import torch
    ws = torch.empty(max(c[5] for c in calls), dtype=torch.uint8, device="cuda")
    first = []
    for c in calls:
        run(c, ws)
        first.append(outputs(c))
    for c, f in zip(calls, first):
        for t in (c[4]["out"], c[4].get("out_scale")):
            if t is not None:
                t.view(torch.uint8).fill_(0xFF)
        ws.fill_(0xFF)                                   # NaN where a part of it would be read before it is written
        run(c, ws)
        assert same(outputs(c), f)


def test_two_graphs_share_a_workspace(calls):
    """Two captured graphs that use one workspace, replayed in turn on one stream with eager work between them."""
    import torch
    from paper_2608_27206_amd import pace
    ws = torch.empty(max(c[5] for c in calls), dtype=torch.uint8, device="cuda")
    halves = (calls[0::2], calls[1::2])
    want = []
    for c in calls:
        run(c, ws)
    torch.cuda.synchronize()
    want = [[outputs(c) for c in h] for h in halves]
    x = dev_bf16(bits_of(np.random.default_rng(1).standard_normal((33, 1296))))
    g = torch.ones(1296, device="cuda")
    q0, s0 = (t.clone() for t in pace.rmsnorm(x, g, residual=x, bits=8)[:2])
    q, s, h = torch.empty_like(q0), torch.empty_like(s0), torch.empty_like(x)
    graphs = []
    for half in halves:
        for c in half:
            run(c, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pace.rmsnorm(x, g, residual=x, bits=8, out=q, scale=s, sum_out=h)
            for c in half:
                run(c, ws)
        graphs.append(graph)
    for turn in range(3):
        for graph, half, w in zip(graphs, halves, want):
            for c in half:
                c[4]["out"].view(torch.uint8).zero_()
            q.view(torch.uint8).zero_()
            graph.replay()
            if turn == 1:
                torch.cuda.synchronize()
            y = pace.rmsnorm(x, g, bits=16)[0]           # eager work between the replays
            assert y.shape == x.shape
            for c, v in zip(half, w):
                assert same(outputs(c), v)
            assert torch.equal(q.view(torch.uint8), q0.view(torch.uint8)) and torch.equal(s, s0)


def test_two_streams(calls):
    """Calls on two streams at once, a workspace each, on inputs made on a third."""
    import torch
    one = torch.empty(max(c[5] for c in calls), dtype=torch.uint8, device="cuda")
    for c in calls:
        run(c, one)
    torch.cuda.synchronize()
    want = [outputs(c) for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    spaces = [one, torch.empty_like(one)]
    for _ in range(5):
        for c in calls:
            c[4]["out"].view(torch.uint8).zero_()
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for c in calls[i::2]:
                    run(c, spaces[i])
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert all(same(outputs(c), w) for c, w in zip(calls, want))


# ---------------------------------------------------------------- past 4 GiB
def test_rows_past_four_gib():
    """300,000 rows of 16,384: 9.8 GB of bf16, 4.9 GB of codes.  Rows at the end as in a call of their own."""
    import torch
    from paper_2608_27206_amd import pace
    M, K, N = 300_000, 16_384, 72
    x = torch.randint(-3, 4, (M, K), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    q, s = pace.quantize_fp8(x)
    y, ys, h = pace.rmsnorm(x, torch.ones(K, device="cuda"), residual=x, bits=8)
    w, ws = pace.quantize_fp8(torch.randn(N, K, device="cuda").to(torch.bfloat16), rows=128)
    c, _ = pace.gemm_fp8(q, s, w, ws)
    torch.cuda.synchronize()
    for a in (0, 131_072 - 8, 262_144 - 8, M - 16):
        rows = slice(a, a + 16)
        q1, s1 = pace.quantize_fp8(x[rows])
        assert torch.equal(q[rows].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[:, rows], s1)
        # the sum of squares of few rows is added in another order
        y1, t1, h1 = pace.rmsnorm(x[rows], torch.ones(K, device="cuda"), residual=x[rows], bits=8)
        assert torch.equal(h[rows], h1) and torch.allclose(ys[:, rows], t1, rtol=1e-5)
        ref = o8.product(code_values(q[rows]), host(s[:, rows].contiguous()).astype(np.float64), code_values(w), host(ws).astype(np.float64), wide=False)
        check_product(c[rows], None, ref, 16)


def test_weights_past_four_gib():
    import torch
    from paper_2608_27206_amd import pace
    N, K = 300_032, 16_384
    w = torch.randint(-3, 4, (N, K), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    q, s = pace.quantize_fp8(w, rows=128)
    del w
    for M in (3, 40):
        x, xs = pace.quantize_fp8(torch.randn(M, K, device="cuda").to(torch.bfloat16))
        for kw in (dict(), dict(epilogue=2, bits=8)):
            y, ys = pace.gemm_fp8(x, xs, q, s, **kw)
            torch.cuda.synchronize()
            X, XS = code_values(x), host(xs).astype(np.float64)
            for a in (0, 131_072, 262_144, N - 256):
                ref = o8.product(X, XS, code_values(q[a:a + 256]), host(s[a // 128:a // 128 + 2]).astype(np.float64), epilogue=kw.get("epilogue", 0), wide=bool(kw))
                if kw:
                    check_product(y[:, a // 2:a // 2 + 128], ys[a // 256:a // 256 + 1], ref, 8)
                else:
                    check_product(y[:, a:a + 256].contiguous(), None, ref, 16)


def test_output_and_residual_past_four_gib():
    import torch
    from paper_2608_27206_amd import pace
    M, N, K = 70_000, 32_776, 128
    x, xs = pace.quantize_fp8(torch.randn(M, K, device="cuda").to(torch.bfloat16))
    w, ws = pace.quantize_fp8(torch.randn(N, K, device="cuda").to(torch.bfloat16), rows=128)
    res = torch.randint(-3, 4, (M, N), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    y, _ = pace.gemm_fp8(x, xs, w, ws, residual=res, epilogue=1)
    torch.cuda.synchronize()
    for a in (0, 32_700, 65_500, M - 40):
        rows = slice(a, a + 40)
        ref = o8.product(code_values(x[rows]), host(xs[:, rows].contiguous()).astype(np.float64), code_values(w), host(ws).astype(np.float64), None, f64(res[rows]), 1, False)
        check_product(y[rows], None, ref, 16)


@pytest.mark.parametrize("M,N,epilogue,bits", [(70_000, 32_776, 0, 16), (140_000, 32_800, 2, 16), (140_000, 65_536, 2, 8)])
def test_output_past_four_gib_of_several_tiles_a_workgroup(M, N, epilogue, bits):
    import torch
    from paper_2608_27206_amd import pace
    K = 528
    x, xs = pace.quantize_fp8(torch.randn(M, K, device="cuda").to(torch.bfloat16))
    w, ws = pace.quantize_fp8(torch.randn(N, K, device="cuda").to(torch.bfloat16), rows=128)
    y, ys = pace.gemm_fp8(x, xs, w, ws, epilogue=epilogue, bits=bits)
    torch.cuda.synchronize()
    for a in (0, M // 2 - 6, M - 12):
        rows = slice(a, a + 12)
        ref = o8.product(code_values(x[rows]), host(xs[:, rows].contiguous()).astype(np.float64), code_values(w), host(ws).astype(np.float64), epilogue=epilogue, wide=bits == 8)
        check_product(y[rows], ys[:, rows].contiguous() if bits == 8 else None, ref, bits)
