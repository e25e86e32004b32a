"""The decode operators as a serving program uses them: after a selection, step by step, in graphs, on other streams,
over pools past 4 GiB; and what PACE_DEBUG=1 finds."""
import os

import numpy as np
import pytest

from oracle import cache as oc
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, say
from tests.test_gpu_cache import SECTIONS, check_attention, f64, make_pool

pytestmark = pytest.mark.gpu


def _w4(rs, n, k, group):
    import torch
    w = rs.integers(0, 256, size=(n, k // 2), dtype=np.uint8)
    s = wl.f32_to_bf16_bits(rs.uniform(0.1, 0.3, size=(n, k // group)).astype(np.float32) / np.float32(np.sqrt(k)))
    return {"w": torch.from_numpy(w).cuda(), "s": dev_bf16(s), "host": (w, wl.bf16_bits_to_f64(s), group)}


def _check_w4(got, x, m, **kw):
    w, s, group = m["host"]
    ref, tol = oc.w4(f64(x), w, s, None, group, **kw)
    assert np.all(np.abs(f64(got) - ref) <= 2.0 ** -8 * np.abs(ref) + tol)


@pytest.mark.parametrize("bits", [16, 8])
def test_decode_after_a_selection(bits):
    """A selection keeps some visual tokens; the kept rows and the text go into the cache with their own positions;
    then three decode steps: projection, append, attention, projection with residual, SwiGLU, down.  Every step
    against the oracle on the inputs that it got."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(40 + bits)
    hq, hkv, d, page, hidden, ffn, nv, text = 8, 2, 128, 32, 256, 384, 150, 12
    dev = "cuda"
    idx, _ = pace.topk_gather(dev_f32(rs.random(nv)), 61)
    rows = torch.cat([idx, torch.arange(nv, nv + text, dtype=torch.int32, device=dev)])
    n = int(rows.numel())
    qkv = dev_bf16(wl.random_bf16(7, (nv + text, (hq + 2 * hkv) * d)))
    part = lambda t, a, b: t[:, a * d:b * d].view(t.shape[0], b - a, d)   # noqa: E731
    grid = np.arange(nv)
    pos = np.stack([np.concatenate([a, 40 + np.arange(text)]) for a in (0 * grid, grid // 15, grid % 15)]).astype(np.int32)
    freq = (1e6 ** (-np.arange(d // 2) * 2 / d)).astype(np.float32)
    cache = pace.KvCache.empty(9, hkv, page, d, dtype=torch.bfloat16 if bits == 16 else torch.float8_e4m3fn)
    table = dev_i32([[5, 0, 8, 3]])
    args = dict(inv_freq=dev_f32(freq), sections=SECTIONS[d])
    say(f"prompt of {n} kept rows, {bits} bits")
    q = pace.cache_append(part(qkv, 0, hq), part(qkv, hq, hq + hkv), part(qkv, hq + hkv, hq + 2 * hkv), cache, dev_i32([0, n]),
                          dev_i32([0]), table, n, positions=dev_i32(pos), rows=rows, **args)
    o, lse = pace.cache_attention(q, cache, dev_i32([0, n]), dev_i32([n]), table, n, n)
    torch.cuda.synchronize()
    src = rows.cpu().numpy()
    X = f64(qkv).reshape(nv + text, hq + 2 * hkv, d)[src]
    turned = oc.rotate(X[:, :hq + hkv], pos[:, src], freq, SECTIONS[d])
    mag = np.abs(X[:, :hq, :d // 2]) + np.abs(X[:, :hq, d // 2:])
    assert np.all(np.abs(f64(q) - turned[:, :hq]) <= 2.0 ** -8 * np.abs(turned[:, :hq]) + 1e-6 * np.concatenate([mag, mag], -1))

    def pools():
        return (f64(cache.k), f64(cache.v)) + ((None, None) if bits == 16 else (f64(cache.k_scale), f64(cache.v_scale)))

    def check(o, lse, q, L, nq):
        ref = oc.attention(f64(q), *(pools()), [0, nq], [L], table.cpu().numpy(), page, d ** -0.5)
        check_attention(f64(o), f64(lse), ref, d, nq)

    check(o, lse, q, n, n)
    if bits == 16:
        # the same tokens through the prefill kernel
        kk = dev_bf16(wl.f32_to_bf16_bits(turned[:, hq:].astype(np.float32)))
        vv = part(qkv, hq + hkv, hq + 2 * hkv)[rows.long()].contiguous()
        z = dev_i32([0])
        o2, lse2, _ = pace.prefill_attention_with_mass(q, kk, vv, dev_i32([0, n]), n, z, dev_i32([0, 0]), 0, 0, z, z, 0, want_mass=False)
        torch.cuda.synchronize()
        assert np.max(np.abs(f64(o) - f64(o2))) <= 2e-2 and np.max(np.abs(f64(lse) - f64(lse2))) <= 1e-3

    w = {name: _w4(rs, a, b, 64) for name, a, b in (("qkv", (hq + 2 * hkv) * d, hidden), ("out", hidden, hq * d),
                                                    ("up", 2 * ffn, hidden), ("down", hidden, ffn))}
    x = dev_bf16(wl.random_bf16(9, (1, hidden)))
    bias = rs.standard_normal((hq + 2 * hkv) * d).astype(np.float32) * 0.02
    for step in range(3):
        L = n + step
        y = pace.gemm_w4(x, w["qkv"]["w"], w["qkv"]["s"], bias=dev_f32(bias))
        p = dev_i32(np.full((3, 1), 40 + text + step))
        q = pace.cache_append(part(y, 0, hq), part(y, hq, hq + hkv), part(y, hq + hkv, hq + 2 * hkv), cache, dev_i32([0, 1]),
                              dev_i32([L]), table, 1, positions=p, **args)
        o, lse = pace.cache_attention(q, cache, dev_i32([0, 1]), dev_i32([L + 1]), table, 1, 128)
        a = pace.gemm_w4(o.view(1, hq * d), w["out"]["w"], w["out"]["s"], residual=x, epilogue=1)
        u = pace.gemm_w4(a, w["up"]["w"], w["up"]["s"], epilogue=2)
        z = pace.gemm_w4(u, w["down"]["w"], w["down"]["s"], residual=a, epilogue=1)
        torch.cuda.synchronize()
        _check_w4(y, x, w["qkv"], bias=bias)
        check(o, lse, q, L + 1, 1)
        _check_w4(a, o.view(1, hq * d), w["out"], residual=f64(x), epilogue=1)
        _check_w4(u, a, w["up"], epilogue=2)
        _check_w4(z, u, w["down"], residual=f64(a), epilogue=1)
        x = z


def _step_inputs(rs, bits, B=5, hq=28, hkv=4, d=128, page=64, most=20):
    import torch
    k, v, ks, vs = make_pool(rs, B * most, hkv, page, d, bits)
    s = {"pool": (k, v, ks, vs), "table": dev_i32(rs.permutation(B * most).reshape(B, most)),
         "qkv": dev_bf16(wl.random_bf16(3, (B, (hq + 2 * hkv) * d))), "ctx": dev_i32([0, 64, 700, 63, 1200][:B]),
         "cu": dev_i32(np.arange(B + 1)), "pos": dev_i32(rs.integers(0, 5000, size=(3, B))),
         "freq": dev_f32(1e6 ** (-np.arange(d // 2) * 2 / d)), "heads": (hq, hkv, d), "B": B, "most": most * page}
    s["x"] = dev_bf16(wl.random_bf16(4, (40, 512)))
    s["w"] = _w4(rs, 700, 512, 64)
    s["one"] = torch.ones((), dtype=torch.int32, device="cuda")
    return s


def _step(pace, s, cache, ctx, out=None):
    """One decode step at ctx cached tokens; out: tensors and workspaces to use."""
    hq, hkv, d = s["heads"]
    B, out = s["B"], out or {}
    part = lambda a, b: s["qkv"][:, a * d:b * d].view(B, b - a, d)   # noqa: E731
    q = pace.cache_append(part(0, hq), part(hq, hq + hkv), part(hq + hkv, hq + 2 * hkv), cache, s["cu"], ctx, s["table"], 1,
                          positions=s["pos"], inv_freq=s["freq"], sections=SECTIONS[d], q_out=out.get("q"))
    o, lse = pace.cache_attention(q, cache, s["cu"], ctx + s["one"], s["table"], 1, s["most"], o=out.get("o"), lse=out.get("lse"),
                                  workspace=out.get("ws"))
    y = pace.gemm_w4(s["x"], s["w"]["w"], s["w"]["s"], out=out.get("y"), workspace=out.get("ws4"))
    return {"q": q, "o": o, "lse": lse, "y": y}


def _same(a, b):
    import torch
    return all(torch.equal(a[k].view(torch.int16 if a[k].dtype == torch.bfloat16 else torch.int32),
                           b[k].view(torch.int16 if b[k].dtype == torch.bfloat16 else torch.int32)) for k in a)


@pytest.mark.parametrize("bits", [16, 8])
def test_two_graphs_of_steps(bits):
    """A step captured in two graphs over two caches (lengths on the device, so that a replay takes the next token),
    replayed in turn with eager steps on a third cache between them: every replay equals the eager step."""
    import torch
    from paper_2608_27206_amd import pace
    s = _step_inputs(np.random.default_rng(bits), bits)
    copy = lambda: pace.KvCache(*(None if t is None else t.clone() for t in s["pool"]))   # noqa: E731
    caches, ctxs = [copy() for _ in range(3)], [s["ctx"].clone() for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(pace, s, copy(), s["ctx"].clone())             # a warm-up on another cache
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_step(pace, s, caches[i], ctxs[i]))
            ctxs[i] += 1
        graphs.append(g)
    say(f"captured two steps, {bits} bits")
    for rep in range(4):
        for i in (0, 1):
            for t in outs[i].values():
                t.fill_(3)
        graphs[0].replay()
        graphs[1].replay()
        eager = _step(pace, s, caches[2], ctxs[2])
        ctxs[2] += 1
        torch.cuda.synchronize()
        assert _same(outs[0], eager) and _same(outs[1], eager), f"replay {rep}"
    for c in caches[:2]:
        assert torch.equal(c.k.view(torch.uint8), caches[2].k.view(torch.uint8))


def test_calls_on_two_streams_at_once():
    import torch
    from paper_2608_27206_amd import pace
    s = _step_inputs(np.random.default_rng(5), 8)
    copy = lambda: pace.KvCache(*(t.clone() for t in s["pool"]))   # noqa: E731
    ref = _step(pace, s, copy(), s["ctx"])
    caches = [copy() for _ in range(2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = _step(pace, s, caches[i], s["ctx"])
    torch.cuda.synchronize()
    assert _same(got[0], ref) and _same(got[1], ref)


@pytest.mark.parametrize("bits", [16, 8])
def test_pool_past_4_gib(bits):
    """Pages whose bytes begin past 2^32: appended to, read, by few and by many rows."""
    import torch
    from paper_2608_27206_amd import pace
    hkv, page, d, hq = 8, 256, 128, 16
    pages = (5 << 30) // (hkv * page * d * bits // 8)
    cache = pace.KvCache.empty(pages, hkv, page, d, dtype=torch.bfloat16 if bits == 16 else torch.float8_e4m3fn)
    table = np.array([[pages - 1, 2, pages - 5, pages // 2 + 1]], np.int32)
    n = 800
    k, v = (wl.random_bf16(i, (n, hkv, d)) for i in (1, 2))
    pace.cache_append(None, dev_bf16(k), dev_bf16(v), cache, dev_i32([0, n]), dev_i32([0]), dev_i32(table), n)
    say(f"{pages} pages, {bits} bits")
    for nq in (1, 70):
        q = wl.random_bf16(3, (nq, hq, d))
        o, lse = pace.cache_attention(dev_bf16(q), cache, dev_i32([0, nq]), dev_i32([n]), dev_i32(table), nq, n)
        torch.cuda.synchronize()
        at = torch.from_numpy(table[0].astype(np.int64)).cuda()
        take = lambda t: f64(t.view(torch.uint8 if bits == 8 else torch.int16)[at].view(t.dtype))   # noqa: E731
        ks, vs = (None, None) if bits == 16 else (f64(cache.k_scale[at]), f64(cache.v_scale[at]))
        K, V = take(cache.k), take(cache.v)
        step = 0.0 if bits == 16 else 2.0 ** -4
        for pool, sc, x in ((K, ks, k), (V, vs, v)):
            x = wl.bf16_bits_to_f64(x)
            for t in (0, 255, 256, n - 1):
                got = pool[t // page, :, t % page] * (1.0 if sc is None else sc[t // page][:, None])
                low = 0.0 if sc is None else 2.0 ** -10 * sc[t // page][:, None]
                assert np.all(np.abs(got - x[t]) <= step * np.abs(x[t]) + low)
        ref = oc.attention(wl.bf16_bits_to_f64(q), K, V, ks, vs, [0, nq], [n], np.arange(4)[None], page, d ** -0.5)
        check_attention(f64(o), f64(lse), ref, d, nq)


def test_repeated_calls_give_the_same_bits():
    import torch
    from paper_2608_27206_amd import pace
    s = _step_inputs(np.random.default_rng(8), 16)
    cache = pace.KvCache(*s["pool"])
    first = {k: t.clone() for k, t in _step(pace, s, cache, s["ctx"]).items()}
    for _ in range(5):
        again = _step(pace, s, cache, s["ctx"])
        torch.cuda.synchronize()
        assert _same(first, again)


def test_binding_refusals_on_the_gpu():
    import torch
    from paper_2608_27206_amd import pace
    s = _step_inputs(np.random.default_rng(9), 16)
    cache = pace.KvCache(*s["pool"])
    hq, hkv, d = s["heads"]
    k = s["qkv"][:, hq * d:(hq + hkv) * d].view(s["B"], hkv, d)
    q = torch.zeros((5, hq, d), dtype=torch.bfloat16, device="cuda")
    app = lambda **kw: pace.cache_append(**{**dict(q=None, k=k, v=k, cache=cache, cu_new=s["cu"], ctx_len=s["ctx"],   # noqa: E731
                                                   block_table=s["table"], max_new=1), **kw})
    att = lambda **kw: pace.cache_attention(**{**dict(q=q, cache=cache, cu_q=s["cu"], seq_len=s["ctx"], block_table=s["table"],   # noqa: E731
                                                      max_q=1, max_len=1280), **kw})
    for bad in (dict(k=k.float()), dict(k=k[:, :2]), dict(v=k[:3]), dict(k=k.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(cu_new=s["cu"].long()), dict(cu_new=s["cu"][:3]), dict(ctx_len=s["ctx"].cpu()), dict(block_table=s["table"][0]),
                dict(block_table=s["table"].t()), dict(positions=s["pos"], inv_freq=s["freq"]), dict(positions=s["pos"][:, :3]),
                dict(positions=s["pos"], inv_freq=s["freq"][:5], sections=SECTIONS[d]), dict(rows=s["ctx"].float()), dict(max_new=6),
                dict(q=q[:, :, :64]), dict(q=q, q_out=q[:3])):
        with pytest.raises(pace.PaceError):
            app(**bad)
    for bad in (dict(q=q.float()), dict(q=q[:, :27]), dict(q=q[:, :, :80]), dict(cu_q=s["cu"][1:]), dict(seq_len=s["ctx"].long()), dict(max_len=1281),
                dict(max_q=6), dict(window=-1), dict(o=q[:2]), dict(lse=torch.zeros(3, device="cuda")), dict(scale=0.0),
                dict(workspace=torch.zeros(64, device="cuda")), dict(workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(pace.PaceError):
            att(**bad)
    w, sc = s["w"]["w"], s["w"]["s"]
    for bad in (dict(x=s["x"].float()), dict(x=s["x"][:, ::2]), dict(w=w[:, :-1]), dict(scale=sc.float()), dict(scale=sc[:, :3]), dict(zero=w),
                dict(bias=s["freq"]), dict(residual=s["x"]), dict(epilogue=1), dict(out=s["x"])):
        with pytest.raises(pace.PaceError):
            pace.gemm_w4(**{**dict(x=s["x"], w=w, scale=sc), **bad})
    att()
    torch.cuda.synchronize()


@pytest.fixture
def debug_env():
    old = os.environ.get("PACE_DEBUG")
    os.environ["PACE_DEBUG"] = "1"
    yield
    if old is None:
        del os.environ["PACE_DEBUG"]
    else:
        os.environ["PACE_DEBUG"] = old


def test_debug_checks(debug_env):
    """Inconsistent lengths, tables and rows come back as errors before any launch."""
    import torch
    from paper_2608_27206_amd import pace
    cache = pace.KvCache(*make_pool(np.random.default_rng(1), 6, 2, 16, 128, 16))
    x = dev_bf16(wl.random_bf16(1, (40, 2, 128)))
    good = dict(cu=[0, 20, 40], ctx=[0, 5], table=[[0, 1], [2, 3]], rows=list(range(40)))
    for bad, word in ((dict(cu=[0, 30, 20]), "cu_new"), (dict(cu=[0, 20, 41]), "cu_new"), (dict(ctx=[0, 13]), "sequence 1"), (dict(ctx=[-1, 5]), "sequence 0"),
                      (dict(table=[[0, 6], [2, 3]]), "block_table"), (dict(table=[[0, 1], [1, 3]]), "written twice"),
                      (dict(rows=[40] + list(range(39))), "rows")):
        c = {**good, **bad}
        with pytest.raises(pace.PaceError, match=word):
            pace.cache_append(None, x, x, cache, dev_i32(c["cu"]), dev_i32(c["ctx"]), dev_i32(c["table"]), 20, rows=dev_i32(c["rows"]))
    pace.cache_append(None, x, x, cache, dev_i32(good["cu"]), dev_i32(good["ctx"]), dev_i32(good["table"]), 20, rows=dev_i32(good["rows"]))
    q = dev_bf16(wl.random_bf16(2, (2, 4, 128)))
    for cu, lens, table, word in (([0, 2, 1], [20, 25], [[0, 1], [2, 3]], "cu_q"), ([0, 1, 2], [20, 33], [[0, 1], [2, 3]], "seq_len"),
                                  ([0, 1, 2], [20, 25], [[0, -1], [2, 3]], "block_table")):
        with pytest.raises(pace.PaceError, match=word):
            pace.cache_attention(q, cache, dev_i32(cu), dev_i32(lens), dev_i32(table), 1, 32)
    # entries past a sequence's pages are not looked at
    pace.cache_attention(q, cache, dev_i32([0, 1, 2]), dev_i32([16, 25]), dev_i32([[0, 99], [2, 3]]), 1, 32)
    torch.cuda.synchronize()


@pytest.mark.parametrize("bits", [16, 8])
def test_pages_that_left_the_window(debug_env, bits):
    """A caller that streams gives back the pages behind the window: their entries are -1, the results stay, and
    PACE_DEBUG complains about the pages that are still seen alone."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(9 + bits)
    page, n, window, sinks = 16, 400, 60, 20
    kc, vc, ks, vs = make_pool(rs, 27, 2, page, 128, bits)
    cache = pace.KvCache(kc, vc, ks, vs)
    q = dev_bf16(wl.random_bf16(3, (4, 8, 128)))
    table = rs.permutation(27)[:25].astype(np.int32)[None]
    first = (n - 3 - window + 1) // page                                # seen by the first of three queries
    gone = table.copy()
    gone[0, 2:first] = -1
    for nq in (1, 3):
        say(f"pages behind the window: bits {bits}, {nq} queries")
        cu, lens = dev_i32([0, nq]), dev_i32([n])
        want = pace.cache_attention(q[:nq], cache, cu, lens, dev_i32(table), nq, n, window=window, sinks=sinks)
        got = pace.cache_attention(q[:nq], cache, cu, lens, dev_i32(gone), nq, n, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[1], want[1])
    for j in (1, first):
        bad = gone.copy()
        bad[0, j] = -1
        with pytest.raises(pace.PaceError, match="block_table"):
            pace.cache_attention(q[:3], cache, cu, lens, dev_i32(bad), 3, n, window=window, sinks=sinks)
    # a sequence without queries is not looked at
    pace.cache_attention(q[:1], cache, dev_i32([0, 1, 1]), dev_i32([n, n]), dev_i32(np.concatenate([gone, 0 * gone - 1])), 1, n,
                         window=window, sinks=sinks)
    torch.cuda.synchronize()
