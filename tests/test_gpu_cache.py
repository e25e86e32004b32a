"""The paged cache and 4-bit weights on the GPU against the float64 oracle (oracle/cache.py).

Tolerances, all from arithmetic: one rounding of an output is at most half a step of its type (bf16 2^-8 of the
value, e4m3 2^-4, or 2^-10 of the scale among its subnormals); the rotation's angle, functions and products in 32 bits stay
within 1e-6 of |x_f| + |x_f+d/2| (half a turn rounded to 24 bits is 2 * 10^-7, the functions 2 ulp, three
products' roundings 2 * 10^-7); a probability rounded to bf16 moves the output by 2^-8 sum P |v|; a score of d
products in 32 bits is off by (d + 8) 2^-24 of scale * sum |q k|, and the exponential and logarithm by 4e-6."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, host, say

pytestmark = pytest.mark.gpu

SECTIONS = {128: (16, 24, 24), 80: (8, 16, 16)}
VALUES = oc.e4m3_values()


def f64(t):
    """A device tensor's values in float64 (e4m3 by the oracle's table)."""
    import torch
    if t.dtype == torch.float8_e4m3fn:
        return VALUES[t.view(torch.uint8).cpu().numpy()]
    if t.dtype == torch.bfloat16:
        return wl.bf16_bits_to_f64(t.view(torch.int16).cpu().numpy().view(np.uint16))
    return t.cpu().numpy().astype(np.float64)


def make_pool(rs, pages, heads, page, dim, bits, scale_of=1.0):
    """Random pages as device tensors; 8 bits: random finite codes and power-of-two scales."""
    import torch
    shape = (pages, heads, page, dim)
    if bits == 16:
        return [dev_bf16(wl.f32_to_bf16_bits(rs.standard_normal(shape).astype(np.float32) * scale_of))
                for _ in range(2)] + [None, None]
    out = []
    for _ in range(2):
        c = rs.integers(0, 0x78, size=shape).astype(np.uint8) | (rs.integers(0, 2, size=shape) << 7).astype(np.uint8)
        out.append(torch.from_numpy(c).cuda().view(torch.float8_e4m3fn))
    # codes up to 240 in magnitude: scales near 1/100 give values of a few units
    out += [dev_f32(scale_of * 2.0 ** rs.integers(-8, -5, size=(pages, heads))) for _ in range(2)]
    return out


def make_table(rs, lens, page, spare=2):
    per = [-(-n // page) for n in lens]
    pages = sum(per) + spare
    order = rs.permutation(pages)
    table = np.full((len(lens), max(1, max(per))), -7, np.int32)     # unused entries are never read
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    return pages, table


def poison(t, keep):
    """NaN in every slot [page, slot] of a pool that no sequence holds."""
    import torch
    raw = t.view(torch.uint8 if t.dtype == torch.float8_e4m3fn else torch.int16)
    dead = torch.from_numpy(~keep).cuda()[:, None, :, None].expand_as(raw)
    raw[dead] = 0x7F if t.dtype == torch.float8_e4m3fn else 0x7FC0


def held_slots(pages, table, lens, page):
    keep = np.zeros((pages, page), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            if 0 <= table[b, j // page] < pages:
                keep[table[b, j // page], j % page] = True
    return keep


# ---------------------------------------------------------------- append
APPEND = [
    # bits, page, heads (q, kv), dim, ctx, new, axes, rows
    (16, 16, (4, 2), 128, [0], [1], 1, False),
    (16, 64, (28, 4), 128, [1183, 0, 63], [1, 1, 1], 3, False),
    (16, 32, (3, 1), 80, [5, 31, 32], [40, 0, 17], 3, True),
    (16, 256, (16, 16), 80, [250], [700], 1, True),
    (8, 16, (4, 2), 128, [0], [1], 1, False),
    (8, 16, (4, 2), 128, [0, 16, 15, 7], [1, 16, 2, 33], 3, False),
    (8, 64, (28, 4), 128, [700, 0, 63, 64], [1, 1, 1, 1], 3, False),
    (8, 32, (8, 8), 80, [3, 0, 95], [90, 0, 1], 1, True),
    (8, 128, (7, 1), 128, [100], [300], 3, True),
    (8, 256, (2, 2), 128, [0, 255], [513, 1], 3, False),
    (8, 256, (2, 2), 80, [17], [240], 3, False),
    (8, 64, (0, 4), 128, [10, 20], [3, 4], 3, False),        # no queries
    (16, 64, (0, 4), 128, [10, 20], [3, 70], 0, False),      # no queries, no rotation
    (8, 64, (6, 2), 128, [10], [70], 0, True),               # no rotation
]


@pytest.mark.parametrize("was_scale", [0.05, 2.0 ** -4], ids=["odd_scales", "powers_of_two"])
@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"bits{c[0]}-p{c[1]}-h{c[2][0]}.{c[2][1]}-d{c[3]}-ctx{c[4]}-new{c[5]}-ax{c[6]}")
def test_append(case, was_scale):
    import torch
    from paper_2608_27206_amd import pace
    bits, page, (hq, hkv), dim, ctx, new, axes, rows = case
    rs = np.random.default_rng(sum(map(ord, str(case))))
    lens = [a + b for a, b in zip(ctx, new)]
    pages, table = make_table(rs, lens, page)
    kc, vc, ks, vs = make_pool(rs, pages, hkv, page, dim, bits, was_scale)   # new tokens are larger: some pages' scales grow
    before = [f64(kc), f64(vc), None if ks is None else f64(ks), None if vs is None else f64(vs)]
    n, n_pad = sum(new), sum(new) + 3                                   # three rows behind the last sequence
    n_src = 2 * n_pad + 5 if rows else n_pad
    qkv = wl.f32_to_bf16_bits(rs.standard_normal((n_src, (hq + 2 * hkv) * dim)).astype(np.float32))
    dq = dev_bf16(qkv)
    part = lambda a, b: dq[:, a * dim:b * dim].view(n_src, b - a, dim)   # noqa: E731
    q, k, v = part(0, hq), part(hq, hq + hkv), part(hq + hkv, hq + 2 * hkv)
    src = np.sort(rs.permutation(n_src)[:n_pad]).astype(np.int32) if rows else np.arange(n_pad, dtype=np.int32)
    pos = rs.integers(0, 1 << 20, size=(max(1, axes), n_src)).astype(np.int32)
    freq = (1e6 ** (-np.arange(dim // 2) * 2 / dim)).astype(np.float32)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    cache = pace.KvCache(kc, vc, ks, vs)
    q_out = torch.full((n_pad, max(hq, 1), dim), 7.0, dtype=torch.bfloat16, device="cuda")
    say(f"append {case}")
    got = pace.cache_append(q if hq else None, k, v, cache, dev_i32(cu), dev_i32(ctx), dev_i32(table), max(new),
                            positions=dev_i32(pos if axes > 1 else pos[0]) if axes else None,
                            inv_freq=dev_f32(freq) if axes else None, sections=SECTIONS[dim] if axes == 3 else None,
                            rows=dev_i32(src) if rows else None, q_out=q_out if hq else None)
    torch.cuda.synchronize()
    X = wl.bf16_bits_to_f64(qkv).reshape(n_src, hq + 2 * hkv, dim)[src[:n]]
    qk, V = X[:, :hq + hkv], X[:, hq + hkv:]
    mag = np.abs(qk)[..., :dim // 2] + np.abs(qk)[..., dim // 2:]
    noise = 1e-6 * np.concatenate([mag, mag], -1) if axes else np.zeros_like(qk)
    if axes:
        qk = oc.rotate(qk, pos[:, src[:n]], freq, SECTIONS[dim] if axes == 3 else None)
    if hq:
        out = f64(got)
        assert np.all(np.abs(out[:n] - qk[:, :hq]) <= 2.0 ** -8 * np.abs(qk[:, :hq]) + noise[:, :hq])
        assert np.all(out[n:] == 7.0), "rows behind the last sequence changed"
    else:
        assert got is None
    for name, x, nz, was, was_s, now, now_s in (("k", qk[:, hq:], noise[:, hq:], before[0], before[2], f64(kc), ks),
                                                ("v", V, np.zeros_like(V), before[1], before[3], f64(vc), vs)):
        ref, s, written = oc.append(was, was_s, x, cu, ctx, table, page, bits)
        tol = oc.append(np.zeros_like(was), None, nz, cu, ctx, table, page, 16)[0]
        w = np.broadcast_to(written[:, None, :, None], ref.shape)
        if bits == 16:
            assert np.array_equal(now[~w], was[~w]), f"{name}: other slots changed"
            assert np.all(np.abs(now - ref)[w] <= (2.0 ** -8 * np.abs(ref) + tol)[w]), name
            continue
        assert np.array_equal(f64(now_s), s), f"{name}: scales"
        assert np.all(np.abs(now - ref)[w] <= (2.0 ** -4 * np.abs(ref) + 2.0 ** -10 + tol / s[:, :, None, None])[w]), name
        # the other slots: left alone, or moved to the new scale: exact between powers of two but for subnormals,
        # one rounding (2^-4) from a scale that is none
        moved = np.broadcast_to((s != was_s)[:, :, None, None], ref.shape)
        step = 2.0 ** -10 + (0.0 if was_scale == 2.0 ** -4 else 2.0 ** -4) * np.abs(ref)
        assert np.all(np.abs(now - ref)[~w] <= np.where(moved, step, 0.0)[~w]), f"{name}: old slots"


@pytest.mark.parametrize("bits", [16, 8])
def test_append_writes_nothing_it_should_not(bits):
    """Bad pages, places past the table and bad source rows are skipped; their neighbours arrive."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(3)
    page, h, dim = 16, 2, 128
    kc, vc, ks, vs = make_pool(rs, 4, h, page, dim, bits)
    was = [f64(kc), f64(vc)]
    x = dev_bf16(wl.random_bf16(5, (60, h, dim)))
    cu, ctx = [0, 20, 40, 60], [0, 0, 20]
    table = np.array([[2, -1], [99, 1], [3, 3]], np.int32)             # the third sequence starts at 20 of 32: 12 fit
    rows = np.arange(60, dtype=np.int32)
    rows[3], rows[42] = -1, 60
    pace.cache_append(None, x, x, pace.KvCache(kc, vc, ks, vs), dev_i32(cu), dev_i32(ctx), dev_i32(table), 20, rows=dev_i32(rows))
    torch.cuda.synchronize()
    xs = wl.bf16_bits_to_f64(wl.random_bf16(5, (60, h, dim)))
    hit = np.zeros((4, page), bool)
    for pg, slot0, r0, n in ((2, 0, 0, 16), (1, 0, 36, 4), (3, 4, 40, 12)):
        for i in range(n):
            if r0 + i not in (3, 42):
                hit[pg, slot0 + i] = True
                for now, s in ((kc, ks), (vc, vs)):
                    val = f64(now)[pg, :, slot0 + i] * (1.0 if s is None else f64(s)[pg][:, None])
                    step = 2.0 ** -4 * np.abs(xs[r0 + i]) + 2.0 ** -10 * f64(s)[pg][:, None] if bits == 8 else 0.0
                    assert np.all(np.abs(val - xs[r0 + i]) <= step)
    for now, old, s in ((kc, was[0], ks), (vc, was[1], vs)):
        other = np.broadcast_to(~hit[:, None, :, None], old.shape).copy()
        other[3, :, :4] = False                                         # may have moved to a larger scale
        assert np.array_equal(f64(now)[other], old[other])


def test_append_values_that_are_not_finite_and_zeros():
    import torch
    from paper_2608_27206_amd import pace
    x = torch.zeros((6, 1, 128), dtype=torch.bfloat16, device="cuda")
    x[1, 0, 5], x[2, 0, 6], x[3, 0, 7], x[3, 0, 8] = float("inf"), float("nan"), 3.0, -float("inf")
    c = pace.KvCache(*(t for t in make_pool(np.random.default_rng(1), 3, 1, 16, 128, 8)))
    # sequence 0: one zero token, then (a second call) a tiny one; sequence 1: the others
    pace.cache_append(None, x, x, c, dev_i32([0, 1, 6]), dev_i32([0, 0]), dev_i32([[0], [1]]), 5)
    torch.cuda.synchronize()
    s, codes = f64(c.v_scale), f64(c.v)
    assert s[0, 0] == 2.0 ** -120 and np.all(codes[0, 0, 0] == 0)
    assert s[1, 0] == 2.0 ** -7 and codes[1, 0, 2, 7] == 384 and codes[1, 0, 0].size == 128      # 3 = 384 * 2^-7
    bad = np.isnan(codes[1, 0, :5])
    assert bad.sum() == 3 and bad[0, 5] and bad[1, 6] and bad[2, 8]
    tiny = torch.full((1, 1, 128), 2.0 ** -100, dtype=torch.bfloat16, device="cuda")
    pace.cache_append(None, tiny, tiny, c, dev_i32([0, 1, 1]), dev_i32([1, 0]), dev_i32([[0], [1]]), 1)
    torch.cuda.synchronize()
    s, codes = f64(c.v_scale), f64(c.v)
    assert np.all(codes[0, 0, 1] * s[0, 0] == 2.0 ** -100) and np.all(codes[0, 0, 0] == 0)


def test_append_scale_at_its_border():
    """448 * 2^e fits exactly, the next bf16 value does not; values near the largest bf16."""
    import torch
    from paper_2608_27206_amd import pace
    tops = [448.0, 450.0, 446.0, 448.0 * 2 ** -10, 450.0 * 2.0 ** -10, 3.38e38, 1e-38]
    x = torch.zeros((len(tops), 1, 80), dtype=torch.bfloat16, device="cuda")
    for i, t in enumerate(tops):
        x[i, 0, 3 * i] = -t
    n = len(tops)
    c = pace.KvCache(*make_pool(np.random.default_rng(1), n, 1, 16, 80, 8))
    pace.cache_append(None, x, x, c, dev_i32(np.arange(n + 1)), dev_i32([0] * n), dev_i32(np.arange(n)[:, None]), 1)
    torch.cuda.synchronize()
    for i in range(n):
        top = float(-x[i, 0, 3 * i].double())
        assert f64(c.k_scale)[i, 0] == oc.page_scale(top)
        got = -f64(c.k)[i, 0, 0, 3 * i] * f64(c.k_scale)[i, 0]
        assert abs(got - top) <= 2.0 ** -4 * top + 2.0 ** -10 * oc.page_scale(top)


# ---------------------------------------------------------------- attention
ATTEND = [
    # bits, page, heads (q, kv), dim, nq, lens, window, sinks
    (16, 16, (4, 2), 128, [1], [1], 0, 0),
    (16, 64, (28, 4), 128, [1, 1, 1, 1], [1, 64, 65, 1183], 0, 0),
    (8, 64, (28, 4), 128, [1, 1, 1, 1], [17, 63, 128, 1000], 0, 0),
    (16, 32, (16, 16), 80, [1, 1], [31, 600], 0, 0),
    (8, 16, (16, 4), 80, [1, 1, 1], [15, 16, 333], 0, 0),
    (8, 128, (5, 1), 80, [2, 3], [300, 3], 0, 0),
    (16, 256, (32, 8), 128, [5, 5], [700, 5], 0, 0),
    (16, 64, (17, 1), 128, [1, 2], [200, 100], 0, 0),
    (8, 256, (40, 2), 128, [3], [513], 0, 0),
    (16, 64, (28, 4), 128, [1, 0, 1], [0, 5, 70], 0, 0),                   # an empty sequence, one without queries
    (16, 64, (4, 2), 128, [5], [3], 0, 0),                                 # two queries before the first token
    (16, 32, (8, 2), 128, [70], [150], 0, 0),
    (8, 64, (28, 4), 128, [33, 1, 129], [33, 40, 200], 0, 0),
    (16, 64, (14, 2), 80, [100], [228], 0, 0),
    (16, 64, (28, 4), 128, [1, 1], [900, 30], 100, 4),
    (8, 16, (8, 2), 128, [1, 4], [777, 500], 64, 64),
    (8, 64, (8, 2), 128, [1], [640], 1, 0),                                # each query sees itself alone
    (16, 32, (8, 2), 128, [40], [300], 33, 5),
    (16, 64, (8, 2), 80, [150, 9], [400, 9], 130, 70),
    (16, 64, (8, 2), 128, [90], [90], 1000, 4),                            # a window longer than the context
    (16, 64, (8, 2), 128, [6], [200], 50, 500),                            # sinks past the end: all keys
    (8, 16, (4, 2), 128, [50], [77], 0, 0),                                # 33 to 128 rows of a KV head
    (8, 32, (16, 4), 80, [20, 11], [100, 300], 0, 0),
    (16, 128, (2, 1), 128, [60], [61], 0, 0),
    (16, 16, (3, 1), 80, [33], [500], 40, 20),
    (16, 64, (4, 2), 128, [40], [2500], 0, 0),                             # split keys, joined
    (8, 128, (8, 2), 128, [40], [1700], 0, 0),
    (8, 16, (4, 2), 80, [1, 2], [3000, 1500], 0, 0),
    (16, 32, (2, 2), 128, [1], [4097], 3000, 100),
    (8, 64, (4, 1), 128, [1] * 70, list(range(70)), 0, 0),                 # many sequences, lengths from 0
    # more than 128 rows of 32 KV heads in all: 256 rows per workgroup
    (16, 64, (64, 32), 128, [70, 3], [300, 200], 0, 0),
    (8, 64, (64, 32), 128, [129], [1500], 0, 0),                           # split keys, joined
    (16, 16, (32, 32), 80, [140], [150], 0, 0),
    (8, 32, (16, 8), 80, [150, 0, 1, 70], [700, 9, 300, 70], 0, 0),
    (16, 128, (16, 8), 128, [0, 133, 200, 66], [0, 133, 100, 260], 0, 0),  # one with queries before the first token
    (8, 16, (28, 4), 128, [40] * 8, [50, 40, 64, 65, 300, 41, 129, 77], 33, 5),
    (16, 64, (64, 32), 80, [100], [1400], 700, 70),
    (8, 256, (64, 32), 128, [65], [65], 20, 0),
]


def _attend_inputs(case, rs):
    bits, page, (hq, hkv), dim, nq, lens, window, sinks = case
    pages, table = make_table(rs, lens, page)
    kc, vc, ks, vs = make_pool(rs, pages, hkv, page, dim, bits)
    q = wl.f32_to_bf16_bits(1.5 * rs.standard_normal((sum(nq) + 2, hq, dim)).astype(np.float32))
    cu = np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)
    return pages, table, kc, vc, ks, vs, q, cu


def check_attention(o, lse, ref, dim, n):
    o_ref, lse_ref, spread, reach = ref
    score = (dim + 8) * 2.0 ** -24 * reach + 4e-6
    tol = (2.0 ** -8 + 2 * score.T[..., None]) * spread + 2.0 ** -8 * np.abs(o_ref)
    bad = np.abs(o[:n] - o_ref[:n]) > tol[:n]
    assert not bad.any(), f"o off at {np.argwhere(bad)[:4]}: {o[:n][bad][:4]} for {o_ref[:n][bad][:4]}"
    gone = lse_ref[:, :n] == -np.inf
    assert np.array_equal(lse[:, :n] == -np.inf, gone)
    off = np.abs(np.where(gone, 0.0, lse[:, :n]) - np.where(gone, 0.0, lse_ref[:, :n]))
    assert np.all(off <= score[:, :n] + 2.0 ** -22 * np.abs(np.where(gone, 0.0, lse_ref[:, :n])))


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"bits{c[0]}-p{c[1]}-h{c[2][0]}.{c[2][1]}-d{c[3]}-nq{c[4]}-len{c[5]}-w{c[6]}.{c[7]}")
def test_attention(case):
    import torch
    from paper_2608_27206_amd import pace
    bits, page, (hq, hkv), dim, nq, lens, window, sinks = case
    rs = np.random.default_rng(sum(map(ord, str(case))))
    pages, table, kc, vc, ks, vs, q, cu = _attend_inputs(case, rs)
    ref = oc.attention(wl.bf16_bits_to_f64(q), f64(kc), f64(vc), None if ks is None else f64(ks),
                       None if vs is None else f64(vs), cu, lens, table, page, dim ** -0.5, window, sinks)
    keep = held_slots(pages, table, lens, page)
    poison(kc, keep)
    poison(vc, keep)
    if ks is not None:
        dead = torch.from_numpy(~keep.any(1)).cuda()
        ks[dead], vs[dead] = float("nan"), float("inf")
    n = int(cu[-1])
    o = torch.full((n + 2, hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((hq, n + 2), 7.0, device="cuda")
    say(f"attend {case}")
    pace.cache_attention(dev_bf16(q), pace.KvCache(kc, vc, ks, vs), dev_i32(cu), dev_i32(lens), dev_i32(table), max(nq),
                         max(lens), window=window, sinks=sinks, o=o, lse=lse)
    torch.cuda.synchronize()
    check_attention(f64(o), f64(lse), ref, dim, n)
    assert np.all(f64(o)[n:] == 7.0) and np.all(f64(lse)[:, n:] == 7.0), "rows behind the last sequence changed"
    # without the LSE, and with looser bounds from the host, the outputs are within the same tolerance
    o2, none = pace.cache_attention(dev_bf16(q), pace.KvCache(kc, vc, ks, vs), dev_i32(cu), dev_i32(lens), dev_i32(table),
                                    n + 2, table.shape[1] * page, window=window, sinks=sinks, want_lse=False)
    assert none is None
    check_attention(f64(o2), f64(lse), ref, dim, n)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("nq,heads", [(1, (4, 2)), (3, (4, 2)), (40, (4, 2)), (200, (4, 2)), (130, (32, 16))])
def test_attention_bad_pages_count_as_unseen(bits, nq, heads):
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(11 * nq + bits)
    case = (bits, 16, heads, 128, [nq, 1], [210, 40], 0, 0)
    pages, table, kc, vc, ks, vs, q, cu = _attend_inputs(case, rs)
    table[0, [1, 5, 6]], table[1] = [-1, pages, 2 ** 31 - 1], -1          # the second sequence sees nothing
    ref = oc.attention(wl.bf16_bits_to_f64(q), f64(kc), f64(vc), None if ks is None else f64(ks),
                       None if vs is None else f64(vs), cu, [210, 40], table, 16, 128 ** -0.5)
    o, lse = pace.cache_attention(dev_bf16(q[:nq + 1]), pace.KvCache(kc, vc, ks, vs), dev_i32(cu), dev_i32([210, 40]), dev_i32(table),
                                  nq, 210)
    torch.cuda.synchronize()
    check_attention(f64(o), f64(lse), [ref[0][:nq + 1], ref[1][:, :nq + 1], ref[2][:nq + 1], ref[3][:, :nq + 1]], 128, nq + 1)
    assert np.all(f64(o)[nq] == 0) and np.all(f64(lse)[:, nq] == -np.inf)


@pytest.mark.parametrize("nq,heads", [(1, (4, 2)), (4, (4, 2)), (20, (4, 2)), (60, (4, 2)), (70, (22, 11))])
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -1.0, 0.0])
def test_attention_does_not_use_scales_past_the_end(nq, heads, scale):
    """Table entries behind a sequence's last page that name a page of NaN with a scale of anything."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(nq)
    lens = [nq + 49, 17 + nq, nq]
    pages, table, kc, vc, ks, vs, q, cu = _attend_inputs((8, 16, heads, 128, [nq] * 3, lens, 0, 0), rs)
    ref = oc.attention(wl.bf16_bits_to_f64(q), f64(kc), f64(vc), f64(ks), f64(vs), cu, lens, np.where(table < 0, 0, table), 16, 128 ** -0.5)
    used = set(table[table >= 0])
    dead = next(p for p in range(pages) if p not in used)
    table[table < 0] = dead
    kc.view(torch.uint8)[dead], vc.view(torch.uint8)[dead] = 0x7F, 0x7F
    ks[dead], vs[dead] = scale, scale
    o, lse = pace.cache_attention(dev_bf16(q[:3 * nq]), pace.KvCache(kc, vc, ks, vs), dev_i32(cu), dev_i32(lens), dev_i32(table), nq, max(lens))
    torch.cuda.synchronize()
    n = 3 * nq
    check_attention(f64(o), f64(lse), [ref[0][:n], ref[1][:, :n], ref[2][:n], ref[3][:, :n]], 128, n)


def test_nothing_to_do():
    import torch
    from paper_2608_27206_amd import pace
    c = pace.KvCache(*make_pool(np.random.default_rng(1), 2, 2, 16, 128, 16))
    x = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    out = pace.cache_append(x, x, x, c, dev_i32([0, 0]), dev_i32([0]), dev_i32([[0]]), 0)
    o, lse = pace.cache_attention(x, c, dev_i32([0, 0]), dev_i32([0]), dev_i32([[0]]), 0, 0)
    assert out.shape == o.shape == (0, 2, 128) and lse.shape == (2, 0)
    # a sequence without tokens or queries next to one with both
    y = dev_bf16(wl.random_bf16(3, (1, 2, 128)))
    pace.cache_append(None, y, y, c, dev_i32([0, 0, 1]), dev_i32([7, 0]), dev_i32([[1], [0]]), 1)
    o, lse = pace.cache_attention(y, c, dev_i32([0, 0, 1]), dev_i32([0, 1]), dev_i32([[1], [0]]), 1, 16)
    torch.cuda.synchronize()
    assert np.array_equal(f64(o), f64(y))          # one key: its value


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("bits,nq,heads", [(16, 6, (4, 2)), (8, 6, (4, 2)), (16, 90, (4, 2)), (8, 200, (4, 2)),
                                           (16, 200, (64, 32)), (8, 150, (32, 32))])
def test_hidden_keys_do_not_matter(bits, nq, heads, window, sinks):
    """NaN and infinities in the K and V of a token reach exactly the queries that see it: all others keep
    their bits."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(nq + window)
    L = nq + 130
    case = (bits, 32, heads, 128, [nq], [L], window, sinks)
    pages, table, kc, vc, ks, vs, q, cu = _attend_inputs(case, rs)
    args = (dev_i32(cu), dev_i32([L]), dev_i32(table), nq, L)
    dq = dev_bf16(q[:nq])
    base, lse0 = pace.cache_attention(dq, pace.KvCache(kc, vc, ks, vs), *args, window=window, sinks=sinks)
    for j in (L - 3, L - nq // 2, 50):
        pg, sl = int(table[0, j // 32]), j % 32
        for which in ("k", "v"):
            k2, v2 = kc.clone(), vc.clone()
            t = (k2 if which == "k" else v2)
            raw = t.view(torch.uint8 if bits == 8 else torch.int16)
            raw[pg, :, sl, ::7] = 0x7F if bits == 8 else 0x7F80          # e4m3 NaN, or bf16 infinity
            raw[pg, :, sl, 3] = 0x7F if bits == 8 else 0x7FC0
            say(f"hidden keys: bits {bits}, {nq} queries, window {window}, {which} of token {j}")
            o, lse = pace.cache_attention(dq, pace.KvCache(k2, v2, ks, vs), *args, window=window, sinks=sinks)
            torch.cuda.synchronize()
            place = L - nq + np.arange(nq)
            sees = (j <= place) & ((window == 0) | (j > place - window) | (j < sinks))
            same = (o.view(torch.int16) == base.view(torch.int16)).flatten(1).all(1).cpu().numpy()
            assert same[~sees].all(), f"queries {np.nonzero(~same & ~sees)[0][:5]} do not see token {j}"
            if which == "v":
                assert torch.equal(lse, lse0)
                # elements 0, 3, 7, ... of V are not finite: those of o are not either, the others stay
                assert not np.isfinite(f64(o)[sees][:, :, [0, 3, 7]]).any()
                assert np.isfinite(f64(o)[sees][:, :, [1, 2, 4]]).all()
            else:
                assert np.isnan(f64(lse).T[sees]).all()


def test_attention_scores_of_minus_infinity():
    """All seen keys score -inf: o = 0, LSE = -inf, as for a query that sees no key.  One finite key takes all."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(2)
    kc, vc, _, _ = make_pool(rs, 8, 1, 16, 128, 16)
    kc[:, :, :, 0] = float("-inf")
    q = torch.ones((2, 2, 128), dtype=torch.bfloat16, device="cuda")
    args = (dev_i32([0, 1, 2]), dev_i32([60, 61]), dev_i32([[0, 1, 2, 3], [4, 5, 6, 7]]), 1, 64)
    kc[5, 0, 3, 0] = 0.0
    o, lse = pace.cache_attention(q, pace.KvCache(kc, vc), *args)
    torch.cuda.synchronize()
    assert np.all(f64(o)[0] == 0) and np.all(f64(lse)[:, 0] == -np.inf)
    assert np.array_equal(f64(o)[1, 0], f64(vc)[5, 0, 3]) and np.isfinite(f64(lse)[:, 1]).all()


def test_attention_large_scores():
    """Scores of a few thousand: one key takes all, nothing overflows."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(6)
    case = (16, 64, (8, 2), 128, [1, 70], [500, 70], 0, 0)
    pages, table, kc, vc, _, _, q, cu = _attend_inputs(case, rs)
    kc *= 200
    ref = oc.attention(wl.bf16_bits_to_f64(q), f64(kc), f64(vc), None, None, cu, [500, 70], table, 64, 128 ** -0.5)
    o, lse = pace.cache_attention(dev_bf16(q), pace.KvCache(kc, vc), dev_i32(cu), dev_i32([500, 70]), dev_i32(table), 70, 500)
    torch.cuda.synchronize()
    check_attention(f64(o), f64(lse), ref, 128, 71)


# ---------------------------------------------------------------- 4-bit weights
W4 = [(1, 1, 32, 32, 0, 0), (1, 64, 128, 128, 1, 0), (3, 17, 96, 32, 1, 1), (1, 4608, 3584, 128, 0, 0), (5, 130, 1280, 64, 1, 2),
      (16, 100, 448, 64, 0, 1), (17, 33, 320, 64, 1, 0), (33, 250, 256, 128, 0, 2), (64, 77, 3424, 32, 1, 1),
      (65, 48, 640, 128, 1, 0), (150, 34, 192, 64, 0, 2), (2, 31, 14336, 128, 1, 0), (8, 2, 288, 32, 0, 2),
      # wider: two tiles a wave, fewer waves per column; odd widths; 9 to 16 rows; many splits
      (8, 8001, 512, 64, 1, 0), (12, 6000, 1056, 32, 0, 1), (16, 20002, 288, 32, 1, 2), (2, 28680, 384, 128, 0, 2),
      (11, 24593, 640, 64, 1, 0), (9, 16400, 128, 128, 0, 1), (5, 32784, 96, 32, 1, 0), (7, 200, 2080, 32, 1, 0),
      (40, 64, 14336, 64, 0, 1), (17, 130, 2016, 32, 1, 2), (64, 3000, 1152, 128, 1, 0), (128, 130, 1024, 128, 0, 2),
      # K in several chunks of x, with few and many columns; split K with up to 16 rows; K under 128
      (8, 5000, 4672, 64, 1, 1), (4, 300, 5152, 32, 0, 0), (13, 16400, 2304, 128, 1, 2), (16, 10000, 2080, 32, 0, 0),
      (10, 130, 8224, 32, 1, 2), (16, 4000, 4096, 128, 0, 1), (1, 77, 14336, 64, 1, 0), (8, 258, 8192, 128, 0, 2),
      (16, 31, 64, 64, 1, 0), (20, 31, 32, 32, 0, 0), (20, 30, 96, 32, 1, 2)]


@pytest.mark.parametrize("M,N,K,group,zero,epilogue", W4)
def test_w4(M, N, K, group, zero, epilogue):
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + N + K)
    x = wl.f32_to_bf16_bits(rs.standard_normal((M, K)).astype(np.float32))
    w = rs.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    s = wl.f32_to_bf16_bits(rs.uniform(0.002, 0.03, size=(N, K // group)).astype(np.float32))
    z = rs.integers(0, 16, size=(N, K // group), dtype=np.uint8) if zero else None
    bias = rs.standard_normal(N).astype(np.float32) if epilogue != 1 else None
    res = wl.f32_to_bf16_bits(rs.standard_normal((M, N)).astype(np.float32)) if epilogue == 1 else None
    ref, tol = oc.w4(wl.bf16_bits_to_f64(x), w, wl.bf16_bits_to_f64(s), z, group, bias,
                     None if res is None else wl.bf16_bits_to_f64(res), epilogue)
    say(f"w4 M={M} N={N} K={K} group={group}")
    cols = ref.shape[1]
    out = torch.full((M + 1, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    pace.gemm_w4(dev_bf16(x), torch.from_numpy(w).cuda(), dev_bf16(s), None if z is None else torch.from_numpy(z).cuda(),
                 bias=None if bias is None else dev_f32(bias), residual=None if res is None else dev_bf16(res),
                 epilogue=epilogue, out=out[:M])
    torch.cuda.synchronize()
    got = f64(out)
    bad = np.abs(got[:M] - ref) > 2.0 ** -8 * np.abs(ref) + tol
    assert not bad.any(), f"{bad.sum()} off, first {np.argwhere(bad)[:3]}: {got[:M][bad][:3]} for {ref[bad][:3]}"
    assert np.all(got[M] == 7.0)
