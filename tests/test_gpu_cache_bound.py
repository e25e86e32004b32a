"""Cache attention under a bound max_len that is not the longest length, as a captured step has it, and at the largest sizes."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_i32, say
from tests.test_gpu_cache import _attend_inputs, check_attention, f64, make_pool

pytestmark = pytest.mark.gpu

CASES = [  # bits, page, heads (q, kv), dim, nq, lens, window, sinks
    (16, 64, (8, 2), 128, [1] * 3, [3000, 700, 1500], 0, 0),                        # up to 16 rows of a KV head
    (8, 64, (8, 2), 128, [1] * 4, [900, 3333, 0, 17], 0, 0),
    (16, 32, (3, 1), 80, [1] * 70, [40 * i for i in range(70)], 0, 0),              # more sequences than a wave has lanes
    (8, 16, (2, 1), 80, [1] * 130, [1100] + [11 * i for i in range(129)], 0, 0),
    (16, 32, (32, 8), 128, [5, 3], [2500, 900], 0, 0),                              # up to 32
    (16, 64, (4, 2), 128, [40], [2500], 0, 0),                                      # up to 128
    (8, 128, (8, 2), 128, [40, 9], [1700, 300], 0, 0),
    (8, 64, (64, 32), 128, [129], [1500], 0, 0),                                    # more
    (16, 64, (28, 4), 128, [1, 1], [1900, 30], 700, 4),
    (16, 16, (8, 2), 80, [40, 3], [1300, 600], 500, 70),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"bits{c[0]}-p{c[1]}-h{c[2][0]}.{c[2][1]}-d{c[3]}-B{len(c[4])}-len{max(c[5])}-w{c[6]}")
def test_a_loose_bound_changes_nothing(case):
    """Against the oracle; and, where no window bounds the keys as well, the rows' keys are split into the parts that the exact
    bound gives them: the same slots of the workspace are written.  (Bits may differ: the join adds up to 8 planned parts in
    another order than more.)"""
    import torch
    from paper_2608_27206_amd import pace
    bits, page, (hq, hkv), dim, nq, lens, window, sinks = case
    rs = np.random.default_rng(sum(map(ord, str(case))))
    pages, table, kc, vc, ks, vs, q, cu = _attend_inputs(case, rs)
    bound = 1 << 17
    wide = np.full((len(lens), bound // page), -1, np.int32)
    wide[:, :table.shape[1]] = table
    cache = pace.KvCache(kc, vc, ks, vs)
    n = sum(nq)
    say(f"loose bound {case}")
    got = []
    for t, most in ((table, max(lens)), (wide, bound)):
        need = pace.lib().pace_cache_attention_workspace_size(n + 2, hq, hkv, dim, bits, len(lens), max(nq), most, window, sinks)
        assert need > 0
        ws = torch.full((need // 4,), -7, dtype=torch.int32, device="cuda")
        o, lse = pace.cache_attention(dev_bf16(q), cache, dev_i32(cu), dev_i32(lens), dev_i32(t), max(nq), most, window=window, sinks=sinks,
                                      workspace=ws.view(torch.uint8))
        torch.cuda.synchronize()
        parts = (ws.view(-1, n + 2, hq, dim + 4)[..., dim] != -7).sum(0)               # each row's parts: their maxima
        got.append((o[:n], lse[:, :n], parts))
    ref = oc.attention(wl.bf16_bits_to_f64(q), f64(kc), f64(vc), None if ks is None else f64(ks), None if vs is None else f64(vs),
                       cu, lens, table, page, dim ** -0.5, window, sinks)
    for o, lse, _ in got:
        check_attention(f64(o), f64(lse), (ref[0][:n], ref[1][:, :n], ref[2][:n], ref[3][:, :n]), dim, n)
    if window == 0:
        assert got[0][2].max() > 1 and torch.equal(got[0][2], got[1][2])


@pytest.mark.parametrize("debug", [False, True])
@pytest.mark.parametrize("nq", [3, 40, 2100])
def test_a_window_near_the_largest_length(nq, debug, monkeypatch):
    """A table of 2^31 - 1,024 tokens, a window one short of that, and queries before the first token: p - window passes -2^31
    for the earliest of 2,100 (they see nothing), and the others see all their keys."""
    import torch
    from paper_2608_27206_amd import pace
    if debug:
        monkeypatch.setenv("PACE_DEBUG", "1")
    rs = np.random.default_rng(nq)
    page, dim, n = 256, 80, 30
    kc, vc, ks, vs = make_pool(rs, 3, 1, page, dim, 16)
    q = wl.random_bf16(nq, (nq, 1, dim))
    pages = (2 ** 31 - 1024) // page
    table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 2
    say(f"window of {pages * page - 1}, {nq} queries of {n} tokens")
    o, lse = pace.cache_attention(dev_bf16(q), pace.KvCache(kc, vc), dev_i32([0, nq]), dev_i32([n]), table, nq, pages * page,
                                  window=pages * page - 1, sinks=5)
    torch.cuda.synchronize()
    ref = oc.attention(wl.bf16_bits_to_f64(q), f64(kc), f64(vc), None, None, [0, nq], [n], np.array([[2]]), page, dim ** -0.5)
    check_attention(f64(o), f64(lse), ref, dim, nq)


@pytest.mark.parametrize("heads,dim,bits", [(1, 128, 16), (2, 80, 8)])
def test_many_sequences_under_a_loose_bound(heads, dim, bits):
    """30,000 sequences of one query, lengths from 0, a table much wider than they are: nothing is split, and no sequence's call
    depends on how many others there are."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(heads)
    B, page = 30000, 16
    lens = rs.integers(0, 33, size=B).astype(np.int32)
    kc, vc, ks, vs = make_pool(rs, 64, heads, page, dim, bits)
    table = rs.integers(0, 64, size=(B, 64)).astype(np.int32)             # sequences may share what they read
    q = wl.random_bf16(5, (B, heads, dim))
    some = rs.permutation(B)[:200]
    say(f"{B} sequences, {heads} heads of {dim}, {bits} bits")
    o, lse = pace.cache_attention(dev_bf16(q), pace.KvCache(kc, vc, ks, vs), dev_i32(np.arange(B + 1)), dev_i32(lens), dev_i32(table), 1, 1024)
    torch.cuda.synchronize()
    ref = oc.attention(wl.bf16_bits_to_f64(q[some]), f64(kc), f64(vc), None if ks is None else f64(ks), None if vs is None else f64(vs),
                       np.arange(201), lens[some], table[some], page, dim ** -0.5)
    check_attention(f64(o)[some], f64(lse)[:, some], ref, dim, 200)
