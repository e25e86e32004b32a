"""What the cache and 4-bit calls refuse, through the C ABI before any launch (CPU: no pointer is read)."""
import ctypes

import pytest

from tests.test_abi import pace

INT3 = ctypes.c_int * 3
P = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1008)


def cache(**kw):
    c = dict(k=0x1000, v=0x1000, k_scale=0x1000, v_scale=0x1000, num_pages=8, heads=2, page=64, dim=128, bits=8)
    c.update(kw)
    return ctypes.byref(pace._KvCacheStruct(*(c[n] for n, _ in pace._KvCacheStruct._fields_)))


def append(c=None, **kw):
    a = dict(q=P, qs=1024, k=P, ks=1024, v=P, vs=1024, n_src=4, Hq=4, rows=None, cu=P, B=1, n_new=4, max_new=4, ctx=P,
             table=P, max_pages=4, pos=P, axes=1, sections=None, freq=P, cache=c or cache(), q_out=P, stream=None)
    a.update(kw)
    return pace.lib().pace_cache_append(*a.values()), pace.lib().pace_last_error().decode()


def attend(c=None, **kw):
    a = dict(q=P, n_q=4, Hq=4, cache=c or cache(), cu=P, B=1, max_q=4, len=P, max_len=100, table=P, max_pages=4, window=0,
             sinks=0, scale=0.1, o=P, lse=None, ws=None, wsb=0, stream=None)
    a.update(kw)
    return pace.lib().pace_cache_attention(*a.values()), pace.lib().pace_last_error().decode()


def w4(**kw):
    a = dict(x=P, w=P, scale=P, zero=None, bias=None, residual=None, C=P, M=1, N=8, K=128, group=64, epilogue=0, ws=None, wsb=0, stream=None)
    a.update(kw)
    return pace.lib().pace_gemm_w4(*a.values()), pace.lib().pace_last_error().decode()


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad,status,word", [
    (dict(k=None), 1, "null"), (dict(v=None), 1, "null"), (dict(bits=4), 1, "bits"), (dict(k_scale=None), 1, "scale"),
    (dict(v_scale=None), 1, "scale"), (dict(k=0x1008), 1, "aligned"), (dict(num_pages=0), 1, "num_pages"),
    (dict(heads=0), 1, "heads"), (dict(page=8), 1, "page"), (dict(page=48), 1, "page"), (dict(page=512), 1, "page"),
    (dict(page=0), 1, "page"), (dict(page=-64), 1, "page"), (dict(dim=64), 2, "head dim")])
def test_caches(call, bad, status, word):
    st, msg = call(cache(**bad))
    assert st == status and word in msg


@pytest.mark.parametrize("call", [append, attend])
def test_tables(call):
    assert call(table=None)[0] == 1 and call(max_pages=0)[0] == 1 and call(B=0)[0] == 1
    assert call(max_pages=1 << 25)[0] == 1        # 2^25 pages of 64 tokens reach 2^31


@pytest.mark.parametrize("bad,word", [
    (dict(k=None), "null"), (dict(v=None), "null"), (dict(cu=None), "null"), (dict(ctx=None), "null"),
    (dict(q_out=None), "q_out"), (dict(Hq=0), "Hq"), (dict(q=ODD), "aligned"), (dict(v=ODD), "aligned"), (dict(q_out=ODD), "aligned"),
    (dict(max_new=5), "max_new"), (dict(n_new=5), "n_new"), (dict(n_src=-1), "n_src"), (dict(max_new=-1), "max_new"),
    (dict(ks=248), "strides"), (dict(vs=260), "strides"), (dict(qs=504), "strides"), (dict(ks=0), "strides"),
    (dict(pos=None), "together"), (dict(freq=None), "together"), (dict(axes=2), "axes"), (dict(axes=3), "sections"),
    (dict(axes=3, sections=INT3(16, 24, 23)), "sections"), (dict(axes=3, sections=INT3(-16, 56, 24)), "sections")])
def test_append(bad, word):
    st, msg = append(**bad)
    assert st == 1 and word in msg


def test_nothing_to_append_is_no_error():
    assert append(n_new=0, max_new=0)[0] == 0 and append(max_new=0)[0] == 0 and append(n_src=0, n_new=0, max_new=0)[0] == 0


@pytest.mark.parametrize("bad,word", [
    (dict(q=None), "null"), (dict(o=None), "null"), (dict(cu=None), "null"), (dict(len=None), "null"), (dict(q=ODD), "aligned"),
    (dict(o=ODD), "aligned"), (dict(Hq=3), "Hq"), (dict(Hq=0), "Hq"), (dict(max_q=5), "max_q"), (dict(max_len=257), "max_len"),
    (dict(max_len=-1), "max_len"), (dict(window=-1), "window"), (dict(sinks=-1), "sinks"), (dict(scale=0.0), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(n_q=-1, max_q=-1), "n_q")])
def test_attention(bad, word):
    st, msg = attend(**bad)
    assert st == 1 and word in msg


def test_no_queries_is_no_error():
    assert attend(n_q=0, max_q=0)[0] == 0 and attend(max_q=0)[0] == 0


def test_attention_workspace():
    size = pace.lib().pace_cache_attention_workspace_size
    need = size(1, 28, 4, 128, 8, 1, 1, 131072, 0, 0)
    if need:                                   # a long context of one row is split: its parts need room
        wide = dict(c=cache(heads=4), Hq=28, n_q=1, max_q=1, max_len=131072, max_pages=2048)
        st, msg = attend(**wide)
        assert st == 3 and "workspace" in msg
        st, msg = attend(ws=P, wsb=need - 1, **wide)
        assert st == 3 and "workspace" in msg
        st, msg = attend(ws=ODD, wsb=need, **wide)
        assert st == 1 and "aligned" in msg
    for bad in ((-1, 28, 4, 128, 8, 1, 1, 9999, 0, 0), (1, 27, 4, 128, 8, 1, 1, 9999, 0, 0), (1, 28, 0, 128, 8, 1, 1, 9999, 0, 0),
                (1, 28, 4, 128, 4, 1, 1, 9999, 0, 0), (1, 28, 4, 128, 8, 0, 1, 9999, 0, 0), (1, 28, 4, 128, 8, 1, 1, -5, 0, 0)):
        assert size(*bad) == 0


@pytest.mark.parametrize("bad,word", [
    (dict(x=None), "null"), (dict(w=None), "null"), (dict(scale=None), "null"), (dict(C=None), "null"), (dict(epilogue=3), "epilogue"),
    (dict(epilogue=-1), "epilogue"), (dict(epilogue=1), "residual"), (dict(epilogue=2, N=7), "even"), (dict(group=16), "group"),
    (dict(group=0), "group"), (dict(K=96), "K="), (dict(K=0), "K="), (dict(M=0), "M="), (dict(N=0), "N="), (dict(x=ODD), "aligned"),
    (dict(w=ODD), "aligned"), (dict(M=1 << 24, K=128), "2 GiB"), (dict(M=65536), "65,535"), (dict(N=1 << 26, K=128), "2 GiB")])
def test_w4(bad, word):
    st, msg = w4(**bad)
    assert st == 1 and word in msg


def test_w4_workspace():
    size = pace.lib().pace_gemm_w4_workspace_size
    assert size(1, 4608, 3584) == 0 and size(8, 28672, 3584) == 0 and size(0, 8, 128) == 0 and size(1, -8, 128) == 0
    for M in (1, 48):                              # long rows of few columns: K is split
        need = size(M, 64, 14336)
        assert need > 0 and need % (M * 64 * 4) == 0
        for ws, wsb in ((None, 0), (P, need - 1)):
            st, msg = w4(M=M, N=64, K=14336, ws=ws, wsb=wsb)
            assert st == 3 and "workspace" in msg
        st, msg = w4(M=M, N=64, K=14336, ws=ODD, wsb=need)
        assert st == 1 and "aligned" in msg


def test_binding_refuses_what_it_cannot_pass_on():
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(pace.PaceError, match="GPU"):
        pace.KvCache(k, k)
    with pytest.raises(pace.PaceError, match="one shape"):
        pace.KvCache(k, k[:2])
    with pytest.raises(pace.PaceError, match="cache type"):
        pace.KvCache(k.half(), k.half())
    k8 = k.to(torch.float8_e4m3fn)
    with pytest.raises(pace.PaceError, match="scales"):
        pace.KvCache(k8, k8)
    with pytest.raises(pace.PaceError, match="scales"):
        pace.KvCache(k8, k8, torch.ones(4, 2), torch.ones(2, 4))
    x, w = torch.zeros((1, 128), dtype=torch.bfloat16), torch.zeros((4, 64), dtype=torch.uint8)
    with pytest.raises(pace.PaceError, match="GPU"):
        pace.gemm_w4(x, w, torch.ones((4, 2), dtype=torch.bfloat16))


BIG = 2 ** 31 - 1


def test_sizes_past_32_bits_are_refused():
    """Products of counts that pass 2^31, or wrap to something small: an error, no division by what is left."""
    for bad in (dict(n_src=BIG, n_new=BIG, max_new=1), dict(n_src=BIG, n_new=BIG, max_new=BIG), dict(B=BIG, n_src=1 << 20, n_new=1 << 20, max_new=1 << 20),
                dict(B=1 << 30, max_new=4), dict(Hq=1 << 24, qs=1 << 31)):
        st, msg = append(**bad)
        assert st == 1 and "too many" in msg, bad
    st, msg = append(c=cache(heads=1 << 24), ks=1 << 31, vs=1 << 31)
    assert st == 1 and "too many" in msg
    for bad in (dict(n_q=BIG, max_q=BIG), dict(n_q=BIG, max_q=1 << 29, Hq=4), dict(B=BIG), dict(B=1 << 29, max_q=0), dict(n_q=1 << 30, max_q=1 << 30, Hq=BIG - 1),
                dict(B=BIG, n_q=BIG, max_q=BIG, Hq=BIG - 1)):
        st, msg = attend(**bad)
        assert st == 1 and "too many" in msg, bad
    size = pace.lib().pace_cache_attention_workspace_size
    for B, n, hq, heads in ((BIG, 1, 4, 4), (1, BIG, 4, 4), (1, 1 << 30, 1 << 20, 1 << 10), (1 << 16, 1 << 16, 1 << 30, 1), (BIG, BIG, BIG, 1), (1, 1, BIG, BIG)):
        assert size(n, hq, heads, 128, 16, B, n, 4096, 0, 0) >= 0
    size = pace.lib().pace_gemm_w4_workspace_size
    for M, N, K in ((1 << 30, 1 << 30, 128), (BIG, BIG, BIG), (1, BIG, 128), (1 << 24, 128, 128), (17, BIG, 1), (BIG, 1, 1)):
        assert size(M, N, K) == 0
