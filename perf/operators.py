"""The operators of a decode step over a pruned context, as a serving program calls them.

After the selection a program keeps the rotated keys and values of the kept tokens in a paged cache
(``cache_append``), answers token by token with attention over that cache (``cache_attention``), and
reads the layers' weights in 4 bits (``gemm_w4``).  Shapes are those of
``paper_2608_27206_amd.workloads`` (28/4 heads of 128, rows of 3584, a 4K frame's 10,549 visual and
128 text tokens, of which 1,055 visual ones are kept) and generic ones beside them.

``run`` computes the plain form in 32-bit torch operations, or with ``own`` the framework's kernels.
"""
import math

import torch

own = False

DEV = "cuda"
THETA = 1.0e6                  # base of the rotation's frequencies
GOLDEN = 0.6180339887498949
E4M3_MAX = 448.0
MIN_EXP = -120                 # least exponent of an 8-bit page's scale
SECTIONS = {128: (16, 24, 24), 80: (8, 16, 16)}   # frequencies of the time, height and width axes


def listed():
    llm = {"hq": 28, "hkv": 4, "d": 128}
    return [
        # one token of one sequence: the shortest call, launch and latency
        {"name": "append_1", "op": "append", **llm, "B": 1, "new": 1, "ctx": 1183, "page": 64, "bits": 16, "axes": 3,
         "rows": 0},
        # a decode step of 64 sequences into 8-bit pages that already hold tokens
        {"name": "append_64_8bit", "op": "append", **llm, "B": 64, "new": 1, "ctx": 700, "page": 64, "bits": 8,
         "axes": 3, "rows": 0},
        # the whole context of a 4K frame written at once after the prefill's projections
        {"name": "append_4k_8bit", "op": "append", **llm, "B": 1, "new": 10677, "ctx": 0, "page": 64, "bits": 8,
         "axes": 3, "rows": 0},
        # one token over the pruned 4K context: the shortest attention call
        {"name": "attend_pruned", "op": "attend", **llm, "B": 1, "nq": 1, "len": 1183, "page": 64, "bits": 16,
         "window": 0, "sinks": 0},
        # a serving batch of unequal contexts up to 16,384 tokens in 8 bits
        {"name": "attend_48_8bit", "op": "attend", **llm, "B": 48, "nq": 1, "len": 16384, "page": 64, "bits": 8,
         "window": 0, "sinks": 0},
        # one long context of odd length
        {"name": "attend_long", "op": "attend", **llm, "B": 1, "nq": 1, "len": 131071, "page": 128, "bits": 16,
         "window": 0, "sinks": 0},
        # streaming: the last 4,096 tokens and the first 64 of contexts up to 32,768
        {"name": "attend_window_8bit", "op": "attend", **llm, "B": 24, "nq": 1, "len": 32768, "page": 64, "bits": 8,
         "window": 4096, "sinks": 64},
        # checking five drafted tokens of eight sequences
        {"name": "attend_draft", "op": "attend", "hq": 32, "hkv": 8, "d": 128, "B": 8, "nq": 5, "len": 8191,
         "page": 32, "bits": 16, "window": 0, "sinks": 0},
        # the last 1,024 tokens of a 4K frame's context over the cached rest: many query rows
        {"name": "attend_chunk", "op": "attend", **llm, "B": 1, "nq": 1024, "len": 10677, "page": 64, "bits": 16,
         "window": 0, "sinks": 0},
        # one row through the fused query, key and value projection
        {"name": "w4_qkv_1", "op": "w4", "M": 1, "N": 4608, "K": 3584, "group": 128, "zero": 0, "epilogue": 0},
        # eight rows through gate and up with their product in the epilogue
        {"name": "w4_gate_up_8", "op": "w4", "M": 8, "N": 28672, "K": 3584, "group": 128, "zero": 1, "epilogue": 2},
        # a batch of 48 rows through the down projection, added to the residual
        {"name": "w4_down_48", "op": "w4", "M": 48, "N": 3584, "K": 14336, "group": 64, "zero": 0, "epilogue": 1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    caps = {}
    for c in listed():
        w = work(c)
        for k in w:
            caps[c["op"], k] = max(caps.get((c["op"], k), 0), w[k])
    while True:
        op = rng.choice(["append", "append", "attend", "attend", "attend", "w4", "w4"])
        if op == "w4":
            g = rng.choice([32, 64, 128])
            e = rng.randrange(3)
            n = _log(rng, 64, 28672)
            c = {"op": op, "M": _log(rng, 1, 64), "N": n + n % 2 if e == 2 else n,
                 "K": max(1, _log(rng, 256, 14336) // g) * g, "group": g, "zero": rng.randrange(2), "epilogue": e}
        else:
            hq, hkv, d = rng.choice([(28, 4, 128), (28, 4, 128), (8, 2, 128), (32, 8, 128), (16, 16, 80), (16, 4, 80)])
            c = {"op": op, "hq": hq, "hkv": hkv, "d": d, "page": rng.choice([16, 32, 64, 128]),
                 "bits": rng.choice([8, 16])}
            if op == "append":
                decode = rng.random() < 0.5
                c.update(B=_log(rng, 1, 64) if decode else _log(rng, 1, 4),
                         new=_log(rng, 1, 4) if decode else _log(rng, 16, 10677), ctx=_log(rng, 1, 1500) - 1,
                         axes=rng.choice([1, 3]), rows=rng.randrange(2))
            else:
                many = rng.random() < 0.3
                n = _log(rng, 1, 131072)
                c.update(B=_log(rng, 1, 3) if many else _log(rng, 1, 64),
                         nq=_log(rng, 16, 1024) if many else rng.choice([1, 1, 1, 2, 5, 8]), len=n,
                         window=rng.choice([0, 0, _log(rng, 16, 8192)]), sinks=rng.choice([0, 4, 64]))
        w = work(c)
        if all(w[k] <= caps[op, k] for k in w) and c.get("B", 1) * c.get("len", 1) <= 32 * 32768:
            return c


def _spread(n, count, least):
    """`count` sizes up to n, the first of them n, spread over [0.2 n, n]."""
    return [max(least, n if b == 0 else int(round(n * (0.2 + 0.8 * ((b * GOLDEN) % 1.0))))) for b in range(count)]


def _lens(c):
    """Per sequence: cached tokens and query tokens (attend)."""
    n = _spread(c["len"], c["B"], 1)
    return n, [min(a, b) for a, b in zip(_spread(c["nq"], c["B"], 1), n)]


def _news(c):
    """Per sequence: tokens in the cache before and new ones (append)."""
    return _spread(c["ctx"], c["B"], 0), _spread(c["new"], c["B"], 1)


def _visible(p, w, s):
    """Keys that the query at place p sees, of window w (0: all) and s sinks."""
    if not w or p < w:
        return p + 1
    return w + min(s, p + 1 - w)


def work(case):
    c = case
    if c["op"] == "w4":
        M, N, K = c["M"], c["N"], c["K"]
        out = M * (N // 2 if c["epilogue"] == 2 else N) * 2
        b = N * K // 2 + N * (K // c["group"]) * (3 if c["zero"] else 2) + M * K * 2 + out
        return {"bytes": b + (out if c["epilogue"] == 1 else 0) + 4 * N, "flops": 2 * M * N * K}
    e = 1 if c["bits"] == 8 else 2
    if c["op"] == "append":
        n = sum(_news(c)[1])
        rot = n * c["d"] * (c["hq"] + c["hkv"])
        return {"bytes": n * c["d"] * (4 * c["hq"] + c["hkv"] * (4 + 2 * e)) + n * c["axes"] * 4, "flops": 3 * rot}
    kept, pairs = 0, 0
    for n, nq in zip(*_lens(c)):
        w, s = c["window"], c["sinks"]
        first = n - nq - w + 1                   # first key in the window of the sequence's first query
        kept += n if not w or first <= s else n - first + s
        pairs += sum(_visible(p, w, s) for p in range(n - nq, n))
    rows = sum(_lens(c)[1]) * c["hq"]
    return {"bytes": kept * c["hkv"] * c["d"] * 2 * e + rows * (c["d"] * 4 + 4), "flops": 4 * c["d"] * c["hq"] * pairs}


# ---------------------------------------------------------------- inputs
def _offsets(n):
    t = torch.zeros(len(n) + 1, dtype=torch.int64)
    t[1:] = torch.cumsum(torch.tensor(n), 0)
    return t.to(torch.int32).to(DEV)


def _i32(n):
    return torch.tensor(n, dtype=torch.int32, device=DEV)


def _pool(c, lens, g):
    """A page pool with keys and values of unit variance (a few keys of three times that) and a table of
    pages in random order; 8-bit pages hold codes and a power-of-two scale for each page and head."""
    per = [-(-n // c["page"]) for n in lens]
    pages, most = max(1, sum(per)) + 3, max(1, max(per))
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = torch.tensor([0] + per[:-1], device=DEV).cumsum(0)[:, None] + torch.arange(most, device=DEV)[None]
    table = order[at.clamp(max=pages - 1)].contiguous()
    out = {"table": table}
    for name in ("k", "v"):
        x = torch.randn(pages, c["hkv"], c["page"], c["d"], generator=g, device=DEV)
        if name == "k":
            x *= 1.0 + 2.0 * (torch.rand(pages, c["hkv"], c["page"], 1, generator=g, device=DEV) < 0.02)
        if c["bits"] == 8:
            top = x.abs().amax((2, 3))
            m, ex = torch.frexp(top)
            s = torch.ldexp(torch.ones_like(top), ex - 9 + (m > 0.875).int())
            out[name + "_pool"] = (x / s[:, :, None, None]).to(torch.float8_e4m3fn)
            out[name + "_scale"] = s
        else:
            out[name + "_pool"] = x.to(torch.bfloat16)
        del x
    return out


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rand = lambda *n: torch.randn(*n, generator=g, device=DEV)   # noqa: E731
    s = {"case": c}
    if c["op"] == "w4":
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = rand(M, K).to(torch.bfloat16)
        s["w"] = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
        s["scale"] = ((0.5 + torch.rand(N, K // c["group"], generator=g, device=DEV)) * 0.2 / math.sqrt(K)).to(torch.bfloat16)
        s["zero"] = torch.randint(5, 12, (N, K // c["group"]), generator=g, device=DEV, dtype=torch.uint8) if c["zero"] else None
        s["bias"] = rand(N) * 0.02 if c["epilogue"] != 1 else None
        s["residual"] = rand(M, N).to(torch.bfloat16) if c["epilogue"] == 1 else None
        return s
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["op"] == "attend":
        lens, nq = _lens(c)
        s.update(_pool(c, lens, g))
        s["q"] = (1.5 * rand(sum(nq), hq, d)).to(torch.bfloat16)
        s["cu"], s["len"] = _offsets(nq), _i32(lens)
        s["max_q"], s["max_len"] = max(nq), max(lens)
        return s
    ctx, new = _news(c)
    s.update(_pool(c, [a + b for a, b in zip(ctx, new)], g))
    n = sum(new)
    src = n if not c["rows"] else 3 * n          # with rows: a third of the source rows is kept, in order
    s["rows"] = None if not c["rows"] else torch.randperm(src, generator=g, device=DEV)[:n].sort().values.to(torch.int32)
    qkv = rand(src, (hq + 2 * hkv) * d).to(torch.bfloat16)       # the fused projection's rows
    s["q"] = qkv[:, :hq * d].view(src, hq, d)
    s["k"] = qkv[:, hq * d:(hq + hkv) * d].view(src, hkv, d)
    s["v"] = qkv[:, (hq + hkv) * d:].view(src, hkv, d)
    s["cu"], s["ctx"], s["max_new"] = _offsets(new), _i32(ctx), max(new)
    at = torch.randint(0, 100000, (1,), generator=g, device=DEV) + torch.arange(src, device=DEV)
    s["pos"] = (at[None] if c["axes"] == 1 else torch.stack([at, at // 137, at % 137 + at // 4])).to(torch.int32).contiguous()
    s["freq"] = (THETA ** (-torch.arange(d // 2, device=DEV, dtype=torch.float64) * 2 / d)).float()
    return s


# ---------------------------------------------------------------- plain forms
def _axis(c):
    """The position axis of each frequency."""
    if c["axes"] == 1:
        return torch.zeros(c["d"] // 2, dtype=torch.int64, device=DEV)
    return torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(SECTIONS[c["d"]], device=DEV))


def _rotated(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_append(s):
    c, P = s["case"], s["case"]["page"]
    n = int(s["q"].shape[0]) if s["rows"] is None else int(s["rows"].shape[0])
    src = torch.arange(n, device=DEV) if s["rows"] is None else s["rows"].long()
    r = torch.arange(n, device=DEV)
    b = torch.searchsorted(s["cu"].long(), r, right=True) - 1
    place = s["ctx"].long()[b] + r - s["cu"].long()[b]
    page, slot = s["table"].long()[b, place // P], place % P
    angle = s["pos"].double()[_axis(c)].t()[src] * s["freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = {"q": _rotated(s["q"][src], cos, sin).to(torch.bfloat16), "k": s["k_pool"], "v": s["v_pool"]}
    for name, x in (("k", _rotated(s["k"][src], cos, sin)), ("v", s["v"][src].float())):
        pool = s[name + "_pool"]
        if c["bits"] == 16:
            pool[page, :, slot] = x.to(torch.bfloat16)
            continue
        scale = s[name + "_scale"]
        at = torch.unique(page)                                  # the pages that get tokens
        of = torch.searchsorted(at, page)
        first = torch.full((len(at),), P, device=DEV).scatter_reduce_(0, of, slot, "amin")   # first new slot of each
        top = torch.zeros(len(at), x.shape[1], device=DEV).scatter_reduce_(0, of[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        m, ex = torch.frexp(top)                                 # top = m 2^ex, m in [1/2, 1); 448 = 0.875 * 2^9
        need = torch.ldexp(torch.ones_like(top), torch.where(top > 0, (ex - 9 + (m > 0.875).int()).clamp(min=MIN_EXP), MIN_EXP))
        old = scale[at]
        new = torch.where(first[:, None] > 0, torch.maximum(old, need), need)
        held = (torch.arange(P, device=DEV) < first[:, None])[:, None, :, None]
        codes = pool[at].float()
        codes = torch.where(held, codes * (old / new)[:, :, None, None], codes)
        pool[at] = codes.to(torch.float8_e4m3fn)
        scale[at] = new
        pool.view(torch.uint8)[page, :, slot] = (x / scale[page][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        out[name + "_scale"] = scale
    return out


def _plain_attend(s):
    c, P, L = s["case"], s["case"]["page"], s["max_len"]
    B, hq, hkv, d = c["B"], c["hq"], c["hkv"], c["d"]
    j = torch.arange(L, device=DEV)
    page, slot = s["table"].long()[:, :-(-L // P)].repeat_interleave(P, 1)[:, :L], (j % P).expand(B, L)
    k, v = s["k_pool"][page, :, slot].float(), s["v_pool"][page, :, slot].float()      # [B, L, hkv, d]
    if c["bits"] == 8:
        k, v = k * s["k_scale"][page][..., None], v * s["v_scale"][page][..., None]
    nq, cu, most = s["cu"].diff().long(), s["cu"].long(), s["max_q"]
    i = torch.arange(most, device=DEV)
    row = (cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)            # padded query rows
    q = s["q"][row].float().view(B, most, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, d)
    p = (s["len"].long() - nq)[:, None] + i                             # their places
    see = j <= p[..., None]
    if c["window"]:
        see &= (j > p[..., None] - c["window"]) | (j < c["sinks"])
    see = see[:, None, :, None].expand(B, hkv, most, hq // hkv, L).reshape(B, hkv, -1, L)
    kept = (j < s["len"][:, None])[:, :, None, None]                    # slots past a sequence's end hold anything
    x = torch.matmul(q, torch.where(kept, k, 0.0).permute(0, 2, 3, 1).contiguous()) / math.sqrt(d)
    x = x.masked_fill(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, torch.where(kept, v, 0.0).permute(0, 2, 1, 3).contiguous()) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    real = i < nq[:, None]
    o = o.view(B, hkv, most, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, most, hq, d)[real]
    lse = lse.view(B, hkv, most, hq // hkv).permute(0, 2, 1, 3).reshape(B, most, hq)[real]
    return {"o": o.to(torch.bfloat16), "lse": lse.t().contiguous()}


def _plain_w4(s):
    c = s["case"]
    q = torch.stack([s["w"] & 15, s["w"] >> 4], -1).view(c["N"], -1, c["group"]).float()
    z = 8.0 if s["zero"] is None else s["zero"].float()[..., None]
    y = s["x"].float() @ ((q - z) * s["scale"].float()[..., None]).view(c["N"], c["K"]).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["epilogue"] == 1:
        y = y + s["residual"].float()
    if c["epilogue"] == 2:
        g, u = y[:, 0::2], y[:, 1::2]
        y = g / (1 + torch.exp(-g)) * u
    return y.to(torch.bfloat16)


def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "w4": _plain_w4}[c["op"]](s)
    from paper_2608_27206_amd import pace
    if c["op"] == "w4":
        return pace.gemm_w4(s["x"], s["w"], s["scale"], s["zero"], bias=s["bias"], residual=s["residual"], epilogue=c["epilogue"])
    cache = pace.KvCache(s["k_pool"], s["v_pool"], s.get("k_scale"), s.get("v_scale"))
    if c["op"] == "attend":
        o, lse = pace.cache_attention(s["q"], cache, s["cu"], s["len"], s["table"], s["max_q"], s["max_len"],
                                      window=c["window"], sinks=c["sinks"])
        return {"o": o, "lse": lse}
    q = pace.cache_append(s["q"], s["k"], s["v"], cache, s["cu"], s["ctx"], s["table"], s["max_new"], positions=s["pos"],
                          inv_freq=s["freq"], sections=SECTIONS[c["d"]] if c["axes"] == 3 else None, rows=s["rows"])
    out = {"q": q, "k": cache.k, "v": cache.v}
    if c["bits"] == 8:
        out.update(k_scale=cache.k_scale, v_scale=cache.v_scale)
    return out


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "w4":
        w = torch.empty(c["N"], c["K"], dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = s["w"] % 16, s["w"] // 16
        for g in range(c["K"] // c["group"]):
            part = w[:, g * c["group"]:(g + 1) * c["group"]]
            part -= 8 if s["zero"] is None else s["zero"][:, g:g + 1]
            part *= s["scale"][:, g:g + 1].double()
        y = torch.mm(s["x"].double(), w.t())
        y += 0 if s["bias"] is None else s["bias"].double()
        y += 0 if s["residual"] is None else s["residual"].double()
        return y if c["epilogue"] != 2 else torch.nn.functional.silu(y[:, ::2]) * y[:, 1::2]
    P, d, group, cu = c["page"], c["d"], c["hq"] // c["hkv"], s["cu"].tolist()
    if c["op"] == "attend":
        o = torch.zeros(cu[-1], c["hq"], d, dtype=torch.float64, device=DEV)
        lse = torch.full((c["hq"], cu[-1]), -math.inf, dtype=torch.float64, device=DEV)
        for b, n in enumerate(s["len"].tolist()):
            own_pages = s["table"][b, :-(-n // P)].long()
            wide = []
            for name in ("k", "v"):
                x = s[name + "_pool"].view(torch.uint8 if c["bits"] == 8 else torch.bfloat16)[own_pages]
                if c["bits"] == 8:
                    x = x.view(torch.float8_e4m3fn).double() * s[name + "_scale"][own_pages].double()[:, :, None, None]
                wide.append(x.double().transpose(0, 1).reshape(c["hkv"], -1, d)[:, :n])
            place = torch.arange(n - (cu[b + 1] - cu[b]), n, device=DEV)[:, None]
            key = torch.arange(n, device=DEV)[None]
            hidden = key > place
            if c["window"]:
                hidden |= (place - key >= c["window"]) & (key >= c["sinks"])
            for h in range(c["hq"]):
                k, v = wide[0][h // group], wide[1][h // group]
                x = torch.mm(s["q"][cu[b]:cu[b + 1], h].double(), k.t()) * d ** -0.5
                x[hidden] = -math.inf
                lse[h, cu[b]:cu[b + 1]] = torch.logsumexp(x, 1)
                o[cu[b]:cu[b + 1], h] = torch.mm(torch.softmax(x, 1), v)
        return {"o": o, "lse": lse}
    rows = range(s["q"].shape[0]) if s["rows"] is None else s["rows"].tolist()
    axis = [0] * (d // 2) if c["axes"] == 1 else [a for a in range(3) for _ in range(SECTIONS[d][a])]
    at = torch.tensor(list(rows), device=DEV)
    turn = torch.polar(torch.ones(len(at), d // 2, dtype=torch.float64, device=DEV),
                       torch.stack([s["pos"][a][at].double() * f for a, f in zip(axis, s["freq"].double())], 1))[:, None]
    rotate = lambda x: (lambda y: torch.cat([y.real, y.imag], -1))(torch.complex(*x.double().chunk(2, -1)) * turn)   # noqa: E731
    out = {"q": rotate(s["q"][at])}
    for name, x in (("k", rotate(s["k"][at])), ("v", s["v"][at].double())):
        eight = c["bits"] == 8
        pool, scale = s[name + "_pool"].double(), s[name + "_scale"].double() if eight else None
        for b, n in enumerate(s["ctx"].tolist()):
            done = cu[b]
            while done < cu[b + 1]:
                slot, page = n % P, int(s["table"][b, n // P])
                take = min(P - slot, cu[b + 1] - done)
                part = x[done:done + take].transpose(0, 1)                 # [hkv, take, d]
                if eight:
                    top = part.abs().amax((1, 2)).clamp(min=448 * 2.0 ** MIN_EXP)
                    need = 2.0 ** torch.ceil(torch.log2(top / 448))
                    if slot:
                        need = torch.maximum(need, scale[page])
                        pool[page, :, :slot] *= (scale[page] / need)[:, None, None]
                    scale[page] = need
                    part = part / need[:, None, None]
                pool[page, :, slot:slot + take] = part
                done, n = done + take, n + take
        out[name] = pool
        if eight:
            out[name + "_scale"] = scale
    return out
