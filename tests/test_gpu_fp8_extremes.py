"""The 8-bit operators at the ends of fp32's range, against the float64 oracle."""
import numpy as np
import pytest

from oracle import fp8 as o8
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, say
from tests.test_gpu_cache import f64
from tests.test_gpu_fp8 import bits_of, check_norm, check_product, make_codes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("M,K", [(4, 16), (4, 1296), (1027, 1024), (1026, 2064), (4, 3584), (3, 8192), (3, 16384), (2, 65536)])
def test_norm_of_rows_whose_squares_leave_fp32(M, K, bits):
    """|h| about 2^e for e on both sides of where K squares pass 2^128, and up to the largest bf16; with one value of that size
    among small ones, too."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + K)
    gamma = (1 + 0.1 * rs.standard_normal(K)).astype(np.float32)
    for e in (55.9, 59.9, 62, 63.9, 80, 120, 126.5):
        x = rs.uniform(0.5, 1, (M, K)) * 2.0 ** e * rs.choice([-1, 1], (M, K))
        r = rs.standard_normal((M, K)) * 2.0 ** (e - 3)
        x[-1], r[-1] = rs.standard_normal(K), 0
        x[-1, K // 2] = 2.0 ** e
        x, r = bits_of(x), bits_of(r)
        say(f"norm of large rows M={M} K={K} 2^{e} bits={bits}")
        y, s, h = pace.rmsnorm(dev_bf16(x), dev_f32(gamma), dev_bf16(r), bits=bits)
        torch.cuda.synchronize()
        H, Y, tol = o8.norm(wl.bf16_bits_to_f64(x), wl.bf16_bits_to_f64(r), gamma.astype(np.float64), float(np.float32(1e-6)))
        assert np.abs(H).max() < 3.38e38                 # finite in bf16, too
        # past 2^126 the root's inverse has lost up to three bits; the small ones of the last row may be subnormal in bf16
        check_norm(y, s, h, H, Y, tol + 2.0 ** -22 * np.abs(Y) + 2.0 ** -134, True, bits)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("M,K", [(4, 16), (1027, 1024), (1026, 2064), (4, 3584), (3, 8192), (3, 16384), (2, 65536)])
def test_norm_of_rows_whose_squares_are_subnormal(M, K, bits):
    """|h| about 2^e down to bf16's subnormals, with eps among their squares, far below and far above them."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + K)
    gamma = (1 + 0.1 * rs.standard_normal(K)).astype(np.float32)
    for e, eps in ((-44, 2.0 ** -92), (-60, 2.0 ** -120), (-64, 1e-40), (-72, 2.0 ** -145), (-76, 2.0 ** -149), (-100, 2.0 ** -149), (-100, 1e-12),
                   (-130, 2.0 ** -149)):
        x = bits_of(rs.uniform(0.5, 1, (M, K)) * 2.0 ** e * rs.choice([-1, 1], (M, K)))
        x[-1] = 0
        say(f"norm of small rows M={M} K={K} 2^{e} eps={eps} bits={bits}")
        y, s, h = pace.rmsnorm(dev_bf16(x), dev_f32(gamma), eps=eps, bits=bits)
        torch.cuda.synchronize()
        H, Y, tol = o8.norm(wl.bf16_bits_to_f64(x), None, gamma.astype(np.float64), float(np.float32(eps)))
        # an output under 2^-126 may be subnormal in bf16
        check_norm(y, s, h, H, Y, tol + 2.0 ** -134, False, bits)


# gates around every place where e^-x, the sigmoid or their reciprocals leave fp32, and between
GATES = np.concatenate([np.linspace(-96, -80, 129), np.linspace(-80, 96, 177), [-3e38, -6e4, -300.0, -201, -200, -199, -1e-3, -1e-30, -2.0 ** -140, 0, 2.0 ** -149,
                                                                                2.0 ** -140, 1e-30, 1e-3, 199, 200, 201, 300, 6e4, 1e30]]).astype(np.float32)


@pytest.mark.parametrize("bits,sums", [(16, 0), (16, 2), (8, 0), (8, 1)])
@pytest.mark.parametrize("M,N,K", [(2, 704, 128), (40, 704, 128), (300, 704, 128), (100, 704, 3600), (700, 3616, 272), (2690, 5952, 976), (4300, 6016, 528)])
def test_swiglu_of_far_gates_within_its_roundings(M, N, K, bits, sums):
    """silu(g) u of biases beside products of zeros: g and u are exact.  What silu may be off: 2^-20.5 of its value and 2^-142 (the sigmoid's
    last subnormal bit, 2^-150, times 93, and the product's), all of it below g = -92.8; the product with u 2^-24, bf16 2^-8 and half its least step."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + N)
    x = torch.zeros((M, K), dtype=torch.float8_e4m3fn, device="cuda")
    w = torch.zeros((N, K), dtype=torch.float8_e4m3fn, device="cuda")
    xs, ws = torch.ones((o8.blocks(K), M), device="cuda"), torch.ones((o8.blocks(N), o8.blocks(K)), device="cuda")
    for e in (0, 20, 100, 127):
        g = np.resize(GATES, N // 2)
        u = (rs.uniform(0.5, 1, N // 2) * 2.0 ** np.where(g < -80, e, min(e, 20)) * rs.choice([-1, 1], N // 2)).astype(np.float32)
        bias = np.stack([g, u], 1).ravel()
        say(f"far gates M={M} N={N} K={K} bits={bits} sums={sums} u to 2^{e}")
        y, s = pace.gemm_fp8(x, xs, w, ws, dev_f32(bias), None, 2, bits, sums)
        torch.cuda.synchronize()
        g, u = g.astype(np.float64), u.astype(np.float64)
        with np.errstate(over="ignore"):
            silu = g / (1 + np.exp(-g))
        off = np.where(g < -92.8, np.abs(silu), 2.0 ** -20.5 * np.abs(silu) + 2.0 ** -142)
        ref, tol = silu * u, off * np.abs(u) + 2.0 ** -24 * np.abs(silu * u) + 2.0 ** -149
        rows = np.unique(np.append(np.arange(0, M, 61), M - 1))
        at = torch.from_numpy(rows).cuda()
        ref, tol = np.repeat(ref[None], len(rows), 0), np.repeat(tol[None], len(rows), 0)
        if bits == 16:
            err = np.abs(f64(y[at]) - ref)
            assert np.all(err <= 2.0 ** -8 * (np.abs(ref) + tol) + tol + 2.0 ** -134)
        else:
            check_product(y.view(torch.uint8)[at].view(torch.float8_e4m3fn), s[:, at], (ref, tol, None), 8)


@pytest.mark.parametrize("sums", [1, 2])
@pytest.mark.parametrize("M,N,K", [(3, 264, 400), (40, 264, 1040), (300, 520, 2064), (2690, 5936, 976)])
def test_products_of_scales_that_are_subnormal(M, N, K, sums):
    """Scales down to 2^-110 each: a block's product of scales is off by at most half a multiple of 2^-149, as are the sums that it enters."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + sums)
    x, _, X, _ = make_codes(rs, M, K, 1)
    w, _, W, _ = make_codes(rs, N, K, 128)
    XS = (rs.uniform(1, 2, (o8.blocks(K), M)) * 2.0 ** -rs.integers(58, 80, (1, M))).astype(np.float32)
    WS = (rs.uniform(1, 2, (o8.blocks(N), o8.blocks(K))) * 2.0 ** -rs.integers(58, 80, (o8.blocks(N), 1))).astype(np.float32)
    say(f"subnormal products of scales M={M} N={N} K={K} sums={sums}")
    y, _ = pace.gemm_fp8(x, dev_f32(XS), w, dev_f32(WS), sums=sums)
    torch.cuda.synchronize()
    m, n = np.unique(np.append(rs.permutation(M)[:40], M - 1)), np.unique(np.append(rs.permutation(N)[:40], N - 1))
    Wn = W[n] * o8.per_value(WS.astype(np.float64), (N, K), 128)[n]
    ref, tol, _ = o8.product(X[m], XS[:, m].astype(np.float64), Wn, np.ones((o8.blocks(len(n)), o8.blocks(K))), wide=sums == 2)
    blocks = sum(np.abs(X[m, k:k + 128]) @ np.abs(W[n, k:k + 128]).T for k in range(0, K, 128))
    tol = tol + 2.0 ** -150 * blocks + (o8.blocks(K) + 64) * 2.0 ** -150
    got = f64(y[torch.from_numpy(m).cuda()][:, torch.from_numpy(n).cuda()])
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * (np.abs(ref) + tol) + tol + 2.0 ** -134)
