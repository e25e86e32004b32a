"""The 8-bit operators at the ends of fp32's range, against the float64 oracle."""
import numpy as np
import pytest

from oracle import fp8 as o8
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, say
from tests.test_gpu_fp8 import bits_of, check_norm

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
