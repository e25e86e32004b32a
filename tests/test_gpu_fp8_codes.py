"""Codes are x / scale, the fp32 quotient rounded to the nearest of the e4m3 values (the even one in the middle of two): exactly, for every
operator that writes codes.  The quotient is numpy's, of the scales that came with the codes; what the norm and the product quantise is
made exact by their inputs."""
import numpy as np
import pytest

from oracle import cache as oc
from oracle import fp8 as o8
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, host, say
from tests.test_gpu_fp8 import bits_of

pytestmark = pytest.mark.gpu

POSITIVE = oc.e4m3_values()[:127]                       # 0 .. 448, by code


def codes_of(y, scale, rows):
    """The codes of y (fp32 values) under the given scales; NaN where y is not finite."""
    s = o8.per_value(scale, y.shape, rows).astype(np.float32)
    with np.errstate(invalid="ignore", under="ignore"):
        q = np.abs(y.astype(np.float32) / s).astype(np.float64)
    low = np.clip(np.searchsorted(POSITIVE, q, side="right") - 1, 0, 126)
    high = np.minimum(low + 1, 126)
    up, down = POSITIVE[high] - q, q - POSITIVE[low]
    code = np.where((up < down) | ((up == down) & (low % 2 == 1)), high, low)
    return np.where(np.isfinite(y), code | (np.signbit(y) << 7), 0x7F).astype(np.uint8)


def same_codes(q, y, scale, rows):
    import torch
    got = q.view(torch.uint8).cpu().numpy()
    got = np.where((got & 0x7F) == 0x7F, 0x7F, got)       # either NaN
    want = codes_of(y, scale, rows)
    wrong = got != want
    assert not wrong.any(), (int(wrong.sum()), wrong.size, np.argwhere(wrong)[:3].tolist())


def spread(rs, M, K):
    """Rows whose blocks lie at magnitudes from 2^-118 to 2^118, with values far below their block's largest, zeros of both signs."""
    x = rs.standard_normal((M, K)) * np.repeat(2.0 ** rs.integers(-118, 119, (M, o8.blocks(K))), 128, 1)[:, :K]
    x *= 2.0 ** -rs.integers(0, 14, x.shape)
    x[:, ::37], x[:, 5::37] = 0.0, -0.0
    return x.astype(np.float32)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 3584), (300, 1296), (130, 144)])
def test_codes_of_rows_and_weights(M, K, rows):
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + K)
    for x in (rs.standard_normal((M, K)), spread(rs, M, K)):
        b = bits_of(x)
        say(f"codes M={M} K={K} rows={rows}")
        q, s = pace.quantize_fp8(dev_bf16(b), rows=rows)
        torch.cuda.synchronize()
        same_codes(q, wl.bf16_bits_to_f64(b), host(s), rows)


@pytest.mark.parametrize("rows", [1, 128])
def test_every_quotient_of_two_bf16_mantissas(rows):
    """Each row holds every mantissa under a largest value of its own: the places where middles between two codes are most common."""
    import torch
    from paper_2608_27206_amd import pace
    m = 1 + np.arange(128) / 128
    blocks = []
    for top in m:
        values = np.where(m <= top, m, m / 2)
        blocks.append(np.stack([np.concatenate([[top], values[1:]]) * 2.0 ** e for e in (0, -97, 100)]))
    x = np.concatenate(blocks) if rows == 1 else np.concatenate([np.repeat(b, 128, 0) for b in blocks])
    b = bits_of(x)
    q, s = pace.quantize_fp8(dev_bf16(b), rows=rows)
    torch.cuda.synchronize()
    same_codes(q, wl.bf16_bits_to_f64(b), host(s), rows)


@pytest.mark.parametrize("M,K", [(3, 1040), (1030, 1040), (2, 4112), (2, 16400)])
def test_codes_of_the_norm(M, K):
    """h = 1 or -1 and a tiny eps: the root is 1, and y is gamma or -gamma."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(K)
    h = rs.choice([-1.0, 1.0], (M, K))
    for gamma in (rs.standard_normal(K).astype(np.float32), spread(rs, 1, K)[0]):
        say(f"norm's codes M={M} K={K}")
        q, s, _ = pace.rmsnorm(dev_bf16(bits_of(h)), dev_f32(gamma), eps=1e-30, bits=8)
        torch.cuda.synchronize()
        same_codes(q, h * gamma, host(s), 1)


@pytest.mark.parametrize("sums", [0, 1])
@pytest.mark.parametrize("M,N,K", [(2, 512, 128), (40, 512, 128), (300, 544, 128), (300, 1056, 1552), (700, 3616, 272), (3000, 6400, 528)])
def test_codes_of_the_product(M, N, K, sums):
    """Products of zeros, gates of 128 (whose sigmoid is 1 in fp32): the output is 128 times the bias of u."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + N)
    x = torch.zeros((M, K), dtype=torch.float8_e4m3fn, device="cuda")
    w = torch.zeros((N, K), dtype=torch.float8_e4m3fn, device="cuda")
    xs, ws = torch.ones((o8.blocks(K), M), device="cuda"), torch.ones((o8.blocks(N), o8.blocks(K)), device="cuda")
    for u in (rs.standard_normal(N // 2).astype(np.float32), spread(rs, 1, N // 2)[0] * np.float32(2.0 ** -7)):
        bias = np.empty(N, np.float32)
        bias[0::2], bias[1::2] = 128, u
        say(f"product's codes M={M} N={N} K={K} sums={sums}")
        q, s = pace.gemm_fp8(x, xs, w, ws, dev_f32(bias), None, 2, 8, sums)
        torch.cuda.synchronize()
        y = 128 * (np.float32(0) + u)                    # the bias is added to sums of 0, so that -0 becomes 0
        same_codes(q, np.repeat(y[None], M, 0), host(s), 1)
