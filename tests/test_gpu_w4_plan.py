"""Where pace_gemm_w4 splits K over workgroups: the size that it asks for, what it uses of it, and its results on both
sides of the choice.  Tolerances as in test_gpu_cache.py: the output's rounding to bf16 (2^-8) and oracle.cache.w4's bound."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2608_27206_amd import workloads as wl
from tests.gpu_util import dev_bf16, dev_f32, say
from tests.test_gpu_cache import f64
from tests.test_gpu_cache import test_w4 as check_w4

pytestmark = pytest.mark.gpu


# M, N, K: rows of a wide product of 9 to 16 rows (whose columns need no split, or do for a last round), long rows of few
# columns on both sides of the borders of 8 and of 16 rows
PLANS = [(16, 16400, 3360), (9, 16384, 4096), (16, 18944, 3584), (16, 16400, 5152), (12, 20480, 5120), (16, 20496, 5120),
         (16, 7680, 5120), (16, 7696, 5120), (13, 12800, 8704), (8, 5136, 14336), (5, 6160, 14336), (8, 4096, 6400), (3, 2816, 6432),
         (8, 64, 6144), (16, 64, 3328), (16, 64, 2944), (17, 64, 768)]


@pytest.mark.parametrize("M,N,K", PLANS)
def test_workspace_is_asked_for_where_it_is_used(M, N, K):
    """For every group: a workspace is written where the size function asks for one, all of what it asks for and no more;
    and the product is right, with a bias and a residual."""
    import torch
    from paper_2608_27206_amd import pace
    rs = np.random.default_rng(M + N + K)
    need = pace.lib().pace_gemm_w4_workspace_size(M, N, K)
    x = wl.f32_to_bf16_bits(rs.standard_normal((M, K)).astype(np.float32))
    w = rs.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    bias, res = rs.standard_normal(N).astype(np.float32), wl.f32_to_bf16_bits(rs.standard_normal((M, N)).astype(np.float32))
    dw, dx, db, dr = torch.from_numpy(w).cuda(), dev_bf16(x), dev_f32(bias), dev_bf16(res)
    some = rs.permutation(N)[:500]                       # columns that are compared with the oracle
    for group in (32, 64, 128):
        if K % group:
            continue
        s = wl.f32_to_bf16_bits(rs.uniform(0.002, 0.03, size=(N, K // group)).astype(np.float32))
        ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        say(f"w4 M={M} N={N} K={K} group={group} workspace {need}")
        got = f64(pace.gemm_w4(dx, dw, dev_bf16(s), bias=db, residual=dr, epilogue=1, workspace=ws))
        torch.cuda.synchronize()
        used = (ws.view(torch.int32) != -0x5A5A5A5B).cpu().numpy()
        assert used[:need // 4].all() and not used[need // 4:].any(), f"{used.sum()} words of {need // 4} used"
        ref, tol = oc.w4(wl.bf16_bits_to_f64(x), w[some], wl.bf16_bits_to_f64(s[some]), None, group, bias[some],
                         wl.bf16_bits_to_f64(res[:, some]), 1)
        assert np.all(np.abs(got[:, some] - ref) <= 2.0 ** -8 * np.abs(ref) + tol)


# two tiles a wave (5 to 8 rows of about 26,700 to 32,768 columns, groups of 64 and 128), and their neighbours on every side
@pytest.mark.parametrize("M,N,K,group,zero,epilogue", [
    (8, 28680, 384, 128, 1, 2), (5, 32768, 640, 64, 0, 1), (6, 26641, 2432, 128, 0, 0), (7, 30002, 192, 64, 1, 2), (8, 26640, 2240, 64, 1, 1),
    (8, 26624, 384, 128, 1, 2), (8, 32770, 256, 64, 1, 2), (4, 30000, 384, 128, 1, 1), (9, 30002, 384, 64, 1, 2), (8, 30000, 288, 32, 1, 2)])
def test_two_tiles_a_wave(M, N, K, group, zero, epilogue):
    check_w4(M, N, K, group, zero, epilogue)
