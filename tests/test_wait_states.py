"""The build ends where a load in inline asm comes too early after the write of a register that it reads (CPU: sources are compiled
and their assembly read, nothing runs)."""
import pytest

from paper_2608_27206_amd import build

LOAD = "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds\n"


def check(text):
    from paper_2608_27206_amd import wait_states
    return wait_states.problems("_Zf:\n" + text)


@pytest.mark.parametrize("text", [
    "\tv_readlane_b32 s6, v9, 3\n\ts_nop 3\n" + LOAD,
    "\tv_readfirstlane_b32 m0, v9\n\ts_nop 0\n" + LOAD,
    ".L1:\n" + LOAD + "\tv_readfirstlane_b32 s4, v2\n\ts_cbranch_scc1 .L1\n",
    "\tv_readlane_b32 s6, v9, 3\n\ts_branch .L2\n.L1:\n\ts_nop 7\n.L2:\n" + LOAD + "\ts_branch .L1\n",
    "\tv_readlane_b32 s6, v9, 3\n\ts_cbranch_vccz .L1\n\ts_nop 7\n.L1:\n" + LOAD,
    "\tv_cmp_gt_u32_e64 s[4:5], v3, v4\n" + LOAD,
    "\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0\n\ts_nop 7\n" + LOAD])
def test_loads_that_come_too_early(text):
    assert check(text)


@pytest.mark.parametrize("text", [
    "\tv_readlane_b32 s6, v9, 3\n\ts_nop 4\n" + LOAD, "\tv_readlane_b32 s8, v9, 3\n" + LOAD, "\ts_mov_b32 s6, 3\n" + LOAD,
    "\tv_readlane_b32 s6, v9, 3\n\ts_endpgm\n.L1:\n" + LOAD,
    "\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0\n\tv_mov_b32 v1, v9\n" + LOAD])
def test_loads_that_do_not(text):
    assert not check(text)


SOURCE = """#include <hip/hip_runtime.h>
__global__ void f(float* p) {{
  asm volatile("v_readfirstlane_b32 s4, %0\\n\\ts_nop {nop}\\n\\tbuffer_load_dwordx4 %0, s[4:7], 0 offen lds\\n\\ts_waitcnt vmcnt(0)"
               ::"v"(threadIdx.x) : "s4", "s5", "s6", "s7", "memory");
  p[threadIdx.x] = 0.f;
}}
"""


@pytest.mark.parametrize("nop", [3, 4])
def test_build_of_a_source(tmp_path, monkeypatch, nop):
    try:
        build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    (tmp_path / "one.hip").write_text(SOURCE.format(nop=nop))
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    if nop < 4:
        with pytest.raises(RuntimeError, match="too early"):
            build._compile("one.hip")
        assert not (tmp_path / "one.o").exists()
    else:
        assert build._compile("one.hip") == str(tmp_path / "one.o")
        assert sorted(f.name for f in tmp_path.iterdir()) == ["one.hip", "one.o"]
