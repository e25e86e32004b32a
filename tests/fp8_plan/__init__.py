"""Which kernels the 8-bit products' plan picks for a call, in which form: the plan's own source, compiled for the CPU."""
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
EPILOGUES = ("bias", "residual", "swiglu")


@functools.lru_cache(None)
def _lib():
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        return None
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "plan.so")
        subprocess.run([cxx, "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-Wno-unused-function",
                        "-I", os.path.join(ROOT, "paper_2608_27206_amd", "csrc"),
                        os.path.join(ROOT, "tests", "fp8_plan", "plan.cpp"), "-o", out], check=True)
        return ctypes.CDLL(out)


def available():
    return _lib() is not None


@functools.lru_cache(None)
def tiles():
    """(rows, columns, stages, groups, wide, has the form that takes tiles in turn) of each tile."""
    out = (ctypes.c_int * 600)()
    n = _lib().fp8_tiles(out)
    return [tuple(out[6 * i:6 * i + 6]) for i in range(n)]


_OUT = (ctypes.c_int * 8)()


def launches(M, N, K, eight, wide):
    n = _lib().fp8_plan(M, N, K, int(eight), int(wide), _OUT)
    return [tuple(_OUT[4 * i:4 * i + 4]) for i in range(n)]


def forms(M, N, K, epilogue, bits, sums):
    """The forms of kernels that the call runs, its tensors 16-byte aligned."""
    eight = bits == 8
    wide = sums == 2 or (sums == 0 and eight)
    name = "eight" if eight else EPILOGUES[epilogue]
    units = eight or (2 * (N // 2 if epilogue == 2 else N)) % 16 == 0     # outputs move 8 at a time
    out = set()
    for t, rows, splits, part in launches(M, N, K, eight, wide):
        if part:
            out.add(("join", name, N % 4 == 0))
        if t < 0:
            out.add(("few rows", "parts" if part else name, N % 4 == 0))
            continue
        bm, bn, stages, groups, _, run = tiles()[t]
        if part:
            out.add((t, "K in parts" if splits > 1 else "one part", N % 4 == 0))
        elif run and _lib().fp8_in_turn(stages, splits, part, N, K, units, epilogue == 1):
            several = -(-rows // bm) * -(-N // bn) > 256
            out.add((t, "in turn", name, "several tiles" if several else "one tile"))
        else:
            ring = groups == 1 and epilogue == 1 and units and -(-K // 128) >= stages
            out.add((t, name, "through the ring" if ring else "units of 8" if units else "smaller units"))
    return out
