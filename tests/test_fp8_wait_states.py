"""The loads of the 8-bit products are inline asm, which the compiler's hazard recogniser does not look into: a scalar register that
the vector unit writes (v_readlane of a spilled descriptor, v_readfirstlane) may be read by a load only five wait states later, and a
register that a matrix product writes only after its passes.  The assembly that is built has to keep both (CPU: it is only read)."""
import re
import subprocess
from collections import defaultdict

import pytest

from paper_2608_27206_amd import build

SCALAR, MATRIX = 5, 19                              # wait states; of the matrix products here none needs more than 19


def numbers(text, kind):
    out = set()
    for lo, hi in re.findall(rf"\b{kind}\[(\d+):(\d+)\]", text):
        out |= set(range(int(lo), int(hi) + 1))
    return out | {int(n) for n in re.findall(rf"\b{kind}(\d+)\b", text)}


def parse(text):
    """Functions of the assembly: instructions (operation, operands), and the places of their labels."""
    fns, body, labels = {}, None, None
    for line in text.splitlines():
        line = line.split(";")[0].split("//")[0].strip()
        name = re.match(r"(\S+):$", line)
        if name:
            if name.group(1).startswith("_Z"):
                body, labels = [], {}
                fns[name.group(1)] = (body, labels)
            elif body is not None:
                labels[name.group(1)] = len(body)
        elif body is not None and line and line[0] not in ".#":
            op, _, rest = line.partition(" ")
            body.append((op, rest.strip()))
    return fns


def vector_writes(op, rest):
    """Scalar registers that the vector unit writes."""
    if not op.startswith("v_"):
        return set()
    first = rest.split(",")[0]
    if "readlane" in op or "readfirstlane" in op or op.startswith("v_cmp"):
        return numbers(first, "s") | ({"m0"} if first.strip() == "m0" else set())
    return numbers(rest.split(",")[1], "s") if "_co_" in op else set()


def hazards(body, labels):
    before = defaultdict(list)                          # label's place -> places of the branches that lead there
    for i, (op, rest) in enumerate(body):
        if op.startswith(("s_branch", "s_cbranch")) and rest in labels:
            before[labels[rest]].append(i)
    found = []

    def back(i, left, scalars, vectors, waited, load, seen):
        """Walks the ways to instruction i backwards, over `left` wait states."""
        while True:
            for j in before.get(i, []):
                if (j, waited) not in seen:
                    seen.add((j, waited))
                    back(j, left, scalars, vectors, waited, load, seen)
            i -= 1
            if i < 0 or body[i][0] in ("s_branch", "s_endpgm"):
                return
            op, rest = body[i]
            if waited < SCALAR and vector_writes(op, rest) & scalars:
                found.append((load, body[i], waited))
            if op.startswith("v_"):
                wrote = numbers(rest.split(",")[0], "v")
                if op.startswith("v_mfma") and wrote & vectors:
                    found.append((load, body[i], waited))
                vectors = vectors - wrote               # a later write is what the load reads
            waited += int(rest, 0) + 1 if op == "s_nop" else 1
            if waited >= left:
                return

    loads = 0
    for i, (op, rest) in enumerate(body):
        if op.startswith("buffer_load") and rest.endswith("lds"):
            loads += 1
            back(i, MATRIX, numbers(rest, "s") | {"m0"}, numbers(rest, "v"), 0, (op, rest), set())
    return loads, found


def test_the_check_itself():
    load = "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds\n"
    run = lambda text: hazards(*parse("_Zf:\n" + text)["_Zf"])   # noqa: E731
    assert run("\tv_readlane_b32 s6, v9, 3\n\ts_nop 3\n" + load)[1]
    assert not run("\tv_readlane_b32 s6, v9, 3\n\ts_nop 4\n" + load)[1]
    assert not run("\tv_readlane_b32 s8, v9, 3\n" + load)[1]
    assert run(".L1:\n" + load + "\tv_readfirstlane_b32 s4, v2\n\ts_cbranch_scc1 .L1\n")[1]
    assert run("\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0\n\ts_nop 7\n" + load)[1]
    assert not run("\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0\n\tv_mov_b32 v1, v9\n" + load)[1]


def test_loads_keep_the_wait_states(tmp_path):
    try:
        hipcc = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = tmp_path / "fp8.s"
    subprocess.run([hipcc, f"--offload-arch={build.ARCH}", "-O3", "-std=c++17", "-S", "--cuda-device-only", "-I", build.ROOT + "/include",
                    build.CSRC + "/fp8.hip", "-o", str(out)] + build.DEVICE_FLAGS, check=True, capture_output=True)
    total = 0
    for name, (body, labels) in parse(out.read_text()).items():
        loads, found = hazards(body, labels)
        total += loads
        assert not found, (name, found[:3])
    assert total > 500
