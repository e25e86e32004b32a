"""Checks the assembly of a HIP source for the wait states that loads in inline asm need.

The compiler's hazard recogniser does not look into inline asm, where the kernels' loads into LDS are.  A scalar register that the
vector unit wrote (v_readlane of a spilled descriptor, v_readfirstlane) may be read by such a load only five wait states later, and a
vector register that a matrix product writes only after its passes.  The build looks at every such load in what it has compiled, over
all ways that lead to it, and ends where one comes too early.
"""
from __future__ import annotations

import re
from collections import defaultdict
from typing import Dict, List, Set, Tuple

SCALAR = 5                                          # wait states after the vector unit's write of a scalar
MATRIX = 19                                         # of the matrix products in use none needs more


def _numbers(text: str, kind: str) -> Set[int]:
    out: Set[int] = set()
    for lo, hi in re.findall(rf"\b{kind}\[(\d+):(\d+)\]", text):
        out |= set(range(int(lo), int(hi) + 1))
    return out | {int(n) for n in re.findall(rf"\b{kind}(\d+)\b", text)}


def _functions(text: str):
    """Each function's instructions (operation, operands), and the places of its labels."""
    fns: Dict[str, Tuple[list, dict]] = {}
    body = labels = None
    for line in text.splitlines():
        line = line.split(";")[0].split("//")[0].strip()
        name = re.match(r"(\S+):$", line)
        if name and not name.group(1).startswith("."):
            body, labels = [], {}
            fns[name.group(1)] = (body, labels)
        elif name and body is not None:
            labels[name.group(1)] = len(body)
        elif body is not None and line and line[0] not in ".#":
            op, _, rest = line.partition(" ")
            body.append((op, rest.strip()))
    return fns


def _scalars_written(op: str, rest: str) -> set:
    """Scalar registers that a vector instruction writes."""
    if not op.startswith("v_"):
        return set()
    operands = rest.split(",")
    if "readlane" in op or "readfirstlane" in op or op.startswith("v_cmp"):
        return _numbers(operands[0], "s") | ({"m0"} if operands[0].strip() == "m0" else set())
    return _numbers(operands[1], "s") if "_co_" in op else set()


def _early(body: list, labels: dict, load: int, before: dict) -> List[str]:
    """What the load at this place comes too early after."""
    op, rest = body[load]
    found: List[str] = []
    # places still to walk back from: the instruction behind, wait states since, vector registers not written since
    todo = [(load, 0, frozenset(_numbers(rest, "v")))]
    scalars = _numbers(rest, "s") | {"m0"}
    seen = set(todo)
    while todo:
        i, waited, vectors = todo.pop()
        ways = [(j, waited, vectors) for j in before.get(i, [])]           # from in front of the branches that lead here
        if i and body[i - 1][0] not in ("s_branch", "s_endpgm"):
            last, args = body[i - 1]
            if waited < SCALAR and _scalars_written(last, args) & scalars:
                found.append(f"{op} {rest}: {waited} wait states after {last} {args}")
            if last.startswith("v_"):
                wrote = _numbers(args.split(",")[0], "v")
                if last.startswith("v_mfma") and wrote & vectors:
                    found.append(f"{op} {rest}: {waited} wait states after {last} {args}")
                vectors = vectors - wrote                                  # a later write is what the load reads
            waited += int(args, 0) + 1 if last == "s_nop" else 1
            if waited < MATRIX:
                ways.append((i - 1, waited, vectors))
        for way in ways:
            if way not in seen:
                seen.add(way)
                todo.append(way)
    return found


def problems(assembly: str) -> List[str]:
    """The loads into LDS that come too early, as texts."""
    found: List[str] = []
    for name, (body, labels) in _functions(assembly).items():
        loads = [i for i, (op, rest) in enumerate(body) if op.startswith("buffer_load") and rest.endswith("lds")]
        before = defaultdict(list)
        for i, (op, rest) in enumerate(body):
            if op.startswith(("s_branch", "s_cbranch")) and rest in labels:
                before[labels[rest]].append(i)
        for i in loads:
            found += [f"{name}: {p}" for p in _early(body, labels, i, before)]
    return found
