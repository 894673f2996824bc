"""The compiled kernels: no wave arrives at a barrier with LDS accesses of its own in flight.  (A barrier orders nothing by itself; the compiler was seen to leave out the wait for
accesses that lie across the back edge of a loop from the barrier.)"""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2508_01989_amd import build

REGISTERS_ONLY = ("ds_bpermute", "ds_permute", "ds_swizzle")


def functions(text):
    lines = text.split("\n")
    at = 0
    while at < len(lines):
        m = re.match(r"^(\S+):\s*; @", lines[at])
        if m:
            end = next(i for i in range(at, len(lines)) if lines[i].startswith(".Lfunc_end"))
            code = [x.split(";")[0].strip() for x in lines[at + 1:end]]
            yield m.group(1), [x for x in code if x and (not x.startswith(".") or re.match(r"\.LBB\w+:", x))]
            at = end
        at += 1


def unwaited(code):
    """Barriers that some path reaches from an LDS access without a wait for it in between."""
    label = {x[:-1]: i for i, x in enumerate(code) if x.endswith(":")}
    before = [[] for _ in code]
    for i, x in enumerate(code):
        op, *rest = x.split()
        if op == "s_branch" or op.startswith("s_cbranch"):
            before[label[rest[0]]].append(i)
        if op not in ("s_branch", "s_endpgm", "s_setpc_b64") and i + 1 < len(code):
            before[i + 1].append(i)
    found = []
    for i, x in enumerate(code):
        if x.split()[0] != "s_barrier":
            continue
        seen, todo = set(), list(before[i])
        while todo:
            j = todo.pop()
            if j in seen:
                continue
            seen.add(j)
            if code[j].startswith("s_waitcnt") and "lgkmcnt(0)" in code[j] or code[j].startswith("s_barrier"):
                continue
            if code[j].startswith("ds_") and not code[j].startswith(REGISTERS_ONLY):
                found.append((i, j, code[j]))
                continue
            todo += before[j]
    return found


def test_the_search_itself():
    loop = [".LBB0_1:", "s_barrier", "ds_write_b128 v0, v[2:5]", "s_cbranch_scc0 .LBB0_1", "s_endpgm"]
    assert unwaited(loop) == [(1, 2, "ds_write_b128 v0, v[2:5]")]
    assert not unwaited(loop[:1] + ["s_waitcnt vmcnt(0) lgkmcnt(0)"] + loop[1:])
    assert unwaited(loop[:1] + ["s_waitcnt lgkmcnt(1)"] + loop[1:])


def test_no_lds_access_in_flight_at_a_barrier(tmp_path):
    sources = [s for s in build.SOURCES if s.endswith(".hip")]
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no compiler")

    def assembly(source):
        out = tmp_path / (source + ".s")
        subprocess.run([hipcc, *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-x", "hip", "--cuda-device-only", "-S",
                        os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
        return out.read_text()

    with ThreadPoolExecutor(len(sources)) as pool:
        texts = list(pool.map(assembly, sources))
    barriers = 0
    for source, text in zip(sources, texts):
        for name, code in functions(text):
            barriers += sum(x.startswith("s_barrier") for x in code)
            assert not unwaited(code), (source, name)
    assert barriers > 100
