"""The workgroup timeline (python -m paper_2508_01989_amd.wgtrace): the tracing build's stamps of either kind of cache can be read."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tracing_build_has_a_reader_for_each_kind_of_cache():
    from paper_2508_01989_amd.build import TRACE_LIB
    if not os.path.exists(TRACE_LIB):
        pytest.skip("the tracing build is not there")
    lib = ctypes.CDLL(TRACE_LIB)
    assert lib.tc_debug_wg_trace and lib.tc_debug_kvq_wg_trace


@pytest.mark.gpu
@pytest.mark.parametrize("workload", ["tiny", "prefill_heavy"])
@pytest.mark.parametrize("kvq", [False, True])
def test_timeline_of_a_launch(workload, kvq):
    cmd = [sys.executable, "-m", "paper_2508_01989_amd.wgtrace", "--workload", workload] + ["--kvq"] * kvq
    print("[case]", " ".join(cmd[1:]), flush=True)
    r = subprocess.run(cmd, cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    took = re.search(r"launch length ([\d.]+) us \((\w+)\)", r.stdout)
    assert took[2] == ("tc_kvq_mixed_attention" if kvq else "tc_mixed_attention")
    assert 1.0 < float(took[1]) < (100.0 if workload == "tiny" else 2000.0), r.stdout
    found = [re.search(p, r.stdout) for p in (r"prefill workgroups: (\d+)", r"decode workgroups: (\d+)", r"grid (\d+) workgroups")]
    prefill, decode, grid = (int(m[1]) if m else 0 for m in found)  # (decodes that the sweeps' workgroups draw have none of their own)
    assert prefill > 0 and prefill + decode == grid
