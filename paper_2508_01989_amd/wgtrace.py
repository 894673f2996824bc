"""Workgroup timeline of one launch of the attention kernel: when every workgroup started, when its prefill
pieces were done, when it ended.  Needs the tracing build of the library
(python -m paper_2508_01989_amd.build --trace), which stamps the times inside the kernel.

    python -m paper_2508_01989_amd.wgtrace --workload prefill_heavy [--kvq]
"""
from __future__ import annotations

import argparse
import ctypes as C
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


class KvqBatch:
    """The same batch over a cache in 8 bits: its tensors, plan and attention call."""

    def __init__(self, batch, device="cuda:0"):
        import torch

        import paper_2508_01989_amd as tc
        from paper_2508_01989_amd.harness import to_dev
        sp, nb = batch.spec, int(batch.num_blocks)
        n = nb * sp.num_kv_heads * sp.block_size * sp.head_dim
        self.spec, self.k, self.v = sp, *(torch.zeros(n, dtype=torch.uint8, device=device) for _ in range(2))
        self.scales = torch.full((nb * sp.num_kv_heads * 2,), 127, dtype=torch.uint8, device=device)
        code = tc.TC_FP16 if getattr(sp, "dtype", "bf16") == "fp16" else tc.TC_BF16
        self.pool = tc.make_kvq_pool(sp.num_q_heads, sp.num_kv_heads, sp.head_dim, nb, self.k, self.v, self.scales, dtype=code)
        self.q, self.k_new, self.v_new = (to_dev(x, device) for x in (batch.q, batch.k_new, batch.v_new))
        self.k_hist, self.v_hist = to_dev(batch.k_hist, device), to_dev(batch.v_hist, device)
        keep = np.flatnonzero(sp.ctx_len > 0)
        if len(keep):
            start = np.concatenate([[0], np.cumsum(sp.ctx_len[keep])]).astype(np.int32)
            history = tc.Plan(self.pool, start, np.zeros(len(keep), np.int32), batch.block_table[keep])
            tc.tc_kvq_append(history, self.pool, self.k_hist, self.v_hist)
            torch.cuda.synchronize()
            history.destroy()
        self.plan = tc.Plan(self.pool, batch.q_start, sp.ctx_len, batch.block_table)
        self.workspace = torch.empty(max(self.plan.workspace_bytes, 16), dtype=torch.uint8, device=device)
        self.out = torch.empty((batch.total_q, sp.num_q_heads, sp.head_dim), dtype=torch.int16, device=device)

    def append(self):
        import paper_2508_01989_amd as tc
        tc.tc_kvq_append(self.plan, self.pool, self.k_new, self.v_new)

    def attention(self):
        import paper_2508_01989_amd as tc
        tc.tc_kvq_mixed_attention(self.plan, self.pool, self.q, self.out, self.spec.scale, self.workspace, self.plan.workspace_bytes)


def stamps(lib, kvq, n):
    """Start, end, place and kind of the first n workgroups of the latest attention launch, int64 [n][4]; kvq: over a cache in 8 bits."""
    buf = np.zeros((n, 4), np.int64)
    read = lib.tc_debug_kvq_wg_trace if kvq else lib.tc_debug_wg_trace
    read.argtypes = [C.c_void_p, C.c_int]
    assert read(buf.ctypes.data, n * 4) == 0
    return buf


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="prefill_heavy", choices=["tiny", "prefill_heavy", "decode_heavy", "pure_decode", "long_prompt"])
    ap.add_argument("--two-launch", action="store_true", help="trace tc_attention_partials (no in-kernel combination) instead of tc_mixed_attention")
    ap.add_argument("--kvq", action="store_true", help="over a cache in 8 bits (tc_kvq_mixed_attention)")
    args = ap.parse_args()
    if args.kvq and args.two_launch:
        ap.error("--two-launch is for a cache in 16 bits")
    import paper_2508_01989_amd as tc
    from paper_2508_01989_amd.build import TRACE_LIB
    if not os.path.exists(TRACE_LIB):
        raise SystemExit(f"{TRACE_LIB} is missing: run `python -m paper_2508_01989_amd.build --trace` first")
    tc.LIB_PATH = TRACE_LIB
    import torch
    import workloads as W
    from paper_2508_01989_amd.harness import DeviceBatch
    idx = ["tiny", "prefill_heavy", "decode_heavy", "pure_decode", "long_prompt"].index(args.workload)
    db = (KvqBatch if args.kvq else DeviceBatch)(W.make_batch(W.config_spec(idx)))
    run = db.attention_partials if args.two_launch else db.attention
    db.append()
    for _ in range(5):
        run()
    torch.cuda.synchronize()
    run()
    torch.cuda.synchronize()
    info = db.plan.info
    n = min(info.grid_blocks, 16384)
    t = stamps(tc.lib(), args.kvq, n)
    t0 = t[:, 0].min()
    start, end = (t[:, 0] - t0) / 100.0, (t[:, 1] - t0) / 100.0  # microseconds
    kind = t[:, 3] & 255
    mid = start + (t[:, 3] >> 8) / 100.0
    print(f"workload {args.workload}: grid {info.grid_blocks} workgroups of {info.block_threads} threads, {info.num_prefill_workgroups} prefill workgroups "
          f"({info.num_prefill_pieces} pieces of {info.num_prefill_items} items), {info.num_decode_items} decode items, decode queue {bool(info.decode_queue)}")
    print(f"launch length {end.max():.1f} us ({'tc_kvq_mixed_attention' if args.kvq else 'tc_attention_partials' if args.two_launch else 'tc_mixed_attention'})")
    pct = [0, 10, 50, 90, 100]
    for k, name in ((0, "prefill workgroups"), (1, "decode workgroups")):
        m = kind == k
        if not m.any():
            continue
        print(f"{name}: {int(m.sum())}")
        print(f"  start      (min 10% median 90% max) us: {np.round(np.percentile(start[m], pct), 1)}")
        if k == 0:
            print(f"  pieces done(min 10% median 90% max) us: {np.round(np.percentile(mid[m], pct), 1)}   sum over workgroups {np.sum(mid[m] - start[m]):.0f} us")
        print(f"  end        (min 10% median 90% max) us: {np.round(np.percentile(end[m], pct), 1)}   sum over workgroups {np.sum(end[m] - start[m]):.0f} us")
    ts = np.linspace(0, end.max(), 11)
    busy_decode = [(int(round(x)), int((((kind == 1) & (start <= x) & (end > x)) | ((kind == 0) & (mid <= x) & (end > x))).sum())) for x in ts]
    print("workgroups on decode items at time t (us):", busy_decode)


if __name__ == "__main__":
    main()
