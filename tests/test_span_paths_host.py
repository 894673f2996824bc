"""Batches whose work lists take the paths that small ones do not: workgroups that run several records one after the other, launches that begin with a mix of sweeps and decode units, more
sweeps than run at a time, and groups that share nothing, whose partial results the last workgroup combines.  Here that their lists are complete and of that shape, on the CPU;
tests/test_gpu_span_paths.py runs them."""
import numpy as np
import pytest

from test_abi_host import tc  # noqa: F401  (the fixture)
from test_span_host import batch, check


def up(n, first, step):
    return [first + step * i for i in range(n)]


MANY = [15, 16] * 9 + [1] * 6
# name: Hq, Hkv, D, q_len, ctx, groups (sequences, shared tokens) or (window, sinks), waves of a workgroup, the path
BATCHES = {
    "shared chained 8": (8, 2, 128, [9] * 12, up(12, 2400, 7), [(12, 2400)], 8, "chained"),
    "shared chained 4": (8, 2, 128, [9] * 12, up(12, 1600, 7), [(12, 1600)], 4, "chained"),
    "shared chained 4, 64": (8, 8, 64, [9] * 12, up(12, 2400, 7), [(12, 2400)], 4, "chained"),
    "window chained 4": (16, 2, 128, [1500], [3], (1500, 0), 4, "chained"),
    "window chained 8": (32, 2, 128, [400, 300] + [1] * 6, [4501, 0] + up(6, 1000, 300), (4300, 3), 8, "chained mix"),
    "window mix 8": (256, 16, 128, MANY, [4500] + up(17, 100, 100) + up(6, 500, 100), (4200, 3), 8, "mix more"),
    "window mix 4": (256, 16, 128, MANY, up(18, 100, 100) + up(6, 500, 100), (700, 3), 4, "mix more"),
    "window mix 4, 64": (256, 16, 64, [15, 16] * 13 + [1] * 6, up(26, 100, 50) + up(6, 500, 100), (700, 3), 4, "mix more"),
    "shared mix 4": (256, 16, 128, MANY, up(24, 160, 7), [(24, 160)], 4, "mix more"),
    "shared mix 8": (256, 16, 128, MANY, [2208] + up(23, 160, 7), [(24, 160)], 8, "mix more"),
    "alone": (8, 1, 64, [1], [7472], [(1, 7440)], 4, "arrivals"),
    "nothing shared": (8, 2, 128, [1, 1], [4000, 5000], [(2, 0)], 4, "arrivals"),
}


def takes_its_path(info, records, name):
    """That a list is of the shape that its batch stands for."""
    waves, path = BATCHES[name][6:]
    D = BATCHES[name][2]
    at_a_time = 256 * (1 if waves == 8 else 2 if D == 128 else 3)  # workgroups that sweep, on 256 compute units
    units = info.num_decode_items * info.waves_per_item // waves
    assert info.block_threads == 64 * waves
    if "chained" in path:  # a record behind another, and a block cut in two whose halves are two workgroups'
        assert (records[:, 15] >= 0).any() and (records[:, 4] >= 0).any()
    if "mix" in path:
        assert units > 0 and info.num_sweep_workgroups + units > at_a_time
    if "more" in path:
        assert info.num_sweep_workgroups > at_a_time
    if "arrivals" in path:
        assert info.num_sweeps == 0 and info.num_merge_items > 0 and info.merge_launch == 0


@pytest.mark.parametrize("name", list(BATCHES))
def test_lists(tc, name):  # noqa: F811
    Hq, Hkv, D, q_len, ctx, over, _, path = BATCHES[name]
    shared = isinstance(over, list)
    q_start, ctx, table, blocks = batch(q_len, ctx, over if shared else None)
    plan = tc.Plan(tc.make_pool(Hq, Hkv, D, blocks), q_start, ctx, table, host_only=True)
    if shared:
        plan.set_shared(np.concatenate([[0], np.cumsum([n for n, _ in over])]), [p for _, p in over])
    else:
        plan.set_window(*over)
    info = plan.span_info(shared)
    takes_its_path(info, plan.span_items(0, shared), name)
    if path != "arrivals":
        check(plan, Hq, Hkv, q_start, ctx, table, *((1 << 31, 0) if shared else over), shared=shared)
        return
    # Groups that share nothing are lists of decodes alone, like those of a window past all tokens: the same items, combined the same way.
    plan.set_window((1 << 31) - 1, 0)
    check(plan, Hq, Hkv, q_start, ctx, table, 1 << 31, 0)
    for kind in range(3):
        assert np.array_equal(plan.span_items(kind, True), plan.span_items(kind, False))
    for field in ("num_merge_items", "merge_launch", "waves_per_item", "grid_blocks", "block_threads", "num_partial_rows"):
        assert getattr(info, field) == getattr(plan.span_info(False), field)
