"""Attention over a window and over shared tokens, on the CPU: the work lists cover what each row attends over exactly once and name every partial result, and what the calls refuse."""
import ctypes as C

import numpy as np
import pytest

import test_abi_host as abi
from test_abi_host import tc  # noqa: F401  (the fixture)

AFTER = (1 << 31) - 1024


def batch(q_len, ctx, groups=None, seed=0, spare=3):
    """q_start, ctx and block tables; groups: (sequences, shared tokens) in order."""
    rng = np.random.default_rng(seed)
    q_len, ctx = np.array(q_len, np.int64), np.array(ctx, np.int64)
    pages = -(-(q_len + ctx) // 16)
    ids = rng.permutation(int(pages.sum()) + spare).astype(np.int32)
    table = np.zeros((len(q_len), int(pages.max(initial=1))), np.int32)
    at = 0
    for s, n in enumerate(pages):
        table[s, :n] = ids[at:at + n]
        at += n
    s = 0
    for n, shared in groups or []:
        table[s:s + n, :shared // 16] = table[s, :shared // 16]
        s += n
    return np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32), ctx.astype(np.int32), table, len(ids)


def places(f):
    """Pages of a list, from (a, h, f, b, c, e)."""
    a, h, fr, b, c, e = (int(x) for x in f)
    return list(range(a)) + list(range(b, c)) + ([a] if h else []) + list(range(fr, b)) + list(range(c, e))


def check(plan, Hq, Hkv, q_start, ctx, table, window, sinks, shared=False):
    """Every (packed row, KV head): its tokens once each, its partial results all in one merge item, or one item that writes its output."""
    G, T = Hq // Hkv, int(q_start[-1])
    info = plan.span_info(shared)
    records, items, merge = (plan.span_items(k, shared) for k in range(3))
    page_off = np.concatenate([[0], np.cumsum(-(-(np.diff(q_start) + ctx) // 16))])
    pages = np.concatenate([table[s, :page_off[s + 1] - page_off[s]] for s in range(len(ctx))])
    seq_of = np.repeat(np.arange(len(ctx)), np.diff(q_start))
    pos = np.arange(T) - q_start[seq_of] + ctx[seq_of]
    longest = int((ctx + np.diff(q_start)).max())
    width = -(-longest // 16) * 16
    seen = np.zeros((T, Hkv, width), np.int8)
    direct = np.zeros((T, Hq), np.int32)
    rows = np.full(info.num_partial_rows, -1, np.int64)  # packed row * Hq + head of each row of the workspace

    def visit(row, n_rows, kvh, first_pos, page_off_, runs, i0, i1, at):
        lst = places(runs)
        assert 0 <= i0 <= i1 and (i0 < i1 or i0 == 0)
        for t in range(row, row + n_rows):
            s = seq_of[t]
            p = AFTER if first_pos == AFTER else pos[t]
            if first_pos != AFTER:
                assert p == first_pos + t - row and page_off_ == page_off[s]
            for i in range(i0, min(i1, len(lst))):
                assert pages[page_off_ + lst[i]] == table[s, lst[i]]  # (of a group: its first sequence's)
                j = np.arange(16 * lst[i], 16 * lst[i] + 16)
                sees = (j <= p) & ((p - j < window) | (j < sinks))
                seen[t, kvh, j[sees]] += 1
                if i < runs[0] + runs[4] - runs[3]:
                    assert sees.all()  # places that need no mask
        for x in range(n_rows * G):
            t, h = row + x // G, kvh * G + x % G
            if at < 0:
                direct[t, h] += 1
            else:
                assert rows[at + x] == -1
                rows[at + x] = t * Hq + h

    for r in records:
        assert r[9] * G <= 256 and r[8] == 0 and r[0] < r[1]
        runs = r[[2, 3, 5, 7, 13, 14]]
        lst = places(runs)
        assert 4 * (r[1] - 1) < len(lst)
        for x in range(16):
            assert r[16 + x] == pages[r[12] + lst[min(4 * r[0] + x, len(lst) - 1)]]
        for h in range(Hkv):
            visit(r[10], r[9], h, r[11], r[12], runs, 4 * r[0], 4 * r[1], -1 if r[4] < 0 else r[4] + h * r[6])
    for d in items:
        if d[2] == d[3]:
            assert d[5] == -1
            continue
        assert d[7] <= 16 and d[7] % G == 0 and d[3] - d[2] <= 64 * info.waves_per_item and d[3] <= len(places(d[8:14]))
        visit(d[4], d[7] // G, d[1], d[0], d[6], d[8:14], d[2], d[3], d[5])
    for t in range(T):
        j = np.arange(width)
        want = (j <= pos[t]) & ((pos[t] - j < window) | (j < sinks))
        assert np.array_equal(seen[t], np.broadcast_to(want, (Hkv, width)).astype(np.int8)), t
    merged = np.zeros((T, Hq), np.int32)
    used = np.zeros(len(rows), np.int32)
    for m in merge:
        assert 0 < m[1] <= 16
        for h in range(Hkv):
            for x in range(m[1] * G):
                t, head = m[0] + x // G, h * G + x % G
                merged[t, head] += 1
                for base, kv, n, step in (m[2:6], m[6:10]):
                    for i in range(n):
                        at = base + h * kv + i * step + x
                        assert rows[at] == t * Hq + head
                        used[at] += 1
    if info.num_merge_items and not info.merge_launch:  # every partial result is waited for by the last of its group
        assert not shared and len(records) == 0 and info.waves_per_item * 64 == info.block_threads
        parts = np.zeros((len(merge), Hkv), np.int32)
        for d in items[items[:, 5] >= 0]:
            assert merge[d[14]][0] == d[4] and merge[d[14]][1] == 1 and d[7] == G and d[15] == merge[d[14]][8]
            parts[d[14], d[1]] += 1
        assert (parts == merge[:, 8:9]).all()
    assert (used == 1).all() and ((direct > 0) ^ (merged > 0)).all() and (direct + merged == 1).all()
    chained = [r[15] for r in records if r[15] >= 0]  # every record is one workgroup's, the first of them or behind another
    runs = info.num_sweep_workgroups // Hkv
    assert sorted(list(range(runs)) + chained) == list(range(len(records))) and runs * Hkv == info.num_sweep_workgroups
    assert info.grid_blocks == info.num_sweep_workgroups + len(items) * info.waves_per_item // (info.block_threads // 64)
    return info


WINDOWS = [(1, 0), (7, 0), (16, 1), (16, 16), (17, 5), (33, 40), (100, 4), (64, 200), (1000, 0), (1 << 30, 3), (5, 1 << 30), ((1 << 31) - 1, (1 << 31) - 1)]


@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (5, 1), (16, 1), (32, 8)])
@pytest.mark.parametrize("window, sinks", WINDOWS)
def test_window_lists(tc, heads, window, sinks):  # noqa: F811
    """Chunks at any offset, decodes of any length, windows and sinks on, beside and across the borders of blocks, and beyond all of the tokens."""
    q_len, ctx = [300, 1, 17, 1, 1, 70, 1, 2], [0, 0, 333, 15, 16, 1000, 700, 31]
    q_start, ctx, table, blocks = batch(q_len, ctx)
    plan = tc.Plan(tc.make_pool(*heads, 128, blocks), q_start, ctx, table, host_only=True)
    plan.set_window(window, sinks)
    check(plan, *heads, q_start, ctx, table, window, sinks)


@pytest.mark.parametrize("window, sinks", WINDOWS)
@pytest.mark.parametrize("n", [1, 3, 40])
def test_window_lists_of_decodes(tc, n, window, sinks):  # noqa: F811
    rng = np.random.default_rng(n)
    ctx = np.concatenate([[0], rng.integers(0, 3000, n - 1)])
    q_start, ctx, table, blocks = batch([1] * n, ctx)
    plan = tc.Plan(tc.make_pool(8, 2, 64, blocks), q_start, ctx, table, host_only=True)
    plan.set_window(window, sinks)
    info = check(plan, 8, 2, q_start, ctx, table, window, sinks)
    assert info.num_sweeps == 0 and info.block_threads == 256


def test_window_list_of_a_long_sequence_is_cut(tc):  # noqa: F811
    for q, offset in ((1, 40000), (20, 20000)):
        q_start, ctx, table, blocks = batch([q], [offset])
        plan = tc.Plan(tc.make_pool(4, 1, 128, blocks), q_start, ctx, table, host_only=True)
        plan.set_window(30000, 4)
        info = check(plan, 4, 1, q_start, ctx, table, 30000, 4)
        assert info.num_partial_rows > 0 and info.grid_blocks > 1
        assert plan.window_workspace_bytes == info.num_partial_rows * (128 + 2) * 4


GROUPS = [
    ([1] * 6, [100, 64, 65, 80, 200, 79], [(6, 64)]),
    ([1] * 90, [32 + 7 * i for i in range(90)], [(90, 32)]),
    ([1] * 5, [100, 64, 65, 80, 200], [(2, 64), (1, 64), (2, 80)]),
    ([1] * 4, [0, 5, 0, 100], [(4, 0)]),
    ([70, 1, 1, 33, 1, 1], [160, 500, 170, 48, 48, 50], [(3, 160), (3, 48)]),
    ([1, 1, 130, 1], [16, 16, 16, 16], [(2, 16), (2, 16)]),
    ([1] * 40 + [3, 9], [2000] * 40 + [2000, 2016], [(42, 2000)]),
    ([300] * 2, [4096, 5000], [(2, 4096)]),
]


@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (5, 1), (16, 1)])
@pytest.mark.parametrize("q_len, ctx, groups", GROUPS)
def test_shared_lists(tc, heads, q_len, ctx, groups):  # noqa: F811
    q_start, ctx, table, blocks = batch(q_len, ctx, groups)
    plan = tc.Plan(tc.make_pool(*heads, 64, blocks), q_start, ctx, table, host_only=True)
    plan.set_shared(np.concatenate([[0], np.cumsum([n for n, _ in groups])]), [p for _, p in groups])
    check(plan, *heads, q_start, ctx, table, 1 << 31, 0, shared=True)


def test_shared_tokens_are_read_once_for_the_group(tc):  # noqa: F811
    q_start, ctx, table, blocks = batch([1] * 64, [1024 + 16] * 64, [(64, 1024)])
    plan = tc.Plan(tc.make_pool(32, 8, 128, blocks), q_start, ctx, table, host_only=True)
    plan.set_shared([0, 64], [1024])
    records = plan.span_items(0, True)
    blocks = 256 // (32 * plan.span_info(True).block_threads // 64)  # 64 rows of four heads are 256 pairs: a sweep or two
    assert (records[:, 1] - records[:, 0]).sum() == blocks * 1024 // 64 and (records[:, 9] == 64 // blocks).all()
    items = plan.span_items(1, True)
    assert (items[:, 3] - items[:, 2]).sum() == 64 * 8 * 2


def test_lists_hold_for_their_batch_only(tc):  # noqa: F811
    q_start, ctx, table, blocks = batch([1, 20], [40, 32], [(2, 32)])
    pool = tc.make_pool(8, 2, 128, blocks, 1 << 20, 1 << 21)
    plan = tc.Plan(pool, q_start, ctx, table, host_only=True)
    call = {False: tc.tc_window_attention, True: tc.tc_shared_attention}
    run = lambda shared: abi._status(tc, lambda: call[shared](plan, pool, 1 << 22, 1 << 23, 0.1, 1 << 24, 1 << 30))  # noqa: E731
    text = lambda shared: (run(shared), tc.last_error())  # noqa: E731
    for shared in (False, True):
        assert text(shared)[0] == tc.TC_ERR_ARG and "set_" in tc.last_error() and plan.span_info(shared).ready == 0
    plan.set_window(10, 2)
    assert plan.span_info().ready == 1 and plan.span_info(True).ready == 0
    plan.set_shared([0, 2], [32])
    for shared in (False, True):
        assert plan.span_info(shared).ready == 1
        assert text(shared)[0] == tc.TC_ERR_ARG and "host-only" in tc.last_error()
    with pytest.raises(tc.TcError):
        plan.set_window(0, 0)
    assert plan.span_info().ready == 0 and plan.span_info(True).ready == 1 and plan.window_workspace_bytes == 0
    plan.update(pool, q_start, ctx, table)
    for shared in (False, True):
        assert plan.span_info(shared).ready == 0 and text(shared)[0] == tc.TC_ERR_ARG
    assert abi._status(tc, lambda: plan.span_items(0)) == tc.TC_ERR_ARG


def test_refusals_of_the_lists(tc):  # noqa: F811
    q_start, ctx, table, blocks = batch([1, 1, 20], [40, 33, 32], [(3, 32)])
    plan = tc.Plan(tc.make_pool(8, 2, 128, blocks), q_start, ctx, table, host_only=True)
    st = lambda fn: abi._status(tc, fn)  # noqa: E731
    for window, sinks in ((0, 0), (-1, 0), (1, -1), (-(1 << 31), 3)):
        assert st(lambda: plan.set_window(window, sinks)) == tc.TC_ERR_ARG
    for starts, lens, want in (([0, 2], [32], tc.TC_ERR_SPAN), ([0, 4], [32], tc.TC_ERR_SPAN), ([1, 3], [32], tc.TC_ERR_SPAN), ([0, 0, 3], [0, 32], tc.TC_ERR_SPAN),
                               ([0, 2, 1, 3], [0, 0, 0], tc.TC_ERR_SPAN), ([0, 100, 3], [16, 16], tc.TC_ERR_SPAN), ([0, 3], [8], tc.TC_ERR_SPAN), ([0, 3], [-16], tc.TC_ERR_SPAN),
                               ([0, 3], [48], tc.TC_ERR_SPAN), ([0], [], tc.TC_ERR_SPAN)):
        assert st(lambda: plan.set_shared(starts, lens)) == want, (starts, lens)
    plan.set_shared([0, 3], [32])
    plan.set_shared([0, 1, 3], [32, 16])
    other = table.copy()
    other[1, 1] = other[2, 2]
    plan = tc.Plan(tc.make_pool(8, 2, 128, blocks), q_start, ctx, other, host_only=True)
    assert st(lambda: plan.set_shared([0, 3], [32])) == tc.TC_ERR_BLOCK
    plan.set_shared([0, 3], [16])
    L = tc.lib()
    assert L.tc_plan_set_window(None, 1, 0, None) == tc.TC_ERR_NULL and L.tc_plan_set_shared(None, 0, None, None, None) == tc.TC_ERR_NULL
    assert L.tc_plan_set_shared(plan.handle, 1, None, None, None) == tc.TC_ERR_NULL
    assert L.tc_window_workspace_bytes(None) == 0 and L.tc_shared_workspace_bytes(None) == 0
    kvq = tc.Plan(tc.make_kvq_pool(8, 2, 128, blocks), q_start, ctx, table, host_only=True)
    assert st(lambda: kvq.set_window(10, 0)) == tc.TC_ERR_SHAPE and st(lambda: kvq.set_shared([0, 3], [32])) == tc.TC_ERR_SHAPE
    with pytest.raises(ValueError):
        plan.set_shared([0, 3], [16, 16])


@pytest.mark.parametrize("shared", [False, True])
def test_refusals_of_the_calls(tc, shared):  # noqa: F811
    q_start, ctx, table, blocks = batch([1] * 8, [4096] * 8, [(8, 4096)])
    pool = tc.make_pool(8, 2, 128, blocks, 1 << 20, 1 << 21)
    plan = tc.Plan(pool, q_start, ctx, table, host_only=True)
    plan.set_window(4000, 4)
    plan.set_shared([0, 8], [4096])
    call = tc.tc_shared_attention if shared else tc.tc_window_attention
    need = plan.shared_workspace_bytes if shared else plan.window_workspace_bytes
    assert need > 0
    run = lambda pool=pool, q=1 << 22, out=1 << 23, scale=0.1, ws=1 << 24, n=need: abi._status(tc, lambda: call(plan, pool, q, out, scale, ws, n))  # noqa: E731
    assert run(q=None) == tc.TC_ERR_NULL and run(out=None) == tc.TC_ERR_NULL
    assert run(q=(1 << 22) + 8) == tc.TC_ERR_ARG and run(out=(1 << 23) + 2) == tc.TC_ERR_ARG
    assert run(ws=None) == tc.TC_ERR_WORKSPACE and run(n=need - 1) == tc.TC_ERR_WORKSPACE and run(ws=(1 << 24) + 8) == tc.TC_ERR_ARG
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert run(scale=scale) == tc.TC_ERR_ARG
    assert run(pool=tc.make_pool(8, 2, 128, blocks, None, 1 << 21)) == tc.TC_ERR_NULL
    assert run(pool=tc.make_pool(8, 2, 128, blocks, 1 << 20, (1 << 21) + 8)) == tc.TC_ERR_ARG
    assert run(pool=tc.make_pool(8, 2, 64, blocks, 1 << 20, 1 << 21)) == tc.TC_ERR_SHAPE
    assert run(pool=tc.make_kvq_pool(8, 2, 128, blocks, 1 << 20, 1 << 21, 1 << 22).base) == tc.TC_ERR_SHAPE
    assert run() == tc.TC_ERR_ARG and "host-only" in tc.last_error()


def test_an_empty_batch_is_a_no_op(tc):  # noqa: F811
    pool = tc.make_pool(8, 2, 128, 32, 1 << 20, 1 << 21)
    plan = tc.Plan(pool, np.zeros(1, np.int32), np.zeros(0, np.int32), np.zeros((0, 1), np.int32), host_only=True)
    plan.set_window(5, 1)
    plan.set_shared([0], [])
    for call in (tc.tc_window_attention, tc.tc_shared_attention):
        call(plan, pool, None, None, 0.0)
    assert plan.window_workspace_bytes == plan.shared_workspace_bytes == 0 and C.sizeof(tc.tc_span_info) == 64


def test_a_window_past_32_bits_is_all_tokens(tc):  # noqa: F811
    plan = abi._plan(tc)
    lists = []
    for window, sinks in (((1 << 31) - 1, (1 << 31) - 1), (1 << 32, 1 << 40)):
        plan.set_window(window, sinks)
        lists.append([plan.span_items(kind) for kind in (0, 1, 2)])
    for a, b in zip(*lists):
        assert np.array_equal(a, b)
    assert abi._status(tc, lambda: plan.set_window((1 << 32) * -1 + 5)) == tc.TC_ERR_ARG


def test_shared_tokens_past_the_position_behind_all_tokens_are_refused(tc):  # noqa: F811
    """A sweep takes its rows to be behind what they share, at 2^31 - 1024: the tokens from there on would be left out."""
    shared = (1 << 31) - 80
    table = np.zeros((2, shared // 16 + 1), np.int32)
    plan = tc.Plan(tc.make_pool(8, 1, 64, 1), np.array([0, 2, 3], np.int32), np.array([shared, shared], np.int32), table, host_only=True)
    assert abi._status(tc, lambda: plan.set_shared([0, 2], [shared])) == tc.TC_ERR_SPAN
    assert abi._status(tc, lambda: plan.set_shared([0, 2], [AFTER + 16])) == tc.TC_ERR_SPAN
    plan.set_shared([0, 2], [AFTER])
    assert plan.span_items(0, True)[:, 11].min() == AFTER  # (and the own position of the chunk)
