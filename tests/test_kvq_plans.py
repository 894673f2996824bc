"""Plans on the CPU: what they say about batches whose tables share blocks, in 8 and in 16 bits, and the forms that chunks take in 8 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest

from test_abi_host import tc  # noqa: F401  (the fixture)


BITS = {8: "make_kvq_pool", 16: "make_pool"}


def plan(tc, ctx, rows, q_len=None, Hq=8, Hkv=2, D=128, nb=4000, bits=8):
    q_len = q_len or [1] * len(ctx)
    table = np.zeros((len(rows), max(len(r) for r in rows)), np.int32)
    for s, r in enumerate(rows):
        table[s, :len(r)] = r
    q_start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    return tc.Plan(getattr(tc, BITS[bits])(Hq, Hkv, D, nb), q_start, np.array(ctx, np.int32), table, host_only=True)


def test_decodes_that_attend_over_a_block_which_gets_rows_have_their_append_apart(tc):
    """Two rows of one request on either side of a page boundary: the second attends over the block that the first's row goes into (and may change the
    scale of), so both may not happen in one launch."""
    many = [[100 + 8 * i + j for j in range(8)] for i in range(400)]
    ctx = [100 + i % 20 for i in range(400)]
    for name, apart, p in [
            ("no block in two places", 0, plan(tc, [15, 16], [[3], [4, 5]])),
            ("a common prompt", 0, plan(tc, [32, 40, 47], [[1, 2, 3], [1, 2, 4], [1, 2, 5]])),
            ("either side of a boundary", 1, plan(tc, [15, 16], [[3], [3, 5]])),
            ("in the other order", 1, plan(tc, [16, 15], [[3, 5], [3]])),
            ("far from the end", 1, plan(tc, [3, 3000], [[7], list(range(20, 200)) + [7] + list(range(200, 207))])),
            ("twice in its own table", 1, plan(tc, [31], [[6, 6]])),
            ("beside a common prompt", 1, plan(tc, [32, 63, 64], [[1, 2, 3], [1, 2, 4, 5], [1, 2, 4, 5, 6]])),
            ("single waves", 0, plan(tc, ctx, many)),
            ("single waves, one of them", 1, plan(tc, ctx[:399] + [100], many[:399] + [many[5][:6] + [many[5][6]]])),
            ("ids whose last bits are alike", 0, plan(tc, [15, 16], [[3], [3 + (1 << 15), 3 + (1 << 16)]], nb=1 << 17)),
            ("the entries beyond the last token do not count", 0, plan(tc, [15, 16], [[3, 5], [4, 5]]))]:
        assert p.info.append_launch == apart, name
    # a batch with a chunk stores its rows first in any case
    assert plan(tc, [0, 3], [[1, 2], [3]], q_len=[20, 1]).info.append_launch == 1


def test_an_update_forgets_the_blocks_of_the_batch_before(tc):
    p = plan(tc, [15, 16], [[3], [3, 5]])
    assert p.info.append_launch == 1
    pool = tc.make_kvq_pool(8, 2, 128, 4000)
    p.update(pool, np.array([0, 1, 2], np.int32), np.array([15, 16], np.int32), np.array([[3, 0], [4, 5]], np.int32))
    assert p.info.append_launch == 0


@pytest.mark.parametrize("seed", range(20))
def test_tables_of_random_batches(tc, seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 30))
    ctx = rng.integers(0, 400, n)
    pages = ctx // 16 + 1
    nb = int(rng.integers(4, 30)) * int(pages.sum())
    rows = [rng.integers(0, nb, k).tolist() for k in pages]
    ids, last = np.concatenate(rows), [r[-1] for r in rows]
    p = plan(tc, ctx, rows, nb=nb)
    assert p.info.append_launch == int(len(set(last)) < sum(int((ids == b).sum()) for b in set(last)))


def test_decodes_in_16_bits_that_attend_over_a_block_which_gets_rows(tc):
    """The same: what the second would find in the first's slot depends on which of them is sooner."""
    for apart, ctx, rows in [(0, [15, 16], [[3], [4, 5]]), (0, [32, 40], [[1, 2, 3], [1, 2, 4]]), (1, [15, 16], [[3], [3, 5]]), (1, [3, 4], [[3], [3]]),
                             (1, [40, 41, 2], [[1, 2, 3], [1, 2, 3], [9]]), (1, [31], [[6, 6]])]:
        assert plan(tc, ctx, rows, bits=16).info.append_launch == apart, rows
    many = [[100 + 8 * i + j for j in range(8)] for i in range(400)]
    ctx = [100 + i % 20 for i in range(400)]
    assert plan(tc, ctx, many, bits=16).info.append_launch == 0
    assert plan(tc, ctx[:399] + [101], many[:399] + [many[0][:7]], bits=16).info.append_launch == 1
    assert plan(tc, [0, 3], [[1, 2], [3]], q_len=[20, 1], bits=16).info.append_launch == 1


def chunk_form(tc, Hq, Hkv, chunks, decodes=(), D=128, bits=8):
    """chunks: (tokens, offset); decodes: contexts"""
    q_len, ctx = [n for n, _ in chunks] + [1] * len(decodes), [c for _, c in chunks] + list(decodes)
    pages = [-(-(n + c) // 16) for n, c in zip(q_len, ctx)]
    start = np.concatenate([[0], np.cumsum(pages)])
    return plan(tc, ctx, [list(range(a, b)) for a, b in zip(start, start[1:])], q_len, Hq, Hkv, D, int(start[-1]) + 1, bits).info


@pytest.mark.parametrize("D", [64, 128])
def test_first_chunks_whose_halves_would_take_two_rounds(tc, D):
    """Items of 128 rows that are more than the compute units run one after the other in 8 bits: items of 256 where they are alike, halves where the
    second round is of short ones."""
    for Hq, Hkv, chunks, rows, items in [(40, 8, [(51, 0)] * 16, 256, 128), (40, 8, [(51, 300)] * 16, 256, 128), (40, 8, [(102, 0)] * 8, 256, 128),
                                         (24, 8, [(85, 0)] * 16, 256, 128), (10, 2, [(51, 0)] * 64, 256, 128), (40, 8, [(816, 0)], 128, 264),
                                         (40, 8, [(405, 0), (400, 0)], 128, 264), (104, 8, [(304, 0)], 128, 272), (40, 8, [(800, 0)], 128, 256)]:
        i = chunk_form(tc, Hq, Hkv, chunks, D=D)
        assert (i.rows_per_prefill_item, i.num_prefill_items, i.block_threads) == (rows, items, 512), chunks[:2]
    # in 16 bits halves of four waves, several to a unit
    i = chunk_form(tc, 40, 8, [(51, 0)] * 16, D=D, bits=16)
    assert (i.rows_per_prefill_item, i.num_prefill_items, i.block_threads) == (128, 384, 256)


def test_chunks_of_few_runs_a_head_are_levelled_in_8_bits(tc):
    """32 KV heads leave seven runs a head beside decodes: too few in 16 bits, where the same batches run whole."""
    for chunk, decodes in [((1136, 174), [999]), ((776, 1489), [441, 3539])]:
        i = chunk_form(tc, 32, 32, [chunk], decodes)
        assert (i.num_prefill_workgroups, i.block_threads) == (7 * 32, 512) and i.num_piece_partials > 0 and i.num_prefill_pieces > i.num_prefill_items
        i = chunk_form(tc, 32, 32, [chunk], decodes, bits=16)
        assert i.num_prefill_workgroups == i.num_prefill_pieces == i.num_prefill_items and i.num_piece_partials == 0


NO_MEMORY = """
import ctypes as C, resource, sys
import numpy as np
import paper_2508_01989_amd as tc
make = getattr(tc, sys.argv[1])
pool = make(8, 2, 128, 100)
shape = pool.base if hasattr(pool, "base") else pool
tc.lib()
n = 1 << 25
q_start, ctx, table = np.arange(n + 1, dtype=np.int32), np.zeros(n, np.int32), np.zeros((n, 1), np.int32)
batch, keep = tc._batch(q_start, ctx, table)
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
p = tc.Plan(pool, [0, 1], [3], [[5]], host_only=True)
resource.setrlimit(resource.RLIMIT_AS, (used + (64 << 20), resource.RLIM_INFINITY))
status = tc.lib().tc_plan_update(p.handle, C.byref(shape), C.byref(batch), None)
assert status == tc.TC_ERR_DEVICE and "memory" in tc.last_error(), (status, tc.last_error())
other = C.c_void_p()
assert tc.lib().tc_plan_create_host(C.byref(shape), C.byref(batch), C.byref(other)) == tc.TC_ERR_DEVICE and not other
info = tc.tc_plan_info()
assert tc.lib().tc_plan_get_info(p.handle, C.byref(info)) == 0 and info.num_seqs == info.total_q == info.append_launch == 0
p.update(pool, [0, 1, 2], [3, 20], [[5, 0], [6, 7]])
assert tc.lib().tc_plan_get_info(p.handle, C.byref(info)) == 0 and info.num_seqs == 2
print("done")
"""


@pytest.mark.parametrize("make", BITS.values())
def test_no_memory_for_a_plan_is_an_error(tc, make):
    """Nothing throws: a batch whose lists do not fit the memory that the process may have gets a status, and the plan serves the next one."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", NO_MEMORY, make], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "done", (r.returncode, r.stderr[-2000:])


@pytest.mark.parametrize("bits", BITS)
def test_pools_of_too_many_blocks_are_refused(tc, bits):
    for nb in (1 << 27, 1 << 59, (1 << 60) + 5, (1 << 62) + 1):  # (times 16 they are 2^31, -2^63 ..)
        with pytest.raises(tc.TcError) as e:
            tc.Plan(getattr(tc, BITS[bits])(8, 2, 128, nb), np.zeros(1, np.int32), np.zeros(0, np.int32), np.zeros((0, 1), np.int32), host_only=True)
        assert e.value.status == tc.TC_ERR_SHAPE
    tc.Plan(getattr(tc, BITS[bits])(8, 2, 128, (1 << 27) - 1), np.array([0, 1]), np.array([3]), np.array([[(1 << 27) - 2]]), host_only=True)
