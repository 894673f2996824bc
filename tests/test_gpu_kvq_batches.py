"""Batches on the GPU whose sequences share blocks that get rows, and special numbers in every form of the 8-bit cache.  Cases, oracle and bounds are those of test_gpu_kvq.py."""
import copy

import numpy as np
import pytest

import oracle
from oracle import kvq
from test_gpu_kvq import HALF_STEP, SPECIAL, Case, Device, bits_of, check_attention, check_cache, tc  # noqa: F401  (tc: the fixture)

pytestmark = pytest.mark.gpu


def both_sides_of_a_boundary(R, Hq, Hkv, D, dtype):
    """R requests with two new rows each, as two decodes: the first ends a block, the second begins the next one and attends over the first."""
    m = [1 + i % 4 for i in range(R)]
    c = copy.copy(Case(f"boundary {R}", Hq, Hkv, D, [1] * (2 * R), [16 * x - 1 + s for x in m for s in (0, 1)], dtype=dtype))
    rng = np.random.default_rng(R)
    c.table, c.k_hist, c.v_hist, c.k_new, c.v_new = (x.copy() for x in (c.table, c.k_hist, c.v_hist, c.k_new, c.v_new))
    for i in range(R):
        a, b, n = c.h_start[2 * i], c.h_start[2 * i + 1], 16 * m[i] - 1
        c.table[2 * i + 1, :m[i]] = c.table[2 * i, :m[i]]
        for hist, new in ((c.k_hist, c.k_new), (c.v_hist, c.v_new)):
            hist[b:b + n] = hist[a:a + n]
            hist[b + n] = 0  # what the slot of the first new row held before
            new[2 * i] = bits_of(rng.standard_normal((Hkv, D), np.float32) * 40, dtype)  # the block's scale grows
    return c


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,Hq,Hkv", [(3, 8, 2), (120, 32, 8)])  # a split is run by a workgroup, by a wave
def test_decodes_that_attend_over_a_block_which_gets_rows(tc, R, Hq, Hkv, dtype):
    c = both_sides_of_a_boundary(R, Hq, Hkv, 64, dtype)
    cache = c.oracle_cache()
    want, bound = c.attention(cache)
    two, one = Device(tc, c, one_by_one=True), Device(tc, c, one_by_one=True)
    assert one.plan.info.append_launch == 1 and (one.plan.info.waves_per_item == 1) == (R == 120)
    print(f"[case] boundary {R} {dtype}", flush=True)
    two.append()
    two.attention()
    check_cache(two, cache, "append")
    check_attention(two.outputs(), want, bound, "two calls")
    for _ in range(3):
        one.out.zero_()
        one.out[-1] = -1
        one.step()
        check_cache(one, cache, "step")
        assert np.array_equal(one.outputs(), two.outputs())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,Hq,Hkv", [(3, 8, 2), (120, 32, 8)])  # a split is run by a workgroup, by a wave
def test_decodes_that_attend_over_a_block_which_gets_rows_in_16_bits(tc, R, Hq, Hkv, dtype):
    """The same batches, and pairs in one block, over a cache in 16 bits: one call gives the bits of the two, and those of the plain form's pools."""
    import torch
    c = both_sides_of_a_boundary(R, Hq, Hkv, 64, dtype)
    ctx = c.ctx.copy()
    for i in range(0, R, 2):  # every other pair one position sooner: both rows in the same block
        ctx[2 * i:2 * i + 2] -= 1
    kv = ctx + 1
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to("cuda:0")  # noqa: E731
    n, code = c.blocks * Hkv * 16 * 64, tc.TC_FP16 if dtype == "fp16" else tc.TC_BF16
    k0, v0 = oracle.new_pool(c.blocks, Hkv, 64)
    for s in range(c.S):
        a = c.h_start[s]
        oracle.kv_append(k0, v0, Hkv, 64, 16, np.array([0, ctx[s]], np.int32), np.zeros(1, np.int32), c.table[s:s + 1], c.k_hist[a:a + ctx[s]], c.v_hist[a:a + ctx[s]])
    q, k_new, v_new, got = up(c.q), up(c.k_new), up(c.v_new), []
    print(f"[case] boundary, 16 bits, {R} {dtype}", flush=True)
    for both in (False, True, True):
        k, v = up(k0), up(v0)
        assert k.numel() == n
        pool = tc.make_pool(Hq, Hkv, 64, c.blocks, k, v, dtype=code)
        plan = tc.Plan(pool, c.q_start, ctx, c.table)
        assert plan.info.append_launch == 1 and (plan.info.waves_per_item == 1) == (R == 120)
        ws = torch.empty(max(16, plan.workspace_bytes), dtype=torch.uint8, device="cuda:0")
        out = torch.zeros((c.S, Hq, 64), dtype=torch.int16, device="cuda:0")
        if both:
            tc.tc_mixed_attention_append(plan, pool, q, k_new, v_new, out, c.scale, ws)
        else:
            tc.tc_kv_append(plan, pool, k_new, v_new)
            tc.tc_mixed_attention(plan, pool, q, out, c.scale, ws)
        torch.cuda.synchronize()
        got.append((k, v, out))
    for x in got[1:]:
        for y, z in zip(got[0], x):
            assert torch.equal(y, z)
    oracle.kv_append(k0, v0, Hkv, 64, 16, c.q_start, ctx, c.table, c.k_new, c.v_new)
    assert np.array_equal(got[0][0].cpu().numpy().view(np.uint16).reshape(k0.shape), k0) and np.array_equal(got[0][1].cpu().numpy().view(np.uint16).reshape(v0.shape), v0)
    args = (Hq, Hkv, 64, 16, c.q_start, ctx, c.table, c.q, c.scale)
    otype = oracle.FP16 if dtype == "fp16" else oracle.BF16
    want, mean = oracle.attention(k0, v0, *args, dtype=otype), oracle.attention(k0, v0 & np.uint16(0x7FFF), *args, dtype=otype)
    bound = HALF_STEP[dtype] * 1.02 * (mean + np.abs(want)) + 1e-30
    if dtype == "fp16":  # (small probabilities, see test_gpu_kvq.py)
        bound += int(kv.max()) * 2.0 ** -25 * max(float(np.abs(kvq.widen(x, "fp16")).max()) for x in (c.v_new, c.v_hist))
    check_attention(kvq.widen(got[0][2].cpu().numpy().view(np.uint16), dtype), want, bound, "16 bits")


def attention_where_finite(c, cache):
    """Case.attention with the bound's largest value taken from the finite ones."""
    plain = copy.copy(c)
    plain.v_new, plain.v_hist = (np.where(np.isfinite(kvq.widen(x, c.dtype)), x, 0).astype(np.uint16) for x in (c.v_new, c.v_hist))
    return plain.attention(cache)  # (the cache holds what the tokens stand for: outputs are those of the batch itself)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", SPECIAL)
def test_rows_beside_nan_are_within_the_bound(tc, name, dtype):
    """The batches of test_gpu_kvq.py with NaN and infinities among the new rows, in either type: what stays finite."""
    shape, marks = SPECIAL[name]
    c = Case(name, *shape, dtype=dtype)
    for x, row, head, d in marks:
        (c.k_new if x == "k" else c.v_new)[row, head, d] = 0x7E01 if dtype == "fp16" else 0x7FC1
    print(f"[case] beside NaN {name} {dtype}", flush=True)
    cache = c.oracle_cache()
    dev = Device(tc, c)
    dev.step()
    check_cache(dev, cache, name)
    want, bound = attention_where_finite(c, cache)
    assert np.isfinite(bound[np.isfinite(want)]).all() and np.isnan(want).any()
    check_attention(dev.outputs(), want, bound, name)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths,long,waves", [("short", True, 4), ("short", False, 1), ("medium", True, 1)])
def test_nan_among_decodes(tc, lengths, long, waves, D, dtype):
    """NaN and infinities among new rows and older ones of decodes of one split and of several, run by workgroups and by single waves: in the rows and heads that
    attend over them, and nowhere else."""
    S, Hq, Hkv = 240, 32, 8
    ctx = [(5 * i) % 50 + (i % 3 == 0) * 16 if lengths == "short" else 300 + 37 * i % 1100 for i in range(S)]
    if long:
        ctx[11], ctx[100], ctx[201] = 1500, 3001, 5000
    c = Case(f"nan waves {D}", Hq, Hkv, D, [1] * S, ctx, dtype=dtype)
    inf, nan = (0x7C00, 0x7E01) if dtype == "fp16" else (0x7F80, 0x7FC1)
    rng = np.random.default_rng(5)
    for i in list(range(0, S, 6)) + [11, 100, 201]:
        x = (c.k_new, c.v_new)[i // 6 % 2]
        x[i, rng.integers(Hkv), rng.integers(D)] = (nan, inf, inf | 0x8000)[i % 3]
    for i in [i for i in (3, 15, 27, 100, 201) if ctx[i] > 0]:
        for x in (c.k_hist, c.v_hist):
            x[c.h_start[i] + rng.integers(ctx[i]), rng.integers(Hkv), rng.integers(D)] = nan
    print(f"[case] NaN among decodes: {lengths} {long} d{D} {dtype}", flush=True)
    cache = c.oracle_cache()
    want, bound = attention_where_finite(c, cache)
    bad = np.isnan(want)
    assert bad.any((1, 2)).sum() >= 40 and not bad.all(2).all(1).any() and np.isfinite(bound[~bad]).all()
    dev = Device(tc, c)
    assert dev.plan.info.waves_per_item == waves and dev.plan.info.append_launch == 0 and (dev.plan.info.num_partials > 0) == long
    dev.step()
    check_cache(dev, cache, "step")
    check_attention(dev.outputs(), want, bound, "step")
    apart = Device(tc, c)
    apart.append()
    apart.attention()
    assert np.array_equal(apart.outputs(), dev.outputs(), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("S,Hq,Hkv", [(6, 8, 2), (240, 32, 8)])  # a split is run by a workgroup, by a wave
def test_outputs_of_decodes_whose_new_values_are_large(tc, S, Hq, Hkv, dtype):
    """New rows of V at the highest exponent of IEEE half (in bf16 at 2^100: sums of numbers of the highest are beyond 32 bits): every output, each row by a bound of its own magnitudes."""
    c = Case(f"large {S}", Hq, Hkv, 64, [1] * S, [(5 * i) % 50 + (i % 3 == 0) * 16 for i in range(S)], dtype=dtype)
    rng = np.random.default_rng(S)
    for i in range(S):
        if i % 2 == 0:
            c.v_new[i] = bits_of((rng.standard_normal((Hkv, 64)) * (15000.0 if dtype == "fp16" else 2.0 ** 100)).astype(np.float32).clip(*(-6e4, 6e4) if dtype == "fp16" else (None, None)), dtype)
            if dtype == "fp16":
                c.v_new[i, 0, 5] = 0x7BFF
    print(f"[case] large {S} {dtype}", flush=True)
    cache = c.oracle_cache()
    assert dtype == "bf16" or (cache.scales == 8 + 127).any()
    dev = Device(tc, c)
    assert (dev.plan.info.waves_per_item == 1) == (S == 240)
    dev.step()
    check_cache(dev, cache, "step")
    got = dev.outputs()
    even = np.arange(S) % 2 == 0
    for some in (even, ~even):
        part = copy.copy(c)
        part.v_new = c.v_new[some]  # (the bound of IEEE half is by the largest value)
        want, bound = part.attention(cache)
        assert np.isfinite(want).all()
        check_attention(got[some], want[some], bound[some], "large" if some is even else "beside")
