"""The KV cache in 8 bits on the GPU: batches whose sequences share blocks, special numbers in every form.  Cases, oracle and bounds are those of test_gpu_kvq.py."""
import copy

import numpy as np
import pytest

from test_gpu_kvq import Case, Device, bits_of, check_attention, check_cache, tc  # noqa: F401  (tc: the fixture)

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
