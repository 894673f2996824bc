"""The KV cache in 8 bits on the GPU, through the C ABI, against the plain form in 64 bits (oracle/kvq.py): bytes and exponents of the cache
equal, what is read back equal, attention within a bound that counts its roundings.

The bound: probabilities and outputs are rounded to nearest in the element type (half a step, h = eps / 2, relative), sums are
held in 32 bits.  With a = sum_j p_j |v_j| / sum_j p_j the rounding of p moves an output by at most h a and its own rounding by at
most h |out|.  A probability of IEEE half below 2^-14 of the reference is rounded in steps of 2^-24 instead, which adds at most 2^-25 |v|
per key, and the probabilities' sum is at least about one.  32-bit arithmetic (score products, exponentials, sums) adds less than a fiftieth of h."""
import copy
import zlib

import numpy as np
import pytest

import oracle
from oracle import kvq

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def tc():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2508_01989_amd as m
    return m


def bits_of(x, dtype):
    if dtype == "fp16":
        return x.astype(np.float16).view(np.uint16)
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


class Case:
    """A batch with a history, its tensors (uint16 patterns) and block tables; rows of very different magnitudes, so that scales grow."""

    def __init__(self, name, Hq, Hkv, D, q_len, ctx, dtype="bf16", spread=3, spare=3):
        rng = np.random.default_rng(zlib.crc32(repr((name, dtype)).encode()))
        self.name, self.Hq, self.Hkv, self.D, self.dtype = name, Hq, Hkv, D, dtype
        self.q_len, self.ctx = np.array(q_len, np.int32), np.array(ctx, np.int32)
        self.S, self.kv = len(q_len), self.q_len + self.ctx
        self.q_start = np.concatenate([[0], np.cumsum(self.q_len)]).astype(np.int32)
        self.h_start = np.concatenate([[0], np.cumsum(self.ctx)]).astype(np.int32)
        pages = -(-self.kv // 16)
        self.blocks = int(pages.sum()) + spare
        ids = rng.permutation(self.blocks).astype(np.int32)
        self.table = np.zeros((self.S, int(pages.max())), np.int32)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = ids[at:at + n]
            at += n
        T, P = int(self.q_start[-1]), int(self.h_start[-1])

        def rows(n, heads):
            x = rng.standard_normal((n, heads, D), np.float32) * np.exp2(rng.integers(-spread, 1, (n, heads, 1))).astype(np.float32)
            return bits_of(x, dtype)

        self.q = bits_of(rng.standard_normal((T, Hq, D), np.float32) * 1.5, dtype)
        self.k_new, self.v_new, self.k_hist, self.v_hist = rows(T, Hkv), rows(T, Hkv), rows(P, Hkv), rows(P, Hkv)
        self.scale = float(np.float32(1.0 / np.sqrt(D)))

    def oracle_cache(self, new=True):
        c = kvq.Cache(self.blocks, self.Hkv, self.D, self.dtype)
        has = np.flatnonzero(self.ctx > 0)
        for s in has:
            a, b = self.h_start[s], self.h_start[s + 1]
            c.append([0, b - a], [0], self.table[s:s + 1], self.k_hist[a:b], self.v_hist[a:b])
        if new:
            c.append(self.q_start, self.ctx, self.table, self.k_new, self.v_new)
        return c

    def attention(self, cache, rows=None):
        """Outputs in 64 bits and the bound of this module's text."""
        code = oracle.FP16 if self.dtype == "fp16" else oracle.BF16
        kp, vp = cache.widened_pools(self.table, self.kv)
        args = (self.Hq, self.Hkv, self.D, 16, self.q_start, self.ctx, self.table, self.q, self.scale, rows)
        out = oracle.attention(kp, vp, *args, dtype=code)
        a = oracle.attention(kp, vp & np.uint16(0x7FFF), *args, dtype=code)
        bound = HALF_STEP[self.dtype] * 1.02 * (a + np.abs(out))
        if self.dtype == "fp16":
            v_max = max(float(np.abs(kvq.widen(x, "fp16")).max()) for x in (self.v_new, self.v_hist) if x.size)
            bound += int(self.kv.max()) * 2.0 ** -25 * v_max
        return out, bound + 1e-30


class Device:
    def __init__(self, tc, c, device="cuda:0", stream=None, poison=0x7F, one_by_one=False):
        import torch
        self.tc, self.c, self.torch = tc, c, torch
        self.stream = stream
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)  # noqa: E731
        n = c.blocks * c.Hkv * 16 * c.D
        self.k, self.v = (torch.full((n,), poison, dtype=torch.uint8, device=device) for _ in range(2))
        self.scales = torch.full((c.blocks * c.Hkv * 2,), 0xFF, dtype=torch.uint8, device=device)
        self.pool = tc.make_kvq_pool(c.Hq, c.Hkv, c.D, c.blocks, self.k, self.v, self.scales, dtype=tc.TC_FP16 if c.dtype == "fp16" else tc.TC_BF16)
        self.q, self.k_new, self.v_new, kh, vh = (up(x) for x in (c.q, c.k_new, c.v_new, c.k_hist, c.v_hist))
        has = np.flatnonzero(c.ctx > 0)
        for part in (has.reshape(-1, 1) if one_by_one else [has] if len(has) else []):
            start = np.concatenate([[0], np.cumsum(c.ctx[part])]).astype(np.int32)
            plan = tc.Plan(self.pool, start, np.zeros(len(part), np.int32), c.table[part])
            tc.tc_kvq_append(plan, self.pool, kh[c.h_start[part[0]]:], vh[c.h_start[part[0]]:])
            torch.cuda.synchronize()
            plan.destroy()
        self.plan = tc.Plan(self.pool, c.q_start, c.ctx, c.table)
        self.workspace = torch.full((max(16, self.plan.workspace_bytes),), 0xAB, dtype=torch.uint8, device=device)
        self.out = torch.full((int(c.q_start[-1]) + 1, c.Hq, c.D), -1, dtype=torch.int16, device=device)  # a row more: nothing may write it
        torch.cuda.synchronize()

    def append(self):
        self.tc.tc_kvq_append(self.plan, self.pool, self.k_new, self.v_new, stream=self.stream)

    def attention(self):
        self.tc.tc_kvq_mixed_attention(self.plan, self.pool, self.q, self.out, self.c.scale, self.workspace, stream=self.stream)

    def step(self):
        self.tc.tc_kvq_mixed_attention_append(self.plan, self.pool, self.q, self.k_new, self.v_new, self.out, self.c.scale, self.workspace,
                                              stream=self.stream)

    def cache(self):
        self.torch.cuda.synchronize()
        c = self.c
        return tuple(x.cpu().numpy().reshape(c.blocks, c.Hkv, -1) for x in (self.k, self.v, self.scales))

    def outputs(self):
        self.torch.cuda.synchronize()
        o = self.out.cpu().numpy().view(np.uint16)
        assert (o[-1] == 0xFFFF).all(), "wrote behind the last row"
        return kvq.widen(o[:-1], self.c.dtype)

    def read(self, seq):
        c, torch = self.c, self.torch
        n = int(c.kv.sum() if seq < 0 else c.kv[seq])
        k = torch.full((n + 1, c.Hkv, c.D), -1, dtype=torch.int16, device=self.k.device)
        v = torch.full_like(k, -1)
        self.tc.tc_kvq_read(self.plan, self.pool, seq, k, v, stream=self.stream)
        torch.cuda.synchronize()
        k, v = (x.cpu().numpy().view(np.uint16) for x in (k, v))
        assert (k[-1] == 0xFFFF).all() and (v[-1] == 0xFFFF).all(), "wrote behind the last token"
        return kvq.widen(k[:-1], c.dtype), kvq.widen(v[:-1], c.dtype)


def check_cache(dev, cache, tag):
    k, v, s = dev.cache()
    assert np.array_equal(s, cache.scales), f"{tag}: exponents differ at {np.argwhere(s != cache.scales)[:4].tolist()}"
    for name, got, want in (("K", k, cache.k), ("V", v, cache.v)):
        bad = np.argwhere(got != want)
        # the sign of a NaN is not defined
        bad = [b for b in bad.tolist() if not (got[tuple(b)] & 0x7F == 0x7F and want[tuple(b)] & 0x7F == 0x7F)]
        assert not bad, f"{tag}: {len(bad)} bytes of {name} differ, first {bad[:4]}"


def check_attention(got, want, bound, tag):
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{tag}: NaN in other places"
    over = np.nan_to_num(np.abs(got - want) / bound)
    assert over.max() <= 1.0, f"{tag}: {over.max():.3f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"
    return over.max()


SHAPES = {
    "one_token": (4, 1, 128, [1], [0]),
    "page_boundaries": (8, 2, 128, [1, 1, 1, 1, 1], [14, 15, 16, 31, 32]),
    "split_boundaries": (8, 2, 128, [1, 1, 1, 1], [126, 127, 128, 255]),
    "decodes_ragged": (32, 8, 128, [1, 1, 1], [3000, 1025, 777]),
    "decodes_of_every_length": (8, 2, 128, [1] * 70, list(range(70))),
    "many_short_decodes": (8, 2, 64, [1] * 600, [(7 * i) % 41 for i in range(600)]),
    "long_decode_many_partials": (8, 2, 128, [1, 1], [20000, 8191]),
    "teams_g16": (16, 1, 128, [1, 1, 1], [5000, 3000, 700]),
    "decodes_d64": (8, 2, 64, [1, 1, 1, 1, 1, 1], [100, 129, 600, 1500, 2047, 4100]),
    "g16_d64": (16, 1, 64, [70, 1, 1], [40, 900, 17]),
    "many_decodes_by_single_waves": (16, 8, 128, [1] * 96, [300 + 37 * i % 1100 for i in range(96)]),
    "two_rows": (4, 1, 128, [2], [0]),
    "ragged_chunk": (8, 2, 128, [77], [0]),
    "chunk_inside_a_page": (8, 2, 128, [5, 3], [3, 20]),
    "chunk_offset_unaligned": (8, 2, 128, [130], [37]),
    "chunk_and_decodes": (8, 2, 128, [40, 1, 70, 1], [5, 99, 300, 0]),
    "mha": (4, 4, 128, [300, 1], [20, 200]),
    "g3": (6, 2, 128, [100, 1], [28, 75]),
    "g5": (10, 2, 128, [120, 1], [0, 260]),
    "three_kv_heads": (12, 3, 128, [50, 1, 1], [100, 300, 15]),
    "five_kv_heads_d64": (5, 5, 64, [90, 1], [1200, 64]),
    "d64_chunk": (8, 2, 64, [200, 1, 1], [45, 1000, 17]),
    "sweeps_of_one_to_four_tiles": (8, 2, 128, [64, 65, 2, 30, 129, 1], [0, 0, 126, 99, 127, 5]),
    "cut_chunk": (32, 8, 128, [64, 1], [5000, 50]),
    "cut_d64": (4, 4, 64, [100, 1], [900, 30]),
    "levelled_chunk": (32, 8, 128, [700], [900]),
    "queue": (32, 8, 128, [520] + [1] * 24, [200] + [1500, 40, 2100, 900, 3300, 64] * 4),
    "chunk_beside_long_decodes": (8, 2, 128, [33] + [1] * 4, [5] + [1023, 1024, 8191, 8192]),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", SHAPES)
def test_step_against_the_plain_form(tc, name, dtype):
    c = Case(name, *SHAPES[name], dtype=dtype)
    print(f"[case] {name} {dtype}: S={c.S} T={int(c.q_start[-1])}", flush=True)
    before, after = c.oracle_cache(new=False), c.oracle_cache()
    dev = Device(tc, c)
    check_cache(dev, before, "history")
    dev.append()
    check_cache(dev, after, "append")
    dev.append()
    check_cache(dev, after, "append again")
    dev.attention()
    want, bound = c.attention(after)
    got = dev.outputs()
    worst = check_attention(got, want, bound, name)
    print(f"  worst {worst:.2f} of the bound", flush=True)
    for s in sorted({0, c.S // 2, c.S - 1}):
        for x, y in zip(dev.read(s), after.read(c.table[s], int(c.kv[s]))):
            assert np.array_equal(x, y), f"sequence {s} read back"
    for i, x in enumerate(dev.read(-1)):
        y = np.concatenate([after.read(c.table[s], int(c.kv[s]))[i] for s in range(c.S)])
        assert np.array_equal(x, y), "all sequences read back"
    # both in one call, on a cache of its own: the same bits
    one = Device(tc, c)
    one.step()
    check_cache(one, after, "step")
    assert np.array_equal(one.outputs(), got)
    one.step()
    check_cache(one, after, "step again")
    assert np.array_equal(one.outputs(), got)


SPECIAL = {
    # NaN and infinities among the new rows: (shape, [(tensor, row, head, element)])
    "chunk": ((8, 2, 128, [300, 1, 1], [70, 40, 500]), [("v", 5, 0, 3), ("v", 130, 1, 127), ("v", 131, 1, 127), ("k", 200, 0, 9), ("v", 299, 0, 64), ("v", 300, 1, 1)]),
    "chunk_d64": ((4, 4, 64, [150, 1], [33, 10]), [("v", 0, 1, 63), ("k", 149, 2, 0), ("v", 77, 3, 31)]),
    "first_chunk": ((16, 1, 128, [65], [0]), [("v", 64, 0, 5), ("v", 63, 0, 6), ("v", 0, 0, 7)]),
    "cut_chunk": ((8, 2, 128, [77], [1500]), [("v", 76, 0, 100), ("v", 1, 1, 0), ("k", 60, 1, 0)]),
    "levelled_chunk": ((32, 8, 128, [700], [900]), [("v", 300, 3, 77), ("v", 699, 4, 0), ("k", 650, 7, 1)]),
    "decodes": ((8, 2, 128, [1, 1, 1], [3, 1000, 64]), [("k", 0, 1, 5), ("v", 2, 0, 99)]),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", SPECIAL)
def test_nan_reaches_the_rows_that_attend_over_it_and_no_others(tc, name, dtype):
    shape, marks = SPECIAL[name]
    c = Case(name, *shape, dtype=dtype)
    inf, nan = (0x7C00, 0x7E01) if dtype == "fp16" else (0x7F80, 0x7FC1)
    for i, (x, row, head, d) in enumerate(marks):
        (c.k_new if x == "k" else c.v_new)[row, head, d] = (inf, nan, inf | 0x8000)[i % 3]
    print(f"[case] special {name} {dtype}", flush=True)
    cache = c.oracle_cache()
    dev = Device(tc, c)
    dev.step()
    check_cache(dev, cache, name)
    want, bound = c.attention(cache)
    assert np.isnan(want).any() and np.isfinite(want).any()
    check_attention(dev.outputs(), want, bound, name)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_pattern_is_quantised_and_read_back(tc, dtype):
    """All 65536 patterns of the type, in blocks of their own and one by one into blocks whose scale then grows, at both ends of the range."""
    u = np.arange(65536, dtype=np.uint16)
    rng = np.random.default_rng(7)
    c = Case("patterns", 4, 2, 64, [512, 512, 1, 1, 1], [0, 0, 0, 1, 2], dtype=dtype)
    c.k_new[:512], c.v_new[:512] = u.reshape(512, 2, 64), u[::-1].reshape(512, 2, 64)  # neighbours share a block
    c.k_new[512:1024], c.v_new[512:1024] = rng.permutation(u).reshape(512, 2, 64), rng.permutation(u).reshape(512, 2, 64)
    big, small = (0x7BFF, 0x0001) if dtype == "fp16" else (0x7F7F, 0x0001)
    c.k_hist[:], c.v_hist[:] = small, 0x0400
    c.k_new[1024:], c.v_new[1024:] = big, 0x8000 | big
    print(f"[case] patterns {dtype}", flush=True)
    cache = c.oracle_cache()
    dev = Device(tc, c)
    dev.append()
    check_cache(dev, cache, dtype)
    for s in range(c.S):
        for x, y in zip(dev.read(s), cache.read(c.table[s], int(c.kv[s]))):
            assert np.array_equal(x, y, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("S,Hq,Hkv", [(6, 8, 2), (240, 32, 8)])  # a split is run by a workgroup, by a wave
def test_new_tokens_of_decodes_at_the_ends_of_the_range(tc, S, Hq, Hkv, dtype):
    """Decodes whose new row is as large or as small as the type allows, or has infinities and NaN beside such numbers: the cache that the attention
    launch leaves, and NaN in the outputs."""
    c = Case(f"ends {S}", Hq, Hkv, 64, [1] * S, [(5 * i) % 50 + (i % 3 == 0) * 16 for i in range(S)], dtype=dtype)
    big, inf, nan = (0x7BFF, 0x7C00, 0x7E01) if dtype == "fp16" else (0x7F7F, 0x7F80, 0x7FC1)
    rng = np.random.default_rng(3)
    for i in range(S):
        for x in (c.k_new, c.v_new):
            x[i] = {0: big, 1: 1, 2: big | 0x8000, 3: x[i], 4: 0, 5: x[i]}[i % 6]
            if i % 6 == 0:
                x[i, 0, ::3] = rng.integers(0, 65536, 22, dtype=np.uint16)
            if i % 6 in (2, 5):
                x[i, 1, [1, 62]] = inf, nan
    print(f"[case] ends {S} {dtype}", flush=True)
    cache = c.oracle_cache()
    dev = Device(tc, c)
    assert (dev.plan.info.waves_per_item == 1) == (S == 240)
    dev.step()
    check_cache(dev, cache, "step")
    got = dev.outputs()
    for i in range(S):
        if i % 6 in (2, 5):  # (the query heads of KV head 1)
            assert np.isnan(got[i, 4:8]).all()
    plain = [i for i in range(S) if i % 6 in (1, 3, 4)]
    ordinary = copy.copy(c)
    ordinary.v_new = c.v_new[plain]  # (the bound of IEEE half is by the largest value)
    want, bound = ordinary.attention(cache)
    check_attention(got[plain], want[plain], bound[plain], "plain rows")
    apart = Device(tc, c)
    apart.append()
    check_cache(apart, cache, "append")
    apart.attention()
    assert np.array_equal(apart.outputs(), got, equal_nan=True)


def test_large_stream_of_decodes_in_one_call_and_in_two(tc):
    """Half a gigabyte of pages, where the append is a launch of its own: the bits of the two calls."""
    import torch
    Hq, Hkv, D, S = 32, 8, 128, 520
    rng = np.random.default_rng(21)
    ctx = rng.integers(440, 560, S).astype(np.int32)
    pages = -(-(ctx + 1) // 16)
    n = int(pages.sum())
    assert n * Hkv * 2 * 16 * D >= 500_000_000
    table = np.zeros((S, int(pages.max())), np.int32)
    ids, at = rng.permutation(n).astype(np.int32), 0
    for i, x in enumerate(pages):
        table[i, :x] = ids[at:at + x]
        at += x
    g = torch.Generator(device="cuda:0").manual_seed(5)
    byte = lambda m, lo, hi: torch.randint(lo, hi, (m,), dtype=torch.uint8, device="cuda:0", generator=g)  # noqa: E731
    pools = [byte(n * Hkv * 16 * D, 0, 0x7F) for _ in range(2)] + [byte(n * Hkv * 2, 115, 122)]
    row = lambda h: torch.randn((S, h, D), device="cuda:0", generator=g).bfloat16()  # noqa: E731
    q, k_new, v_new = row(Hq), row(Hkv), row(Hkv)
    got = []
    print("[case] large stream", flush=True)
    for both in (False, True):
        k, v, s = (x.clone() for x in pools)
        pool = tc.make_kvq_pool(Hq, Hkv, D, n, k, v, s)
        plan = tc.Plan(pool, np.arange(S + 1, dtype=np.int32), ctx, table)
        assert plan.info.waves_per_item == 1
        ws = torch.empty(max(16, plan.workspace_bytes), dtype=torch.uint8, device="cuda:0")
        out = torch.empty((S, Hq, D), dtype=torch.bfloat16, device="cuda:0")
        if both:
            tc.tc_kvq_mixed_attention_append(plan, pool, q, k_new, v_new, out, D ** -0.5, ws)
        else:
            tc.tc_kvq_append(plan, pool, k_new, v_new)
            tc.tc_kvq_mixed_attention(plan, pool, q, out, D ** -0.5, ws)
        torch.cuda.synchronize()
        got.append((k, v, s, out))
    for x, y in zip(*got):
        assert torch.equal(x, y)
    assert torch.isfinite(got[0][3].float()).all() and not torch.equal(got[0][0], pools[0])


def test_sequences_that_share_their_first_blocks(tc):
    """The whole blocks of a common prompt may stand in several tables: nothing is appended to them."""
    c = copy.copy(Case("shared", 8, 2, 128, [1, 1, 20], [100, 130, 97]))
    c.k_hist, c.v_hist, c.table = c.k_hist.copy(), c.v_hist.copy(), c.table.copy()
    for s in (1, 2):
        c.table[s, :6] = c.table[0, :6]
        for x in (c.k_hist, c.v_hist):
            x[c.h_start[s]:c.h_start[s] + 96] = x[:96]
    print("[case] shared blocks", flush=True)
    cache = c.oracle_cache()
    dev = Device(tc, c, one_by_one=True)  # (a call whose rows go to the same block twice is refused)
    dev.step()
    check_cache(dev, cache, "step")
    want, bound = c.attention(cache)
    check_attention(dev.outputs(), want, bound, "shared")


def test_blocks_beyond_two_and_four_gigabytes(tc):
    """The same batch at the far end of pools of 4.5 GB each: byte offsets pass 32 bits."""
    import torch
    c = Case("far", 16, 8, 128, [70, 1, 1], [100, 1300, 17])
    cache = c.oracle_cache()
    want, bound = c.attention(cache)
    far = 275000  # blocks before this batch's, 16 KiB each
    near = Device(tc, c)
    near.step()
    n = c.Hkv * 16 * c.D
    k = torch.zeros((far + c.blocks) * n, dtype=torch.uint8, device="cuda:0")
    v = torch.zeros_like(k)
    s = torch.zeros((far + c.blocks) * c.Hkv * 2, dtype=torch.uint8, device="cuda:0")
    fresh = Device(tc, c)
    k[far * n:], v[far * n:], s[far * c.Hkv * 2:] = fresh.k, fresh.v, fresh.scales
    pool = tc.make_kvq_pool(c.Hq, c.Hkv, c.D, far + c.blocks, k, v, s)
    plan = tc.Plan(pool, c.q_start, c.ctx, c.table + far)
    print("[case] far blocks", flush=True)
    tc.tc_kvq_mixed_attention_append(plan, pool, fresh.q, fresh.k_new, fresh.v_new, fresh.out, c.scale, fresh.workspace)
    out = fresh.outputs()
    assert np.array_equal(out, near.outputs())
    check_attention(out, want, bound, "far")
    assert torch.equal(k[far * n:], near.k) and torch.equal(v[far * n:], near.v) and torch.equal(s[far * c.Hkv * 2:], near.scales)
    assert not k[:far * n].any() and not v[:far * n].any() and not s[:far * c.Hkv * 2].any()
    n_tok = int(c.kv[1])
    ko = torch.empty((n_tok, c.Hkv, c.D), dtype=torch.int16, device="cuda:0")
    vo = torch.empty_like(ko)
    tc.tc_kvq_read(plan, pool, 1, ko, vo)
    torch.cuda.synchronize()
    for x, y in zip((ko, vo), cache.read(c.table[1], n_tok)):
        assert np.array_equal(kvq.widen(x.cpu().numpy().view(np.uint16), "bf16"), y)


def test_generation_over_one_plan_object(tc):
    """As a serving loop runs it: prompts in two chunks of odd lengths, then token by token beside each other, one plan object updated for every
    iteration; then the requests move into other blocks (read, append) and go on.  Cache and outputs of every iteration."""
    import torch
    rng = np.random.default_rng(11)
    Hq, Hkv, D, lens, steps = 8, 2, 128, [45, 97], 20
    total = [n + steps + 3 for n in lens]
    blocks = 40
    ids = rng.permutation(blocks).astype(np.int32)
    width = -(-max(total) // 16)
    table, table2 = ids[:2 * width].reshape(2, width), ids[2 * width:4 * width].reshape(2, width)
    rows = lambda n, h: bits_of(rng.standard_normal((n, h, D), np.float32) * np.exp2(rng.integers(-6, 3, (n, h, 1))).astype(np.float32), "bf16")  # noqa: E731
    q, k, v = ([rows(n, h) for n in total] for h in (Hq, Hkv, Hkv))
    cache = kvq.Cache(blocks, Hkv, D)
    dk, dv = (torch.full((blocks * Hkv * 16 * D,), 0x7F, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    ds = torch.full((blocks * Hkv * 2,), 0xFF, dtype=torch.uint8, device="cuda:0")
    pool = tc.make_kvq_pool(Hq, Hkv, D, blocks, dk, dv, ds)
    up = lambda x: torch.from_numpy(np.concatenate(x).view(np.int16)).to("cuda:0")  # noqa: E731
    done, plan, scale = [0, 0], None, float(np.float32(D ** -0.5))

    def iterate(seqs, counts, tab):
        nonlocal plan
        q_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        ctx = np.array([done[s] for s in seqs], np.int32)
        tab = np.ascontiguousarray(tab[seqs])
        part = lambda x: [x[s][done[s]:done[s] + n] for s, n in zip(seqs, counts)]  # noqa: E731
        if plan is None:
            plan = tc.Plan(pool, q_start, ctx, tab)
        else:
            plan.update(pool, q_start, ctx, tab)
        ws = torch.empty(max(16, plan.workspace_bytes), dtype=torch.uint8, device="cuda:0")
        out = torch.empty((int(q_start[-1]), Hq, D), dtype=torch.int16, device="cuda:0")
        tc.tc_kvq_mixed_attention_append(plan, pool, up(part(q)), up(part(k)), up(part(v)), out, scale, ws)
        torch.cuda.synchronize()
        cache.append(q_start, ctx, tab, np.concatenate(part(k)), np.concatenate(part(v)))
        kp, vp = cache.widened_pools(tab, ctx + counts)
        args = (Hq, Hkv, D, 16, q_start, ctx, tab, np.concatenate(part(q)), scale)
        want, mean = oracle.attention(kp, vp, *args), oracle.attention(kp, vp & np.uint16(0x7FFF), *args)
        check_attention(kvq.widen(out.cpu().numpy().view(np.uint16), "bf16"), want, HALF_STEP["bf16"] * 1.02 * (mean + np.abs(want)) + 1e-30, f"at {done}")
        for s, n in zip(seqs, counts):
            done[s] += n

    def same_cache():
        for x, y in ((dk, cache.k), (dv, cache.v), (ds, cache.scales)):
            assert np.array_equal(x.cpu().numpy().reshape(y.shape), y)

    print("[case] generation", flush=True)
    iterate([0], [30], table)
    iterate([0, 1], [15, 50], table)
    iterate([1], [47], table)
    for _ in range(steps):
        iterate([0, 1], [1, 1], table)
    same_cache()
    plan.update(pool, np.array([0, 1, 2], np.int32), np.array(done, np.int32) - 1, table)
    n = sum(done)
    ko = torch.empty((n, Hkv, D), dtype=torch.int16, device="cuda:0")
    vo = torch.empty_like(ko)
    tc.tc_kvq_read(plan, pool, -1, ko, vo)
    q_start = np.concatenate([[0], np.cumsum(done)]).astype(np.int32)
    plan.update(pool, q_start, np.zeros(2, np.int32), table2)
    tc.tc_kvq_append(plan, pool, ko, vo)
    torch.cuda.synchronize()
    was = [cache.read(table[s], done[s]) for s in range(2)]
    cache.append(q_start, np.zeros(2, np.int32), table2, ko.cpu().numpy().view(np.uint16), vo.cpu().numpy().view(np.uint16))
    for s in range(2):
        for x, y in zip(was[s], cache.read(table2[s], done[s])):
            assert np.array_equal(x, y)
    same_cache()
    for _ in range(3):
        iterate([1, 0], [1, 1], table2)
    same_cache()


@pytest.mark.parametrize("name", ["decodes_ragged", "many_decodes_by_single_waves", "chunk_and_decodes", "queue", "long_decode_many_partials"])
def test_step_captured_in_a_graph_and_on_another_stream(tc, name):
    import torch
    c = Case(name, *SHAPES[name])
    eager = Device(tc, c)
    eager.step()
    want, (k, v, s) = eager.outputs(), eager.cache()
    print(f"[case] graph {name}", flush=True)
    stream = torch.cuda.Stream()
    dev = Device(tc, c, stream=stream)
    with torch.cuda.stream(stream):
        dev.step()
    stream.synchronize()
    assert np.array_equal(dev.outputs(), want)
    fresh = [x.clone() for x in (dev.k, dev.v, dev.scales)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dev.step()
    torch.cuda.synchronize()
    for i in range(4):
        dev.out.zero_()
        dev.out[-1] = -1
        eager.step()  # eager work of the same kernels between the replays
        graph.replay()
        assert np.array_equal(dev.outputs(), want), f"replay {i}"
        for x, y in zip(fresh, (dev.k, dev.v, dev.scales)):
            assert torch.equal(x, y)
        assert np.array_equal(eager.outputs(), want)
    for x, y in zip(dev.cache(), (k, v, s)):
        assert np.array_equal(x, y)


def test_two_calls_at_once_on_two_streams(tc):
    """Plans, workspaces and caches of their own: nothing is shared."""
    import torch
    cases = [Case(n, *SHAPES[n]) for n in ("queue", "decodes_ragged")]
    alone = []
    for c in cases:
        d = Device(tc, c)
        d.step()
        alone.append((d.outputs(), d.cache()))
    streams = [torch.cuda.Stream() for _ in cases]
    devs = [Device(tc, c, stream=s) for c, s in zip(cases, streams)]
    print("[case] two streams", flush=True)
    for _ in range(6):
        for d in devs:
            d.step()
    for d, (out, cache) in zip(devs, alone):
        assert np.array_equal(d.outputs(), out)
        for x, y in zip(d.cache(), cache):
            assert np.array_equal(x, y)


@pytest.mark.parametrize("Hq,Hkv,D", [(257, 257, 64), (1024, 1024, 64), (130, 130, 128)])
def test_many_kv_heads(tc, Hq, Hkv, D):
    """More KV heads than compute units, and a number that no workgroup's waves divide."""
    c = Case("heads", Hq, Hkv, D, [20, 1, 1], [7, 33, 100], spread=1)
    cache = c.oracle_cache()
    print(f"[case] {Hkv} heads", flush=True)
    dev = Device(tc, c)
    dev.step()
    check_cache(dev, cache, "heads")
    check_attention(dev.outputs(), *c.attention(cache), "heads")
    for s in range(c.S):
        for x, y in zip(dev.read(s), cache.read(c.table[s], int(c.kv[s]))):
            assert np.array_equal(x, y)


@pytest.mark.parametrize("seed", range(4))
def test_attention_equals_that_of_a_cache_in_16_bits_which_holds_what_is_read_back(tc, seed):
    """Random batches of every form: append, attention, read, append to a cache in 16 bits, attention there.  Both attentions are over the same
    numbers, so they differ by at most the sum of their bounds; the mean magnitude in them comes from the 16-bit attention over |v|."""
    import random

    import torch
    rng, gen = random.Random(seed), torch.Generator(device="cuda:0").manual_seed(seed)
    for i in range(25):
        Hkv, G, D, dtype = rng.choice([1, 2, 3, 4, 8, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), rng.choice([64, 128]), rng.choice(["bf16", "fp16"])
        batch = [(int(2 ** rng.uniform(1, 11)), rng.choice([0, int(2 ** rng.uniform(0, 12))])) for _ in range(rng.choice([0, 1, 1, 2, 3]))]
        batch += [(1, int(2 ** rng.uniform(0, 11))) for _ in range(rng.choice([0, 1, 3, 10, 40, 200]))] or [(1, rng.randrange(30000))]
        rng.shuffle(batch)
        q_len, ctx = (np.array(x, np.int32) for x in zip(*batch))
        print(f"[case] {seed}.{i} {G * Hkv}/{Hkv} d{D} {dtype} chunks {[b for b in batch if b[0] > 1]} decodes {int((q_len == 1).sum())}", flush=True)
        kv = q_len + ctx
        q_start, all_rows = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (q_len, kv))
        pages = -(-kv // 16)
        blocks = int(pages.sum()) + 2
        ids, table, at = np.random.default_rng(i).permutation(blocks).astype(np.int32), np.zeros((len(kv), int(pages.max())), np.int32), 0
        for s, n in enumerate(pages):
            table[s, :n] = ids[at:at + n]
            at += n
        Hq, n, code = G * Hkv, blocks * Hkv * 16 * D, tc.TC_FP16 if dtype == "fp16" else tc.TC_BF16
        T = torch.float16 if dtype == "fp16" else torch.bfloat16
        row = lambda m, h: torch.randn((m, h, D), device="cuda:0", generator=gen).to(T)  # noqa: E731
        fill = lambda m, x, t: torch.full((m,), x, dtype=t, device="cuda:0")  # noqa: E731
        k8, v8, scales = fill(n, 0x7F, torch.uint8), fill(n, 0x7F, torch.uint8), fill(blocks * Hkv * 2, 0xFF, torch.uint8)
        k16, v16, v_abs = (fill(n, -1, torch.int16) for _ in range(3))
        pool = tc.make_kvq_pool(Hq, Hkv, D, blocks, k8, v8, scales, dtype=code)
        pool16, absolute = (tc.make_pool(Hq, Hkv, D, blocks, k16, x, dtype=code) for x in (v16, v_abs))
        old = np.flatnonzero(ctx > 0)
        if len(old):
            start = np.concatenate([[0], np.cumsum(ctx[old])]).astype(np.int32)
            history = tc.Plan(pool, start, np.zeros(len(old), np.int32), table[old])
            tc.tc_kvq_append(history, pool, row(int(start[-1]), Hkv), row(int(start[-1]), Hkv))
            torch.cuda.synchronize()
        m, total, scale = int(q_start[-1]), int(kv.sum()), D ** -0.5
        q, k_new, v_new = row(m, Hq), row(m, Hkv), row(m, Hkv)
        plan = tc.Plan(pool, q_start, ctx, table)
        ws = fill(max(16, plan.workspace_bytes), 0xAB, torch.uint8)
        out, want, mean = (torch.empty((m, Hq, D), dtype=T, device="cuda:0") for _ in range(3))
        tc.tc_kvq_mixed_attention_append(plan, pool, q, k_new, v_new, out, scale, ws)
        k, v = (torch.empty((total, Hkv, D), dtype=T, device="cuda:0") for _ in range(2))
        tc.tc_kvq_read(plan, pool, -1, k, v)
        whole, plan16 = tc.Plan(pool16, all_rows, np.zeros(len(kv), np.int32), table), tc.Plan(pool16, q_start, ctx, table)
        tc.tc_kv_append(whole, pool16, k, v)
        v_abs.copy_(v16 & 0x7FFF)
        ws16 = fill(max(16, plan16.workspace_bytes), 0xAB, torch.uint8)
        tc.tc_mixed_attention(plan16, pool16, q, want, scale, ws16)
        tc.tc_mixed_attention(plan16, absolute, q, mean, scale, ws16)
        torch.cuda.synchronize()
        h = HALF_STEP[dtype]
        bound = 2 * h * 1.02 * (mean.double() * (1 + 3 * h) + want.double().abs() * (1 + h))
        if dtype == "fp16":
            bound += 2 * int(kv.max()) * 2.0 ** -25 * v.double().abs().max()
        over = ((out.double() - want.double()).abs() / (bound + 1e-30)).max().item()
        assert over <= 1.0, over
