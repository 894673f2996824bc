"""Norm and rotation of the rows of q and k on the GPU, through the C ABI, against the plain form in 64 bits (oracle/rows.py), and the form that appends against
the two calls it stands for, bit for bit.

The bound: the result is rounded once (half a step, relative; half of the smallest step below the smallest normal number).  Before that, in 32 bits (u = 2^-24): the sum
of D squares takes a chain of 12 additions at most and a product each, 13 u, which the root halves; mean, eps, root, quotient, weight and product add 6 u.  A rotation's
products and their sum add 2 u of |a| + |b|, and cos and sin are each off by less than 4 u (their argument's rounding, pi u, included).  Together below 20 u (|a| + |b|); 32 u is taken."""
import zlib

import numpy as np
import pytest

from oracle import kvq
from oracle.rows import norm_rotate

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
SMALLEST = {"bf16": 2.0 ** -133 / 2, "fp16": 2.0 ** -24 / 2}
EPS = 1e-6


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
    """A batch, its rows in one tensor [T][pad + Hq + 2 Hkv][D] (uint16 patterns) and block tables over a pool with blocks to spare."""

    def __init__(self, Hq, Hkv, D, q_len, ctx, dtype="bf16", rotary=None, adjacent=False, base=10000.0, pad=0, seed=0):
        rng = np.random.default_rng(zlib.crc32(repr((Hq, Hkv, D, q_len, ctx, dtype, rotary, adjacent, seed)).encode()))
        self.Hq, self.Hkv, self.D, self.dtype, self.adjacent = Hq, Hkv, D, dtype, adjacent
        self.rotary = D if rotary is None else rotary
        self.q_len, self.ctx = np.array(q_len, np.int32), np.array(ctx, np.int32)
        self.q_start = np.concatenate([[0], np.cumsum(self.q_len)]).astype(np.int32)
        self.T = int(self.q_start[-1])
        pages = -(-(self.q_len.astype(np.int64) + self.ctx) // 16)
        first = self.ctx // 16  # pages before the new rows share one block: nothing is written there
        self.blocks = int((pages - first).sum()) + 3
        ids = rng.permutation(self.blocks).astype(np.int32)
        self.table = np.full((len(q_len), int(pages.max())), ids[-1], np.int32)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, first[s]:n] = ids[at:at + n - first[s]]
            at += n - first[s]
        self.rows = bits_of(rng.standard_normal((self.T, pad + Hq + 2 * Hkv, D), np.float32) * np.exp2(rng.integers(-6, 7, (self.T, 1, 1))), dtype)
        self.pad = pad
        self.weights = [bits_of(1 + 0.3 * rng.standard_normal(D), dtype) for _ in range(2)]
        self.freq = base ** (-2.0 * np.arange(self.rotary // 2) / max(self.rotary, 1))
        self.positions = np.concatenate([np.arange(c, c + n) for n, c in zip(self.q_len, self.ctx)]) if len(q_len) else np.zeros(0, int)

    def parts(self):
        a = self.pad
        return self.rows[:, a:a + self.Hq], self.rows[:, a + self.Hq:a + self.Hq + self.Hkv], self.rows[:, a + self.Hq + self.Hkv:]

    def want(self, which, weight=True, positions=None):
        x = kvq.widen(np.ascontiguousarray(self.parts()[which]), self.dtype)
        w = kvq.widen(self.weights[which], self.dtype) if weight else None
        y, size = norm_rotate(x, w, EPS, self.freq, self.rotary, self.adjacent, self.positions if positions is None else positions)
        return y, HALF_STEP[self.dtype] * np.abs(y) + 32 * 2.0 ** -24 * (1 + HALF_STEP[self.dtype]) * size + SMALLEST[self.dtype]


class Device:
    def __init__(self, tc, c, device="cuda:0", poison=-1, stream=None):
        import torch
        self.tc, self.c, self.torch, self.stream = tc, c, torch, stream
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)  # noqa: E731
        self.rows, self.weights = up(c.rows), [up(w) for w in c.weights]
        self.freq = torch.from_numpy(c.freq).to(device)
        n = c.blocks * c.Hkv * 16 * c.D
        self.k_pool, self.v_pool, self.k_ref, self.v_ref = (torch.full((n,), poison, dtype=torch.int16, device=device) for _ in range(4))
        dt = tc.TC_FP16 if c.dtype == "fp16" else tc.TC_BF16
        self.pool, self.ref = (tc.make_pool(c.Hq, c.Hkv, c.D, c.blocks, k, v, dtype=dt) for k, v in ((self.k_pool, self.v_pool), (self.k_ref, self.v_ref)))
        self.plan = tc.Plan(self.pool, c.q_start, c.ctx, c.table)
        self.q_out, self.q_out2 = (torch.full((c.T + 1, c.Hq, c.D), poison, dtype=torch.int16, device=device) for _ in range(2))
        self.k_out = torch.full((c.T + 1, c.Hkv, c.D), poison, dtype=torch.int16, device=device)
        torch.cuda.synchronize()

    def of(self, weights=(True, True), positions=None, **kw):
        c, a = self.c, self.c.pad
        r = self.rows
        return self.tc.make_qkv_rows(r[:, a:a + c.Hq], r[:, a + c.Hq:a + c.Hq + c.Hkv], r[:, a + c.Hq + c.Hkv:], q_weight=self.weights[0] if weights[0] else None,
                                     k_weight=self.weights[1] if weights[1] else None, eps=EPS, freq=self.freq if c.rotary else None, rotary_dim=c.rotary,
                                     adjacent=c.adjacent, positions=positions, **kw)

    def host(self, t):
        self.torch.cuda.synchronize()
        return t.cpu().numpy().view(np.uint16)

    def values(self, t):
        o = self.host(t)
        assert (o[-1] == 0xFFFF).all(), "wrote behind the last row"
        return kvq.widen(o[:-1], self.c.dtype)


def check(tc, c, weights=(True, True), positions=None):
    d = Device(tc, c)
    rows = d.of(weights, None if positions is None else d.torch.from_numpy(positions.astype(np.int32)).cuda())
    tc.tc_qk_norm_rotate(d.plan, rows, d.q_out, d.k_out)
    for which, got in ((0, d.values(d.q_out)), (1, d.values(d.k_out))):
        want, bound = c.want(which, weights[which], positions)
        assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())
    # and with the append: bit for bit the two calls, every other byte of the pool left alone
    tc.tc_qk_norm_rotate_append(d.plan, d.pool, rows, d.q_out2)
    v = d.rows[:, c.pad + c.Hq + c.Hkv:].contiguous()
    tc.tc_kv_append(d.plan, d.ref, d.k_out, v)
    assert np.array_equal(d.host(d.q_out), d.host(d.q_out2))
    assert np.array_equal(d.host(d.k_pool), d.host(d.k_ref)) and np.array_equal(d.host(d.v_pool), d.host(d.v_ref))
    return d


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(8, 8), (10, 2), (1, 1), (16, 1)])
def test_batches_of_all_kinds(tc, heads, D, dtype):
    """Decodes on first, middle and last tokens of a page, chunks that begin and end inside pages, single tokens at position 0."""
    check(tc, Case(*heads, D, [1, 1, 1, 1, 37, 5, 16, 1, 33, 2], [0, 15, 16, 1000, 0, 14, 32, 7, 12345, 31], dtype))


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("D, rotary", [(128, 0), (128, 8), (128, 48), (128, 64), (128, 120), (64, 8), (64, 24), (64, 32)])
def test_part_of_a_head_is_rotated(tc, D, rotary, adjacent):
    check(tc, Case(6, 3, D, [1, 20, 1], [100, 7, 3], "fp16", rotary, adjacent))


@pytest.mark.parametrize("weights", [(False, False), (True, False), (False, True)])
def test_norm_of_one_or_none(tc, weights):
    check(tc, Case(8, 2, 128, [1, 40, 1], [9, 100, 63]), weights)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_far_positions(tc, dtype):
    """Angles of some 10^6 and 10^9 turns' worth of radians, from the plan and given."""
    check(tc, Case(4, 2, 64, [1, 17], [1 << 20, (1 << 20) + 77], dtype, base=500000.0))
    c = Case(4, 2, 64, [1, 17], [5, 77], dtype)
    check(tc, c, positions=np.concatenate([[2 ** 31 - 1, 2 ** 30 + 1, 0, -7], np.arange(14) * 99999989]))


def test_rows_apart_and_packed(tc):
    """q, k and v in a tensor with more in it, and rows that are their own output."""
    import torch
    check(tc, Case(8, 2, 128, [1, 23], [4, 50], pad=3))
    c = Case(8, 2, 128, [1, 23], [4, 50])
    d = check(tc, c)
    q, k = (d.rows[:, a:b].contiguous() for a, b in ((0, 8), (8, 10)))
    rows = tc.make_qkv_rows(q, k, q_weight=d.weights[0], k_weight=d.weights[1], eps=EPS, freq=d.freq)
    tc.tc_qk_norm_rotate(d.plan, rows, q, k)
    torch.cuda.synchronize()
    assert torch.equal(q, d.q_out[:-1]) and torch.equal(k, d.k_out[:-1])


@pytest.mark.parametrize("dtype, sizes", [("bf16", [0, -149, -120, 120, 126]), ("fp16", [0, -24, 15])])
def test_values_at_the_ends_of_the_type(tc, dtype, sizes):
    """Heads whose squares leave 32 bits, at either end, and heads of zeros."""
    c = Case(4, 2, 128, [len(sizes) + 1], [11], dtype)
    x = kvq.widen(c.rows, dtype)
    x = x / np.abs(x).max((1, 2), keepdims=True)
    scale = np.array([2.0 ** s for s in sizes] + [0.0])[:, None, None]
    with np.errstate(over="ignore"):
        c.rows = bits_of(x * scale, dtype)
    check(tc, c)


def test_nan_and_infinity_stay_in_their_head(tc):
    c = Case(4, 2, 64, [6], [3])
    c.rows[2, 1, 5], c.rows[3, 5, 0], c.rows[4, 0, 7] = 0x7FC0, 0x7F80, 0xFF80
    d = Device(tc, c)
    tc.tc_qk_norm_rotate(d.plan, d.of(), d.q_out, d.k_out)
    got = np.concatenate([d.values(d.q_out), d.values(d.k_out)], 1)
    bad = np.zeros((6, 6), bool)
    bad[2, 1] = bad[3, 5] = bad[4, 0] = True
    assert np.array_equal(np.isnan(got).any(-1), bad) and np.isnan(got[2, 1]).all()


def test_large_batches(tc):
    """More workgroups than run at once: 515 decodes, and a chunk of 3001."""
    rng = np.random.default_rng(5)
    check(tc, Case(10, 2, 64, [1] * 515, rng.integers(0, 300, 515).tolist(), "fp16"))
    check(tc, Case(5, 1, 128, [3001, 1], [13, 5]))


def test_rows_of_a_plan_for_a_cache_in_8_bits(tc):
    """tc_qk_norm_rotate serves both kinds of plan: what it leaves is appended by tc_kvq_append."""
    import torch
    c = Case(8, 2, 128, [1, 23, 1], [4, 50, 15])
    d = check(tc, c)
    n = c.blocks * c.Hkv * 16 * c.D
    k8, v8, scales = (torch.zeros(m, dtype=torch.uint8, device="cuda:0") for m in (n, n, c.blocks * c.Hkv * 2))
    pool = tc.make_kvq_pool(c.Hq, c.Hkv, c.D, c.blocks, k8, v8, scales)
    plan = tc.Plan(pool, c.q_start, c.ctx, c.table)
    d.q_out2.fill_(-1)
    k_out = torch.empty_like(d.k_out)
    tc.tc_qk_norm_rotate(plan, d.of(), d.q_out2, k_out)
    tc.tc_kvq_append(plan, pool, k_out, d.rows[:, 10:].contiguous())
    torch.cuda.synchronize()
    assert torch.equal(d.q_out2, d.q_out) and torch.equal(k_out[:-1], d.k_out[:-1])
    assert int(k8.max()) > 0 and int(scales.max()) > 0


def test_in_a_graph_and_on_another_stream(tc):
    import torch
    c = Case(8, 2, 128, [1, 23, 1], [4, 50, 15])
    d = check(tc, c)
    q, kp, vp = d.q_out.clone(), d.k_pool.clone(), d.v_pool.clone()
    s = torch.cuda.Stream()
    rows = d.of()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        tc.tc_qk_norm_rotate_append(d.plan, d.pool, rows, d.q_out2, stream=torch.cuda.current_stream())
    for _ in range(3):
        for t in (d.q_out2, d.k_pool, d.v_pool):
            t.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(d.q_out2[:-1], q[:-1]) and torch.equal(d.k_pool, kp) and torch.equal(d.v_pool, vp)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("D, rotary", [(128, 0), (128, 48), (64, 0), (64, 24)])
def test_elements_behind_the_rotated_ones_keep_every_bit(tc, D, rotary, adjacent, dtype):
    """Without a weight the rest of a head is a copy: infinities, NaN, zeros of either sign and the smallest numbers reach no other element."""
    nan, inf = (0x7E00, 0x7C00) if dtype == "fp16" else (0x7FC0, 0x7F80)
    c = Case(6, 3, D, [1, 20, 1], [100, 7, 3], dtype, rotary, adjacent)
    rng = np.random.default_rng(D + rotary)
    some = rng.random(c.rows.shape) < 0.2
    some[..., :rotary] = False
    c.rows[some] = rng.choice(np.array([nan, inf, inf | 0x8000, 0x8000, 0, 1, 0x8001], np.uint16), int(some.sum()))
    d = Device(tc, c)
    rows = d.of((False, False))
    tc.tc_qk_norm_rotate(d.plan, rows, d.q_out, d.k_out)
    for which, t in ((0, d.q_out), (1, d.k_out)):
        assert np.array_equal(d.host(t)[:-1][..., rotary:], c.parts()[which][..., rotary:])
        want, size = norm_rotate(kvq.widen(np.ascontiguousarray(c.parts()[which][..., :rotary]), dtype), None, EPS, c.freq, rotary, adjacent, c.positions)
        assert np.all(np.abs(d.values(t)[..., :rotary] - want) <= HALF_STEP[dtype] * np.abs(want) + 32 * 2.0 ** -24 * (1 + HALF_STEP[dtype]) * size + SMALLEST[dtype])
    tc.tc_qk_norm_rotate_append(d.plan, d.pool, rows, d.q_out2)
    tc.tc_kv_append(d.plan, d.ref, d.k_out, d.rows[:, c.Hq + c.Hkv:].contiguous())
    assert np.array_equal(d.host(d.q_out), d.host(d.q_out2)) and np.array_equal(d.host(d.k_pool), d.host(d.k_ref)) and np.array_equal(d.host(d.v_pool), d.host(d.v_ref))



@pytest.mark.parametrize("adjacent", [False, True])
def test_weights_at_the_ends_of_the_type(tc, adjacent):
    """Rows of 2^-46 and 2^46 with weights of 2^100 and 2^-100, and elements that are zero: the root and the weight lie apart by more than 32 bits hold, the results do not."""
    c = Case(4, 2, 128, [1, 20], [9, 100], "bf16", None, adjacent)
    rng = np.random.default_rng(4)
    x = rng.standard_normal(c.rows.shape) * np.exp2(rng.choice([-46, 0, 46], c.rows.shape[:1]))[:, None, None]
    x[rng.random(x.shape) < 0.1] = 0
    c.rows = bits_of(x.astype(np.float32), "bf16")
    c.weights = [bits_of(((1 + 0.3 * rng.standard_normal(128)) * np.exp2(rng.choice([-100, 0, 100], 128))).astype(np.float32), "bf16") for _ in range(2)]
    d = Device(tc, c)
    eps = float(np.float32(1e-37))
    a = c.Hq
    rows = tc.make_qkv_rows(d.rows[:, :a], d.rows[:, a:a + 2], d.rows[:, a + 2:], d.weights[0], d.weights[1], eps, d.freq, adjacent=adjacent)
    tc.tc_qk_norm_rotate(d.plan, rows, d.q_out, d.k_out)
    for which, t in ((0, d.q_out), (1, d.k_out)):
        want, size = norm_rotate(kvq.widen(np.ascontiguousarray(c.parts()[which]), "bf16"), kvq.widen(c.weights[which], "bf16"), eps, c.freq, 128, adjacent, c.positions)
        bound = HALF_STEP["bf16"] * np.abs(want) + 32 * 2.0 ** -24 * (1 + HALF_STEP["bf16"]) * size + SMALLEST["bf16"]
        got = d.values(t)
        assert np.all(np.abs(got - want) <= bound), (int(np.isnan(got).sum()), float(np.nanmax(np.abs(got - want) / bound)))


@pytest.mark.parametrize("D, heads, dtype", [(128, (5, 1), "bf16"), (64, (4, 2), "fp16")])
def test_a_workgroup_to_each_page(tc, D, heads, dtype):
    """A chunk of so many pages that each has one workgroup, whose waves take one task after the other."""
    check(tc, Case(*heads, D, [6400, 1], [13, 5], dtype))
