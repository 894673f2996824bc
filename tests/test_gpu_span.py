"""Attention over a window with sinks, and of sequences that share cached tokens, on the GPU through the C ABI, against the plain form in 64 bits (oracle/span.py).

The bound: probabilities and outputs are rounded to nearest in the element type (half a step, h = eps / 2, relative), sums are held in 32 bits.  With
a = sum_j p_j |v_j| / sum_j p_j the rounding of p moves an output by at most h a and its own rounding by at most h |out|.  A probability of IEEE half below 2^-14 of the
reference is rounded in steps of 2^-24 instead, which adds at most 2^-25 |v| per key, and the probabilities' sum is at least about one.  32-bit arithmetic (score products,
exponentials, sums) adds less than a fiftieth of h."""
import zlib

import numpy as np
import pytest

from oracle import kvq
from oracle.span import attend
from test_gpu_rows import bits_of
from test_span_host import batch

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def tc():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2508_01989_amd as m
    return m


class Case:
    def __init__(self, Hq, Hkv, D, q_len, ctx, dtype="bf16", groups=None, seed=0, gain=1.5, spare=3):
        rng = np.random.default_rng(zlib.crc32(repr((Hq, Hkv, D, q_len, ctx, dtype, groups, seed)).encode()))
        self.Hq, self.Hkv, self.D, self.dtype, self.groups = Hq, Hkv, D, dtype, groups
        self.q_len, self.ctx = np.array(q_len, np.int64), np.array(ctx, np.int64)
        self.kv = self.q_len + self.ctx
        self.q_start, self.ctx32, self.table, self.blocks = batch(q_len, ctx, groups, seed, spare)
        self.T = int(self.q_start[-1])
        self.scale = float(np.float32(1.0 / np.sqrt(D)))
        self.q = bits_of(rng.standard_normal((self.T, Hq, D), np.float32) * gain, dtype)
        self.k, self.v = ([bits_of(rng.standard_normal((int(n), Hkv, D), np.float32), dtype) for n in self.kv] for _ in range(2))
        s = 0
        for n, shared in groups or []:
            for i in range(s, s + n):
                for x in (self.k, self.v):
                    x[i][:shared] = x[s][:shared]
            s += n

    def want(self, window=1 << 40, sinks=0, some=None):
        """Outputs and bounds; `some`: of at most that many rows of each sequence (the others are None)."""
        w = lambda x: kvq.widen(x, self.dtype)  # noqa: E731
        rng = np.random.default_rng(1)
        out, bound = np.full((self.T, self.Hq, self.D), np.nan), np.full((self.T, self.Hq, self.D), np.inf)
        for s, n in enumerate(self.q_len):
            a = int(self.q_start[s])
            rows = np.arange(n) if some is None or n <= some else np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, some)]))
            o, size = attend(w(self.q[a:a + n]), w(self.k[s]), w(self.v[s]), int(self.ctx[s]), self.scale, window, sinks, rows)
            out[a + rows] = o
            bound[a + rows] = HALF_STEP[self.dtype] * 1.02 * (size + np.abs(o)) + 1e-30
            if self.dtype == "fp16":
                bound[a + rows] += int(self.kv[s]) * 2.0 ** -25 * float(np.abs(w(self.v[s])).max())
        return out, bound


class Device:
    """The case's tensors; pools poisoned, then every token appended (its own rows too)."""

    def __init__(self, tc, c, device="cuda:0", stream=None, blocks=None, offset=0):
        import torch
        self.tc, self.c, self.torch, self.stream = tc, c, torch, stream
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)  # noqa: E731
        blocks = c.blocks if blocks is None else blocks
        n = blocks * c.Hkv * 16 * c.D
        self.k_pool, self.v_pool = (torch.full((n,), -1, dtype=torch.int16, device=device) for _ in range(2))
        self.pool = tc.make_pool(c.Hq, c.Hkv, c.D, blocks, self.k_pool, self.v_pool, dtype=tc.TC_FP16 if c.dtype == "fp16" else tc.TC_BF16)
        self.table = c.table + offset
        for s in range(len(c.kv)):
            plan = tc.Plan(self.pool, np.array([0, c.kv[s]], np.int32), np.zeros(1, np.int32), self.table[s:s + 1])
            tc.tc_kv_append(plan, self.pool, up(c.k[s]), up(c.v[s]))
            torch.cuda.synchronize()
        self.q = up(c.q)
        self.plan = tc.Plan(self.pool, c.q_start, c.ctx32, self.table)
        self.out = torch.full((c.T + 1, c.Hq, c.D), -1, dtype=torch.int16, device=device)  # a row more: nothing may write it
        self.ws = {}
        torch.cuda.synchronize()

    def set(self, window=None, sinks=0):
        """A window, or (without one) the case's groups."""
        self.shared = window is None
        if self.shared:
            g = self.c.groups
            self.plan.set_shared(np.concatenate([[0], np.cumsum([n for n, _ in g])]), [p for _, p in g], stream=self.stream)
        else:
            self.plan.set_window(window, sinks, stream=self.stream)
        n = self.plan.shared_workspace_bytes if self.shared else self.plan.window_workspace_bytes
        self.workspace = self.torch.full((max(16, n),), 0xAB, dtype=self.torch.uint8, device=self.out.device)
        return self

    def run(self, out=None, stream=None):
        call = self.tc.tc_shared_attention if self.shared else self.tc.tc_window_attention
        call(self.plan, self.pool, self.q, self.out if out is None else out, self.c.scale, self.workspace, stream=stream or self.stream)

    def outputs(self):
        self.torch.cuda.synchronize()
        o = self.out.cpu().numpy().view(np.uint16)
        assert (o[-1] == 0xFFFF).all(), "wrote behind the last row"
        return o[:-1].copy()

    def values(self):
        return kvq.widen(self.outputs(), self.c.dtype)

    def poke(self, s, j, k=None, v=None, d=None):
        """Another K or V pattern for token j of sequence s (element d or all), in the pool and in the case."""
        c = self.c
        block, t = int(self.table[s, j // 16]), j % 16
        dd = np.arange(c.D) if d is None else np.array([d])
        slot = t & 3 | (t & 4) << 1 | (t & 8) >> 1
        for pool, bits, mine, at in ((self.k_pool, k, c.k, (dd // 8 * 16 + t) * 8 + dd % 8), (self.v_pool, v, c.v, dd * 16 + slot)):
            if bits is None:
                continue
            p = pool.view(-1, c.Hkv, 16 * c.D)
            p[block, :, self.torch.from_numpy(at).to(p.device)] = int(np.array([bits], np.uint16).view(np.int16)[0])
            mine[s][j][:, dd] = bits


def check(d, window=None, sinks=0, some=None):
    d.set(window, sinks)
    d.run()
    got = d.values()
    want, bound = d.c.want(1 << 40 if window is None else window, sinks, some)
    have = ~np.isnan(want)
    assert not np.isnan(got).any()
    worst = float((np.abs(got - want) / bound)[have].max())
    assert worst <= 1, worst
    return d


MIXED = ([40, 1, 17, 1, 1, 70, 1, 2], [0, 0, 333, 15, 16, 200, 700, 31])
WINDOWS = [(1, 0), (7, 0), (16, 16), (17, 5), (33, 40), (100, 4), (64, 200), (1000, 0), (5, 1 << 30), ((1 << 31) - 1, (1 << 31) - 1)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads, D", [((8, 2), 128), ((8, 8), 64), ((5, 1), 128), ((16, 1), 64)])
def test_windows_of_mixed_batches(tc, heads, D, dtype):
    """Windows and sinks on, beside and across the borders of blocks, and beyond all of the tokens; chunks at any offset; decodes from their first token on."""
    d = Device(tc, Case(*heads, D, *MIXED, dtype))
    for window, sinks in WINDOWS:
        check(d, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads, D", [((8, 2), 128), ((8, 8), 64), ((5, 1), 64), ((16, 1), 128)])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_windows_of_decodes(tc, n, heads, D, dtype):
    ctx = [0] + np.random.default_rng(n).integers(0, 1500, n - 1).tolist()
    d = Device(tc, Case(*heads, D, [1] * n, ctx, dtype))
    for window, sinks in WINDOWS:
        check(d, window, sinks)


def test_long_window_of_one_decode(tc):
    """Cut into many parts, which a second launch combines."""
    d = check(Device(tc, Case(8, 2, 128, [1], [20000])), 17000, 33)
    assert d.plan.span_info().num_merge_items > 0
    check(Device(tc, Case(4, 4, 64, [1, 1], [9000, 12001], "fp16")), 8999, 0)


@pytest.mark.parametrize("heads, D, dtype", [((8, 2), 128, "bf16"), ((4, 4), 64, "fp16")])
def test_long_chunks(tc, heads, D, dtype):
    """Few sweeps, cut into pieces, and more than a chip has units for; windows shorter and longer than a row block."""
    d = Device(tc, Case(*heads, D, [777], [3001], dtype))
    for window, sinks in ((50, 0), (1000, 4), (3500, 20)):
        check(d, window, sinks, some=12)
    d = Device(tc, Case(16, 8, D, [2050, 1], [13, 900], dtype))
    for window, sinks in ((100, 3), (1500, 0)):
        check(d, window, sinks, some=12)


@pytest.mark.parametrize("D, dtype, window, sinks", [(128, "bf16", 2100, 5), (64, "fp16", 2301, 0), (128, "fp16", 40000, 0)])
def test_more_blocks_than_workgroups_at_a_time(tc, D, dtype, window, sinks):
    """Whole blocks of rows, of which the first of a sequence have one tile and the last ones dozens."""
    d = check(Device(tc, Case(32, 2, D, [2600, 2203], [0, 2100], dtype)), window, sinks, some=40)
    first = d.outputs()
    d.out.fill_(-1)
    d.run()
    assert np.array_equal(d.outputs(), first)


def test_a_window_past_every_token_is_mixed_attention(tc):
    import torch
    c = Case(8, 2, 128, *MIXED)
    d = check(Device(tc, c), 1 << 30, 0)
    out = torch.empty_like(d.out)
    ws = torch.empty(max(16, d.plan.workspace_bytes), dtype=torch.uint8, device="cuda:0")
    tc.tc_mixed_attention(d.plan, d.pool, d.q, out, c.scale, ws)
    torch.cuda.synchronize()
    a, b = d.values(), kvq.widen(out[:-1].cpu().numpy().view(np.uint16), "bf16")
    _, bound = c.want()
    assert np.all(np.abs(a - b) <= 2 * bound)


GROUPS = [
    ([1] * 6, [100, 64, 65, 80, 200, 79], [(6, 64)]),
    ([1] * 90, [32 + 7 * i for i in range(90)], [(90, 32)]),
    ([1] * 5, [100, 64, 65, 80, 200], [(2, 64), (1, 64), (2, 80)]),
    ([1] * 4, [0, 5, 0, 100], [(4, 0)]),
    ([70, 1, 1, 33, 1, 1], [160, 500, 170, 48, 48, 50], [(3, 160), (3, 48)]),
    ([1, 1, 130, 1], [16, 16, 16, 16], [(2, 16), (2, 16)]),
    ([1] * 40 + [3, 9], [1008] * 40 + [1008, 1024], [(42, 1008)]),
    ([150] * 2, [2048, 2100], [(2, 2048)]),
    ([1] * 2, [4096, 5000], [(2, 4096)]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads, D", [((8, 2), 128), ((8, 8), 64), ((5, 1), 64), ((16, 1), 128)])
@pytest.mark.parametrize("q_len, ctx, groups", GROUPS)
def test_shared_tokens(tc, q_len, ctx, groups, heads, D, dtype):
    """Groups of two to ninety, one alone, none; decodes and chunks; what is shared from one block to thousands of tokens, own tokens from the new one on."""
    check(Device(tc, Case(*heads, D, q_len, ctx, dtype, groups)), some=12)


def test_large_group(tc):
    check(Device(tc, Case(8, 2, 128, [1] * 300, (512 + np.random.default_rng(3).integers(0, 200, 300)).tolist(), "bf16", [(300, 512)])))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_attended_over_may_be_anything(tc, D, dtype):
    """NaN and infinities in K and V of one token: the rows that attend over it get them, the others keep every bit."""
    nan, inf = (0x7E00, 0x7C00) if dtype == "fp16" else (0x7FC0, 0x7F80)
    window, sinks = 40, 5
    for s, j in ((0, 3), (0, 20), (0, 64), (0, 99), (2, 300), (2, 334), (5, 4), (5, 5), (5, 150), (5, 200), (5, 230), (6, 661), (6, 660), (6, 3), (1, 0)):
        for which, bits in (("k", nan), ("v", nan), ("v", inf)):
            c = Case(8, 2, D, [100, 1, 17, 1, 1, 70, 1, 2], MIXED[1], dtype)
            d = Device(tc, c).set(window, sinks)
            d.run()
            clean = d.outputs()
            d.poke(s, j, **{which: bits})
            d.out.fill_(-1)
            d.run()
            got, values = d.outputs(), d.values()
            pos = np.concatenate([np.arange(a, a + n) for n, a in zip(c.q_len, c.ctx)])
            seq = np.repeat(np.arange(len(c.ctx)), c.q_len)
            sees = (seq == s) & (j <= pos) & ((pos - j < window) | (j < sinks))
            assert np.array_equal(got[~sees], clean[~sees]), (s, j, which)
            if bits == inf:
                assert (values[sees] == np.inf).all(), (s, j, which)
            else:
                assert np.isnan(values[sees]).all(), (s, j, which)


def test_one_element_of_one_token(tc):
    """An infinity of either sign, in one element, and both signs of it in what some rows attend over."""
    c = Case(4, 2, 64, [64], [0])
    d = Device(tc, c).set(20, 2)
    d.poke(0, 10, v=0x7F80, d=7)
    d.poke(0, 25, v=0xFF80, d=7)
    d.run()
    got = d.values()
    p = np.arange(64)
    ten, twentyfive = (p >= 10) & (p < 30), (p >= 25) & (p < 45)
    assert (got[ten & ~twentyfive][..., 7] == np.inf).all() and (got[~ten & twentyfive][..., 7] == -np.inf).all() and np.isnan(got[ten & twentyfive][..., 7]).all()
    assert np.isfinite(got[~ten & ~twentyfive]).all() and np.isfinite(np.delete(got, 7, -1)).all()


def test_blocks_outside_the_window_may_belong_to_anyone(tc):
    """The table's entries for blocks that no row attends over name a block full of NaN."""
    import torch
    c = Case(8, 2, 128, [30, 1], [500, 700], spare=3)
    d = Device(tc, c)
    used = set(c.table[0, :34]) | set(c.table[1, :44])
    free = next(b for b in range(c.blocks) if b not in used)
    table = d.table.copy()
    window, sinks = 100, 20
    for s, (first, last) in enumerate(((500, 529), (700, 700))):
        for page in range(last // 16 + 1):
            if page * 16 >= sinks and page * 16 + 15 < first - window + 1:
                table[s, page] = free
    d.plan = tc.Plan(d.pool, c.q_start, c.ctx32, table)
    check(d, window, sinks)
    assert (table == free).sum() > 20 and torch.isnan(d.k_pool.view(torch.bfloat16)).any()


GRAPHS = {  # q_len, ctx, groups, window: partial results combined by a second launch, by the last workgroup to leave one, or none
    "chunk": ([1] * 20 + [33], [1024 + 9 * i for i in range(21)], [(21, 1024)], 900),
    "decodes": ([1] * 3, [4096, 5000, 4111], [(3, 4096)], 4000),
    "short": ([1] * 3, [64, 80, 100], [(3, 64)], 50),
}


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("name", list(GRAPHS))
def test_graphs_streams_and_workspaces(tc, name, shared):
    """Captured and replayed with eager work between, on another stream, and two plans at a time on workspaces of their own: the same bits every time."""
    import torch
    q_len, ctx, groups, window = GRAPHS[name]
    c = Case(8, 2, 128, q_len, ctx, "bf16", groups)
    d = Device(tc, c)
    d.set() if shared else d.set(window, 4)
    info = d.plan.span_info(shared)
    assert (info.num_merge_items > 0, info.merge_launch) == {"chunk": (True, 1), "decodes": (True, int(shared)), "short": (shared, int(shared))}[name]
    d.run()
    want = d.outputs()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        d.run(stream=torch.cuda.current_stream())
    for _ in range(3):
        d.out.fill_(-1)
        d.workspace.fill_(0x7F)
        g.replay()
        assert np.array_equal(d.outputs(), want)
        d.run()
        assert np.array_equal(d.outputs(), want)
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [Device(tc, c) for _ in streams]
    for x in both:
        x.set() if shared else x.set(window, 4)
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st in zip(both, streams):
            x.run(stream=st)
    for x in both:
        assert np.array_equal(x.outputs(), want)


def test_lists_are_made_anew(tc):
    """One plan through several windows and batches, shorter and longer, as a serving loop has it."""
    c, c2 = Case(8, 2, 128, [1] * 9, [300 + i for i in range(9)]), Case(8, 2, 128, [50, 1], [0, 2000])
    d, d2 = Device(tc, c), Device(tc, c2)
    for x in (d, d2, d):
        d.plan.update(x.pool, x.c.q_start, x.c.ctx32, x.table)
        x.plan = d.plan
        for window, sinks in ((10, 0), (400, 2)):
            check(x, window, sinks)


def test_offsets_past_32_bits(tc):
    """Blocks whose elements lie beyond 2^31 of the pool's start."""
    c = Case(8, 8, 128, [20, 1, 1, 1], [64, 300, 290, 64], "bf16", [(4, 64)])
    blocks = (1 << 31) // (8 * 16 * 128) + c.blocks + 1
    d = Device(tc, c, blocks=blocks, offset=blocks - c.blocks)
    check(d, 50, 4)
    check(d)


def test_norm_rotation_append_and_both_attentions(tc):
    """The operators one after the other, as a layer of each kind has them: rows normalised, rotated and appended, then attention over a window, over shared tokens, and over everything."""
    import torch

    from oracle.rows import norm_rotate
    from test_gpu_rows import EPS
    c = Case(8, 2, 128, [1] * 5 + [40], [64 + 31 * i for i in range(6)], "bf16", [(6, 64)])
    d = Device(tc, c)
    rng = np.random.default_rng(8)
    rows = bits_of(rng.standard_normal((c.T, 12, 128), np.float32), "bf16")
    weights = [bits_of(1 + 0.2 * rng.standard_normal(128), "bf16") for _ in range(2)]
    freq = 10000.0 ** (-np.arange(64) / 64.0)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()  # noqa: E731
    t, w, f = up(rows), [up(x) for x in weights], torch.from_numpy(freq).cuda()
    tc.tc_qk_norm_rotate_append(d.plan, d.pool, tc.make_qkv_rows(t[:, :8], t[:, 8:10], t[:, 10:], w[0], w[1], EPS, f), d.q)
    torch.cuda.synchronize()
    # what went into the attention is taken from the device, so that its bound holds for it, and compared with the plain form itself
    pos = np.concatenate([np.arange(a, a + n) for n, a in zip(c.q_len, c.ctx)])
    c.q = d.q.cpu().numpy().view(np.uint16)
    for s in range(6):
        one = tc.Plan(d.pool, np.array([0, c.q_len[s]], np.int32), c.ctx32[s:s + 1], d.table[s:s + 1])
        k, v = (torch.empty((int(c.kv[s]), 2, 128), dtype=torch.int16, device="cuda:0") for _ in range(2))
        tc.tc_kv_gather(one, d.pool, 0, k, v)
        torch.cuda.synchronize()
        k, v = k.cpu().numpy().view(np.uint16), v.cpu().numpy().view(np.uint16)
        a, b = int(c.q_start[s]), int(c.q_start[s + 1])
        assert np.array_equal(k[:c.ctx[s]], c.k[s][:c.ctx[s]]) and np.array_equal(v[:c.ctx[s]], c.v[s][:c.ctx[s]]) and np.array_equal(v[c.ctx[s]:], rows[a:b, 10:])
        want, size = norm_rotate(kvq.widen(np.ascontiguousarray(rows[a:b, 8:10]), "bf16"), kvq.widen(weights[1], "bf16"), EPS, freq, 128, False, pos[a:b])
        assert np.all(np.abs(kvq.widen(k[c.ctx[s]:], "bf16") - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size)
        c.k[s], c.v[s] = k, v
    check(d, 60, 4)
    check(d)
    out = torch.empty_like(d.out)
    ws = torch.empty(max(16, d.plan.workspace_bytes), dtype=torch.uint8, device="cuda:0")
    tc.tc_mixed_attention(d.plan, d.pool, d.q, out, c.scale, ws)
    torch.cuda.synchronize()
    _, bound = c.want()
    assert np.all(np.abs(kvq.widen(out[:-1].cpu().numpy().view(np.uint16), "bf16") - d.values()) <= 2 * bound)
