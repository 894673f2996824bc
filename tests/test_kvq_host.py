"""The KV cache in 8 bits, on the CPU: the plain form that the GPU tests compare with, the plans, and what the calls refuse."""
import ctypes as C

import numpy as np
import pytest

import test_abi_host as abi
import workloads as W
from oracle import kvq
from test_abi_host import tc  # noqa: F401  (the fixture)


def test_e4m3_numbers():
    n = kvq.NUMBER
    assert (n[0x00], n[0x01], n[0x08], n[0x38], n[0x7E], n[0xFE]) == (0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -448.0)
    assert np.isnan(n[0x7F]) and np.isnan(n[0xFF]) and np.all(np.diff(n[:127]) > 0) and np.array_equal(n[128:255], -n[:127])


@pytest.mark.parametrize("top", [448.0, 240.0])
def test_encoding_is_to_the_nearest_and_ties_go_to_the_even_byte(top):
    """Against a search over all numbers: every number, every middle between two, and either side of both."""
    m = kvq.NUMBER[:127]
    mid = (m[1:] + m[:-1]) / 2
    x = np.concatenate([m, mid, np.nextafter(mid, 0), np.nextafter(mid, 500), [460.0, 1e30, 2.0 ** -10, 2.0 ** -11]])
    x = np.concatenate([x, -x])
    got = kvq.encode(x, top)
    a = np.minimum(np.abs(x), top)
    d = np.abs(a[:, None] - m[None, :])
    near = d == d.min(1, keepdims=True)
    for i in range(len(x)):
        c = np.flatnonzero(near[i])
        want = c[0] if len(c) == 1 else [b for b in c if b % 2 == 0][0]
        assert got[i] & 0x7F == want and (got[i] >> 7) == np.signbit(x[i])
    assert kvq.encode(np.array([np.nan, np.inf, -np.inf])).tolist() == [0x7F] * 3


@pytest.mark.parametrize("D", [64, 128])
def test_layout_places_every_element_once(D):
    c = kvq.Cache(1, 1, D)
    for p in c.places:
        assert sorted(p.reshape(-1).tolist()) == list(range(16 * D))


def bf16(rng, shape, lo=-6, hi=6):
    x = rng.standard_normal(shape, np.float32) * np.exp2(rng.integers(lo, hi, shape[:2] + (1,))).astype(np.float32)
    u = x.view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def test_scale_is_the_smallest_that_holds_the_block():
    rng = np.random.default_rng(0)
    c = kvq.Cache(4, 2, 64)
    k, v = bf16(rng, (16, 2, 64)), bf16(rng, (16, 2, 64))
    c.append([0, 16], [0], np.array([[2]]), k, v)
    for x, new in enumerate((k, v)):
        amax = np.abs(kvq.widen(new, "bf16")).max((0, 2))
        scale = 2.0 ** (c.scales[2, :, x].astype(float) - 127)
        assert np.all(amax <= 448 * scale) and np.all(amax > 448 * scale / 2)
    kk, vv = c.read([2], 16)
    for got, new in ((kk, k), (vv, v)):
        want = kvq.widen(new, "bf16")
        step = np.maximum(np.abs(want) * 2.0 ** -4, 2.0 ** -10 * np.exp2(c.scales[2].max() - 127.0))
        assert np.all(np.abs(got - want) <= step)  # half a step: 2^-4 relative, or half of the smallest number
    assert (c.k[[0, 1, 3]] == 0x7F).all() and (c.scales[[0, 1, 3]] == 0xFF).all()


def test_rows_one_by_one_differ_from_all_at_once_below_the_normal_numbers_only():
    """A scale that grows shifts exponents: rows appended one by one stand for what they do appended at once, but for numbers that round
    twice, below 2^-6 of the scale."""
    rng = np.random.default_rng(1)
    k, v = bf16(rng, (37, 2, 64)), bf16(rng, (37, 2, 64))
    table = np.array([[3, 0, 1]])
    a, b = kvq.Cache(4, 2, 64), kvq.Cache(4, 2, 64)
    a.append([0, 37], [0], table, k, v)
    for i in range(37):
        b.append([0, 1], [i], table, k[i:i + 1], v[i:i + 1])
    assert np.array_equal(a.scales, b.scales)
    for x, y in zip(a.tensors(), b.tensors()):
        x, y = kvq.NUMBER[x[table[0]]], kvq.NUMBER[y[table[0]]]
        same = (x == y) | np.isnan(x)
        assert np.all(np.abs(x[~same]) < 2.0 ** -6) and np.all(np.abs(x[~same] - y[~same]) <= 2.0 ** -9) and 0 < (~same).mean() < 0.05


def test_what_was_read_appends_to_the_same_numbers():
    rng = np.random.default_rng(2)
    for dtype in ("bf16", "fp16"):
        a, b = kvq.Cache(6, 2, 64, dtype), kvq.Cache(6, 2, 64, dtype)
        k, v = (x if dtype == "bf16" else kvq.widen(x, "bf16").astype(np.float16).view(np.uint16) for x in (bf16(rng, (40, 2, 64)), bf16(rng, (40, 2, 64))))
        for i in range(40):
            a.append([0, 1], [i], np.array([[5, 1, 0]]), k[i:i + 1], v[i:i + 1])
        kk, vv = a.read([5, 1, 0], 40)
        b.append([0, 40], [0], np.array([[2, 3, 4]]), kvq.narrow(kk, dtype), kvq.narrow(vv, dtype))
        for x, y in zip((kk, vv), b.read([2, 3, 4], 40)):
            assert np.array_equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_extreme_rows_stay_exact_and_finite(dtype):
    """The largest, the smallest and special numbers of either type: what the cache stands for is a number of the type."""
    u = np.arange(65536, dtype=np.uint16).reshape(512, 2, 64)
    c = kvq.Cache(32, 2, 64, dtype)
    c.append([0, 512], [0], np.arange(32)[None, :], u, u)
    k, v = c.read(np.arange(32), 512)
    finite = np.isfinite(kvq.widen(u, dtype))
    assert np.array_equal(np.isfinite(k), finite) and np.array_equal(np.isfinite(v), finite) and np.array_equal(np.isnan(k), ~finite)
    kvq.narrow(np.where(finite, k, 0.0), dtype)  # (asserts that nothing is rounded)


class _Kvq:
    """The binding, with plans for caches in 8 bits in the place of the others."""

    def __init__(self, tc):
        self._tc = tc

    def __getattr__(self, name):
        return getattr(self._tc, name)

    def make_pool(self, *a, **kw):
        return self._tc.make_kvq_pool(*a, **kw)


@pytest.mark.parametrize("idx", [0, 1, 2, 3, 4])
def test_work_lists_of_the_configurations(tc, idx):
    sp = W.config_spec(idx)
    table, _, nb = W.make_tables(sp, np.random.default_rng(3))
    info = abi.check_work_list(_Kvq(tc), sp, table, nb)
    assert idx == 3 or info.block_threads == 512  # beside a chunk: the form that has a kernel for such a cache


@pytest.mark.parametrize("seed", range(40))
def test_work_lists_of_random_batches(tc, seed):
    rng = np.random.default_rng(9000 + seed)
    Hkv, G = int(rng.choice([1, 2, 4, 8, 32])), int(rng.choice([1, 2, 3, 5, 8, 16]))
    n_pf, n_dec = int(rng.integers(0, 4)), int(rng.integers(0, 60))
    q_len = [int(rng.integers(2, 900)) for _ in range(n_pf)] + [1] * max(n_dec, n_pf == 0)
    short = seed % 2
    ctx = [int(rng.integers(0, 60 if short else 6000)) for _ in q_len]
    sp = W.custom_spec(f"kvq{seed}", Hkv * G, Hkv, int(rng.choice([64, 128])), q_len, ctx)
    table, _, nb = W.make_tables(sp, rng)
    info = abi.check_work_list(_Kvq(tc), sp, table, nb)
    assert n_pf == 0 or info.block_threads == 512


def _plan(tc, kvq_pool=True, Hq=8, Hkv=2, D=128, q_len=(5, 1), ctx=(3, 40), nb=32, **kw):
    table, _, _ = W.make_tables(W.custom_spec("x", Hq, Hkv, D, q_len, ctx, num_blocks=nb), np.random.default_rng(0))
    qs = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    pool = (tc.make_kvq_pool if kvq_pool else tc.make_pool)(Hq, Hkv, D, nb, **kw)
    return tc.Plan(pool, qs, np.asarray(ctx, np.int32), table, host_only=True)


def _status(tc, fn, *a, **kw):
    with pytest.raises(tc.TcError) as e:
        fn(*a, **kw)
    assert tc.last_error() != ""
    return e.value.status


A = 4096  # an aligned address: nothing reads it, every call below ends at a check


def _pool(tc, Hq=8, Hkv=2, D=128, nb=32, k_pool=A, v_pool=A, scales=A, **kw):
    return tc.make_kvq_pool(Hq, Hkv, D, nb, k_pool, v_pool, scales, **kw)


def _calls(tc, p, pool, rows=A, q=A, out=A, scale=0.1, ws=A, ws_bytes=1 << 30):
    return {"append": lambda: tc.tc_kvq_append(p, pool, rows, rows),
            "read": lambda: tc.tc_kvq_read(p, pool, 0, out, out),
            "attention": lambda: tc.tc_kvq_mixed_attention(p, pool, q, out, scale, ws, ws_bytes),
            "step": lambda: tc.tc_kvq_mixed_attention_append(p, pool, q, rows, rows, out, scale, ws, ws_bytes)}


def test_pool_refusals(tc):
    p = _plan(tc)
    bad = [(dict(scales=None), tc.TC_ERR_NULL), (dict(k_pool=None), tc.TC_ERR_NULL), (dict(v_pool=None), tc.TC_ERR_NULL),
           (dict(k_pool=A + 8), tc.TC_ERR_ARG), (dict(v_pool=A + 1), tc.TC_ERR_ARG), (dict(scales=A + 1), tc.TC_ERR_ARG),
           (dict(Hq=4), tc.TC_ERR_SHAPE), (dict(D=64), tc.TC_ERR_SHAPE), (dict(nb=33), tc.TC_ERR_SHAPE), (dict(dtype=tc.TC_FP16), tc.TC_ERR_SHAPE)]
    for kw, status in bad:
        for name, call in _calls(tc, p, _pool(tc, **kw)).items():
            assert _status(tc, call) == status, (kw, name)
    for name, call in _calls(tc, p, _pool(tc)).items():  # nothing wrong but that the plan has no device copy
        assert _status(tc, call) == tc.TC_ERR_ARG and "host-only" in tc.last_error(), name
    L, vp = tc.lib(), C.c_void_p
    assert L.tc_kvq_append(None, C.byref(_pool(tc)), vp(A), vp(A), None) == tc.TC_ERR_NULL
    assert L.tc_kvq_append(p.handle, None, vp(A), vp(A), None) == tc.TC_ERR_NULL


def test_argument_refusals(tc):
    p, pool = _plan(tc, q_len=(1, 1), ctx=(30000, 40), nb=2000), _pool(tc, nb=2000)
    assert p.workspace_bytes > 0
    for kw, status, names in [
            (dict(rows=None), tc.TC_ERR_NULL, ("append", "step")), (dict(rows=A + 4), tc.TC_ERR_ARG, ("append", "step")),
            (dict(q=None), tc.TC_ERR_NULL, ("attention", "step")), (dict(q=A + 2), tc.TC_ERR_ARG, ("attention", "step")),
            (dict(out=None), tc.TC_ERR_NULL, ("read", "attention", "step")), (dict(out=A + 8), tc.TC_ERR_ARG, ("read", "attention", "step")),
            (dict(ws=None), tc.TC_ERR_WORKSPACE, ("attention", "step")), (dict(ws_bytes=16), tc.TC_ERR_WORKSPACE, ("attention", "step")),
            (dict(ws=A + 4), tc.TC_ERR_ARG, ("attention", "step"))]:
        for name in names:
            assert _status(tc, _calls(tc, p, pool, **kw)[name]) == status and "host-only" not in tc.last_error(), (kw, name)
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        for name in ("attention", "step"):
            assert _status(tc, _calls(tc, p, pool, scale=scale)[name]) == tc.TC_ERR_ARG and "scale" in tc.last_error()
    for seq in (-2, 2, 1 << 30):
        assert _status(tc, tc.tc_kvq_read, p, pool, seq, A, A) == tc.TC_ERR_ARG and "sequence" in tc.last_error()


def test_plans_and_pools_of_one_kind_are_not_for_the_other(tc):
    q, h = _plan(tc), _plan(tc, kvq_pool=False)
    pool_q, pool_h = _pool(tc), tc.make_pool(8, 2, 128, 32, A, A)
    for name, call in _calls(tc, h, pool_q).items():
        assert _status(tc, call) == tc.TC_ERR_SHAPE, name
    half = tc.tc_kvq_pool(pool_h, A)  # a pool in 16 bits behind the other's struct
    for name, call in _calls(tc, q, half).items():
        assert _status(tc, call) == tc.TC_ERR_SHAPE, name
    for pool in (pool_q.base, pool_h):
        for fn, args in [(tc.tc_kv_append, (A, A)), (tc.tc_mixed_attention, (A, A, 0.1, A, 1 << 30)), (tc.tc_mixed_attention_append, (A, A, A, A, 0.1, A, 1 << 30)),
                         (tc.tc_mixed_attention_static, (A, A, 0.1)), (tc.tc_attention_partials, (A, A, 0.1, A, 1 << 30)), (tc.tc_split_merge, (A, A, 1 << 30)),
                         (tc.tc_kv_gather, (0, A, A)), (tc.tc_kv_export, (0, [A], [A], A)), (tc.tc_kv_import, (0, [A], [A], A))]:
            assert _status(tc, fn, q, pool, *args) == tc.TC_ERR_SHAPE, fn.__name__
    assert tc.tc_kv_transfer_bytes(q, 0, 1) == 0


def test_dtypes_that_are_none(tc):
    for dtype in (0, 3, 4, -1, 32 | tc.TC_BF16, -16):
        with pytest.raises(tc.TcError) as e:
            _plan(tc, kvq_pool=False, dtype=dtype)
        assert e.value.status == tc.TC_ERR_SHAPE
        if dtype >= 0:
            assert _status(tc, _plan, tc, dtype=dtype) == tc.TC_ERR_SHAPE


def test_empty_batch_and_too_many_tokens(tc):
    pool = _pool(tc)
    p = tc.Plan(pool, np.zeros(1, np.int32), np.zeros(0, np.int32), np.zeros((0, 1), np.int32), host_only=True)
    tc.tc_kvq_append(p, pool, None, None)
    tc.tc_kvq_mixed_attention(p, pool, None, None, 0.1)
    tc.tc_kvq_mixed_attention_append(p, pool, None, None, None, None, 0.1)
    tc.tc_kvq_read(p, pool, -1, None, None)
    assert _status(tc, tc.tc_kvq_read, p, pool, 0, A, A) == tc.TC_ERR_ARG
    # sequences that share their blocks: 2^31 tokens in all are too many rows for one read
    n = 1 << 21
    table = np.zeros((1 << 10, n // 16), np.int32)
    big = tc.Plan(pool, np.arange((1 << 10) + 1, dtype=np.int32), np.full(1 << 10, n - 1, np.int32), table, host_only=True)
    assert _status(tc, tc.tc_kvq_read, big, pool, -1, A, A) == tc.TC_ERR_ARG and "2^31" in tc.last_error()
    assert _status(tc, tc.tc_kvq_read, big, pool, 5, A, A) == tc.TC_ERR_ARG and "host-only" in tc.last_error()


def test_two_sequences_that_append_to_the_same_block_are_refused(tc):
    """Attention over what is there, and reading it, are not: both may end in a block that they share."""
    pool = _pool(tc)
    for q_len, ctx, rows in [((1, 1), (20, 25), ((3, 7), (9, 7))), ((40, 1), (0, 3), ((1, 2, 3), (2, 0, 0))), ((1, 1, 1), (0, 16, 31), ((5, 0), (6, 4), (6, 5))),
                             ((17,), (0,), ((4, 4),))]:
        table = np.zeros((len(rows), 3), np.int32)
        for s, r in enumerate(rows):
            table[s, :len(r)] = r
        p = tc.Plan(pool, np.concatenate([[0], np.cumsum(q_len)]), np.array(ctx), table, host_only=True)
        calls = _calls(tc, p, pool)
        for name in ("append", "step"):
            assert _status(tc, calls[name]) == tc.TC_ERR_BLOCK, (q_len, name)
        for name in ("read", "attention"):
            assert _status(tc, calls[name]) == tc.TC_ERR_ARG and "host-only" in tc.last_error(), (q_len, name)
    # the shared blocks of a common prompt get no rows
    p = tc.Plan(pool, np.array([0, 1, 3]), np.array([35, 34]), np.array([[1, 2, 3], [1, 2, 4]]), host_only=True)
    for name, call in _calls(tc, p, pool).items():
        assert _status(tc, call) == tc.TC_ERR_ARG and "host-only" in tc.last_error(), name
