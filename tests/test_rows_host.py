"""What tc_qk_norm_rotate and tc_qk_norm_rotate_append refuse (no GPU needed), and the plain form that the GPU tests compare with."""
import numpy as np
import pytest

import test_abi_host as abi
from oracle.rows import norm_rotate
from test_abi_host import tc  # noqa: F401  (the fixture)


def test_plain_form_against_one_pair_at_a_time():
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((3, 2, 8)), rng.standard_normal(8)
    freq, pos = np.array([1.0, 0.25]), [0, 3, 100]
    for adjacent in (False, True):
        got, _ = norm_rotate(x, w, 1e-3, freq, 4, adjacent, pos)
        for t in range(3):
            for h in range(2):
                y = x[t, h] / np.sqrt(np.mean(x[t, h] ** 2) + 1e-3) * w
                want = y.copy()
                for i in range(2):
                    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + 2)
                    c, s = np.cos(pos[t] * freq[i]), np.sin(pos[t] * freq[i])
                    want[a], want[b] = y[a] * c - y[b] * s, y[b] * c + y[a] * s
                assert np.allclose(got[t, h], want, rtol=1e-13, atol=1e-13)


def rows_of(tc, **change):  # noqa: F811
    """Good arguments (addresses that are never used: a host-only plan is refused last), some of them changed."""
    r = tc.tc_qkv_rows(4096, 8192, 16384, 12 * 128, 12 * 128, 12 * 128, 65536, 69632, 1e-6, 128, 73728, 0, None)
    for k, v in change.items():
        setattr(r, k, v)
    return r


REFUSALS = [
    ("TC_ERR_SHAPE", dict(rotary_dim=-8)), ("TC_ERR_SHAPE", dict(rotary_dim=136)), ("TC_ERR_SHAPE", dict(rotary_dim=4)),
    ("TC_ERR_NULL", dict(q=None)), ("TC_ERR_NULL", dict(k=None)), ("TC_ERR_NULL", dict(freq=None)),
    ("TC_ERR_ARG", dict(q=4098)), ("TC_ERR_ARG", dict(k=8200)), ("TC_ERR_ARG", dict(q_weight=65544)), ("TC_ERR_ARG", dict(k_weight=69634)),
    ("TC_ERR_ARG", dict(freq=73732)), ("TC_ERR_ARG", dict(positions=4098)),
    ("TC_ERR_ARG", dict(q_stride=8 * 128 - 8)), ("TC_ERR_ARG", dict(k_stride=2 * 128 - 8)), ("TC_ERR_ARG", dict(q_stride=-2048)),
    ("TC_ERR_ARG", dict(q_stride=8 * 128 + 4)), ("TC_ERR_ARG", dict(k_stride=2 * 128 + 1)),
    ("TC_ERR_ARG", dict(eps=0.0)), ("TC_ERR_ARG", dict(eps=float("nan"))), ("TC_ERR_ARG", dict(eps=float("inf"))), ("TC_ERR_ARG", dict(eps=-1.0)),
]
REFUSALS_V = [("TC_ERR_NULL", dict(v=None)), ("TC_ERR_ARG", dict(v=16392)), ("TC_ERR_ARG", dict(v_stride=2 * 128 - 8)), ("TC_ERR_ARG", dict(v_stride=2 * 128 + 12))]


@pytest.mark.parametrize("want, change", REFUSALS + REFUSALS_V)
def test_refusals(tc, want, change):  # noqa: F811
    plan = abi._plan(tc)
    pool = tc.make_pool(8, 2, 128, 32, 1 << 20, 1 << 21)
    want = getattr(tc, want)
    if (want, change) not in [(getattr(tc, w), c) for w, c in REFUSALS_V]:
        assert abi._status(tc, lambda: tc.tc_qk_norm_rotate(plan, rows_of(tc, **change), 1 << 22, 1 << 23)) == want
        assert "host-only" not in tc.last_error()
    assert abi._status(tc, lambda: tc.tc_qk_norm_rotate_append(plan, pool, rows_of(tc, **change), 1 << 22)) == want
    assert "host-only" not in tc.last_error()


def test_refusals_of_outputs_pools_and_plans(tc):  # noqa: F811
    plan, rows = abi._plan(tc), rows_of(tc)
    pool = tc.make_pool(8, 2, 128, 32, 1 << 20, 1 << 21)
    st = lambda fn: abi._status(tc, fn)  # noqa: E731
    assert st(lambda: tc.tc_qk_norm_rotate(plan, rows, None, 1 << 23)) == tc.TC_ERR_NULL
    assert st(lambda: tc.tc_qk_norm_rotate(plan, rows, 1 << 22, None)) == tc.TC_ERR_NULL
    assert st(lambda: tc.tc_qk_norm_rotate(plan, rows, (1 << 22) + 8, 1 << 23)) == tc.TC_ERR_ARG
    assert st(lambda: tc.tc_qk_norm_rotate(plan, rows, 1 << 22, (1 << 23) + 2)) == tc.TC_ERR_ARG
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, pool, rows, None)) == tc.TC_ERR_NULL
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, pool, rows, (1 << 22) + 8)) == tc.TC_ERR_ARG
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, tc.make_pool(8, 2, 128, 32, None, 1 << 21), rows, 1 << 22)) == tc.TC_ERR_NULL
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, tc.make_pool(8, 2, 128, 32, (1 << 20) + 8, 1 << 21), rows, 1 << 22)) == tc.TC_ERR_ARG
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, tc.make_pool(8, 2, 64, 32, 1 << 20, 1 << 21), rows, 1 << 22)) == tc.TC_ERR_SHAPE
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, tc.make_kvq_pool(8, 2, 128, 32, 1 << 20, 1 << 21, 1 << 22).base, rows, 1 << 22)) == tc.TC_ERR_SHAPE
    # every argument good: a plan without a device copy is what is left to refuse
    assert st(lambda: tc.tc_qk_norm_rotate(plan, rows, 1 << 22, 1 << 23)) == tc.TC_ERR_ARG
    assert st(lambda: tc.tc_qk_norm_rotate_append(plan, pool, rows, 1 << 22)) == tc.TC_ERR_ARG
    # without weights eps is not looked at, without rotation freq is not
    assert "host-only" in _text(tc, lambda: tc.tc_qk_norm_rotate(plan, rows_of(tc, q_weight=None, k_weight=None, eps=0.0, rotary_dim=0, freq=None), 1 << 22, 1 << 23))


def _text(tc, fn):  # noqa: F811
    with pytest.raises(tc.TcError) as e:
        fn()
    return str(e.value)


def test_an_empty_batch_is_a_no_op(tc):  # noqa: F811
    pool = tc.make_pool(8, 2, 128, 32, 1 << 20, 1 << 21)
    plan = tc.Plan(pool, np.zeros(1, np.int32), np.zeros(0, np.int32), np.zeros((0, 1), np.int32), host_only=True)
    tc.tc_qk_norm_rotate(plan, tc.tc_qkv_rows(), None, None)
    tc.tc_qk_norm_rotate_append(plan, pool, tc.tc_qkv_rows(), None)


def test_rows_whose_heads_are_not_adjacent_are_refused(tc):  # noqa: F811
    import torch
    x = torch.zeros(4, 8, 2, 64)
    with pytest.raises(ValueError):
        tc.make_qkv_rows(x[:, :, 0], x[:, :, 1])


def test_strides_of_tensors(tc):  # noqa: F811
    """A single token's stride says nothing; rows of two dimensions; freq and positions of another width."""
    import torch
    x = torch.zeros(1, 8, 64, dtype=torch.bfloat16)
    rows = tc.make_qkv_rows(x.expand(1, 8, 64).as_strided((1, 8, 64), (7, 64, 1)), torch.zeros(3, 1024, dtype=torch.bfloat16)[:, 512:])
    assert rows.q_stride == 512 and rows.k_stride == 1024
    with pytest.raises(ValueError):
        tc.make_qkv_rows(x, torch.zeros(1024, 3, dtype=torch.bfloat16).t())
    with pytest.raises(ValueError):
        tc.make_qkv_rows(x, x, freq=torch.zeros(32))
    with pytest.raises(ValueError):
        tc.make_qkv_rows(x, x, positions=torch.zeros(1, dtype=torch.int64))


def test_rows_that_are_not_packed_are_not_their_own_output(tc):  # noqa: F811
    plan = abi._plan(tc)
    pool = tc.make_pool(8, 2, 128, 32, 1 << 20, 1 << 21)
    wide = rows_of(tc, q=1 << 22, q_stride=8 * 128 + 8)
    assert abi._status(tc, lambda: tc.tc_qk_norm_rotate(plan, wide, 1 << 22, 1 << 23)) == tc.TC_ERR_ARG and "packed" in tc.last_error()
    assert abi._status(tc, lambda: tc.tc_qk_norm_rotate_append(plan, pool, wide, 1 << 22)) == tc.TC_ERR_ARG and "packed" in tc.last_error()
    assert abi._status(tc, lambda: tc.tc_qk_norm_rotate(plan, rows_of(tc, k=1 << 23, k_stride=2 * 128 + 8), 1 << 22, 1 << 23)) == tc.TC_ERR_ARG and "packed" in tc.last_error()


def test_frequencies_and_positions_that_do_not_fit_are_refused(tc):  # noqa: F811
    """The kernel reads rotary_dim / 2 adjacent frequencies, and adjacent positions: fewer of them, others in between or another type would be read behind the end or wrongly."""
    import torch
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    freq, positions = torch.ones(32, dtype=torch.float64), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(freq=freq, rotary_dim=72), dict(freq=freq[:3], rotary_dim=8), dict(freq=freq[::2]), dict(freq=freq[:1].expand(8)), dict(freq=torch.ones(32, dtype=torch.int64)),
               dict(positions=positions.float()), dict(positions=torch.zeros(6, dtype=torch.int32)[::2]), dict(positions=positions[:1].expand(3))):
        with pytest.raises(ValueError):
            tc.make_qkv_rows(x, x, **kw)
    rows = tc.make_qkv_rows(x, x, freq=freq, rotary_dim=16, positions=positions)  # more of them are no harm
    assert rows.rotary_dim == 16 and rows.freq == freq.data_ptr() and rows.positions == positions.data_ptr()
    assert tc.make_qkv_rows(x, x, freq=freq).rotary_dim == 64 and tc.make_qkv_rows(x, x, freq=1 << 20, rotary_dim=128).rotary_dim == 128


def test_rows_and_weights_of_another_type_are_refused(tc):  # noqa: F811
    """Weights in 32 bits, as checkpoints often hold them, would be read as patterns of 16; so would weights in the other 16-bit type, and rows of either kind."""
    import torch
    x, w = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    make = tc.make_qkv_rows
    for q, k, v, kw in ((x, x, None, dict(q_weight=w.float())), (x, x, None, dict(k_weight=w.double())), (x, x, None, dict(k_weight=w.half())), (x, x.half(), None, {}), (x, x, x.half(), {}),
                        (x.float(), x.float(), None, {}), (x, x.float(), None, {}), (x, x, x.float(), {}), (1 << 20, x.float(), None, dict(q_stride=128)),
                        (1 << 20, x, None, dict(q_stride=128, k_weight=w.half())), (x.view(torch.int16), x.view(torch.int16), None, dict(q_weight=w, k_weight=w.half())), (1 << 20, 1 << 21, None, dict(q_stride=128, k_stride=128, q_weight=w.float()))):
        with pytest.raises(ValueError):
            make(q, k, v, **kw)
    for kw in (dict(q_weight=w[:32]), dict(k_weight=torch.ones(128, dtype=torch.bfloat16)), dict(q_weight=torch.ones(128, dtype=torch.bfloat16)[::2]), dict(k_weight=w[:1].expand(64))):
        with pytest.raises(ValueError):  # a weight for each element of a head, one after the other
            make(x, x, **kw)
    bits = x.view(torch.int16)  # patterns, whose type nothing says
    for q, k, v, a, b in ((x, x, x, w, w), (bits, bits, bits, w, w), (x, bits, None, w.view(torch.int16), None), (x.view(3, 128), x, x, w, w)):
        rows = make(q, k, v, a, b)
        assert (rows.q, rows.q_weight, rows.k_weight) == (q.data_ptr(), a.data_ptr(), None if b is None else b.data_ptr())


def test_rows_hold_their_tensors(tc):  # noqa: F811
    """What a call is given may be made in the call: it lives as long as the rows do."""
    import gc
    import weakref

    import torch
    for wide in (False, True):  # the usual call and any other
        x = [torch.zeros(3, 2, 64, dtype=torch.bfloat16) for _ in range(3)]
        x = [t.view(3, 128) for t in x] if wide else x
        more = [torch.ones(64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16), torch.ones(32, dtype=torch.float64), torch.zeros(3, dtype=torch.int32)]
        refs = [weakref.ref(t) for t in x + more]
        rows = tc.make_qkv_rows(*x, more[0], more[1], freq=more[2], positions=more[3])
        del x, more
        gc.collect()
        assert all(r() is not None for r in refs)
        assert rows.positions == refs[-1]().data_ptr()
        del rows
        gc.collect()
        assert all(r() is None for r in refs)
