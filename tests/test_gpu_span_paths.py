"""The batches of tests/test_span_paths_host.py on the GPU, against the plain form in 64 bits, with the bound of tests/test_gpu_span.py; and what is not finite in tokens that some rows of a sweep
attend over and others do not, where the sweep is cut, one of several of its workgroup, or of eight waves."""
import numpy as np
import pytest

from test_gpu_span import Case, Device, check, tc  # noqa: F401  (the fixture)
from test_span_paths_host import BATCHES, takes_its_path

pytestmark = pytest.mark.gpu


def device(tc, name, dtype="bf16"):  # noqa: F811
    Hq, Hkv, D, q_len, ctx, over, _, _ = BATCHES[name]
    shared = isinstance(over, list)
    d = Device(tc, Case(Hq, Hkv, D, q_len, ctx, dtype, over if shared else None))
    mask = (None, 0) if shared else over
    d.set(*mask)
    takes_its_path(d.plan.span_info(shared), d.plan.span_items(0, shared), name)
    return d, mask


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", list(BATCHES))
def test_outputs(tc, name, dtype):  # noqa: F811
    """Against the plain form, and once more over a workspace and outputs of other contents: the same bits."""
    d, mask = device(tc, name, dtype)
    check(d, *mask, some=3)
    first = d.outputs()
    for _ in range(2):
        d.out.fill_(-1)
        d.workspace.fill_(0x7F)
        d.run()
        assert np.array_equal(d.outputs(), first)


# name: (sequence, token) pairs: at a window's end, its beginning, a sink, the token behind the sinks (no row's), a row's own, one of all rows; of shared tokens in their first and last block, and own ones
TOKENS = {
    "window chained 8": [(0, 1), (0, 2), (0, 3), (0, 202), (0, 450), (0, 600), (0, 2000), (0, 4501), (0, 4700), (0, 4900), (1, 0), (1, 33), (1, 299), (3, 5), (7, 2500)],
    "window chained 4": [(0, 0), (0, 1), (0, 500), (0, 777), (0, 1502)],
    "window mix 8": [(0, 1), (0, 302), (0, 310), (0, 316), (0, 4500), (0, 4514), (5, 400), (17, 1)],
    "shared chained 8": [(0, 0), (0, 2399), (0, 2400), (3, 2405), (3, 2421), (3, 2425), (11, 2477), (11, 2485)],
    "shared chained 4, 64": [(0, 1111), (0, 2399), (2, 2400), (2, 2414), (2, 2418)],
    "shared mix 8": [(0, 7), (0, 159), (0, 2208), (0, 2215), (7, 160), (7, 202), (20, 290)],
    "alone": [(0, 0), (0, 7439), (0, 7440), (0, 7472)],
}


@pytest.mark.parametrize("name", list(TOKENS))
def test_what_is_not_attended_over_may_be_anything(tc, name):  # noqa: F811
    """NaN in K, NaN and infinities of either sign in V, of one token: the rows that attend over it get them, the others keep every bit."""
    d, mask = device(tc, name)
    c, groups = d.c, d.c.groups
    d.run()
    clean = d.outputs()
    pos = np.concatenate([np.arange(a, a + n) for n, a in zip(c.q_len, c.ctx)])
    seq = np.repeat(np.arange(len(c.ctx)), c.q_len)
    window, sinks = (1 << 40, 0) if groups else mask
    prefix = groups[0][1] if groups else 0
    pools = d.k_pool.clone(), d.v_pool.clone()
    for s, j in TOKENS[name]:
        for which, bits in (("k", 0x7FC0), ("v", 0x7FC0), ("v", 0x7F80), ("v", 0xFF80)):
            d.poke(s, j, **{which: bits})
            d.out.fill_(-1)
            d.run()
            got, values = d.outputs(), d.values()
            sees = ((seq == s) | (j < prefix)) & (j <= pos) & ((pos - j < window) | (j < sinks))
            assert np.array_equal(got[~sees], clean[~sees]), (s, j, which)
            if bits == 0x7FC0:
                assert np.isnan(values[sees]).all(), (s, j, which)
            else:
                assert (values[sees] == (np.inf if bits == 0x7F80 else -np.inf)).all(), (s, j, which)
            d.k_pool.copy_(pools[0])
            d.v_pool.copy_(pools[1])
