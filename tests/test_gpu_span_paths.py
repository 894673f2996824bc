"""The batches of tests/test_span_paths_host.py on the GPU, against the plain form in 64 bits, with the bound of tests/test_gpu_span.py."""
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
