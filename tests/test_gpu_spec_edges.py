"""Calls of a speculative step at the edges of what their documentation allows."""
import numpy as np
import pytest

import paper_2507_17769_b200 as ps
from paper_2507_17769_b200 import binding as B
from spec_util import Cache, tree_masks

pytestmark = pytest.mark.gpu


def status_of(f):
    with pytest.raises(ps.PsError) as e:
        f()
    return e.value


@pytest.mark.parametrize("heads,fp8", [((8, 2, 128), False), ((8, 8, 64), False), ((8, 2, 128), True)])
@pytest.mark.parametrize("entry", [-1, -2, -3, -8, -(2 ** 31), 2 ** 31 - 1])
def test_every_page_outside_the_pool_is_reported(heads, fp8, entry):
    """... inside a sequence; entries behind its end are not looked at."""
    import torch

    prior, nodes = np.array([100, 30], dtype=np.int32), np.array([5, 2], dtype=np.int32)
    c = Cache(*heads, prior + nodes, seed=51, fp8=fp8).fill()
    mask, _ = tree_masks(nodes, 1, np.random.default_rng(1))
    q = c.normal(7, heads[0], heads[2])
    want = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    for page in (0, 3, 6):  # (the last holds drafted tokens)
        table = c.table.clone()
        table[0, page] = entry
        out, lse = c.pa.run_tree(q, table, mask, prior, nodes)
        assert status_of(c.pa.check_pool).status == B.PS_ERR_BOUNDS
        assert torch.equal(out[5:], want[0][5:]) and torch.equal(lse[5:], want[1][5:])
    table = c.table.clone()
    table[0, 7:], table[1, 2:] = entry, entry
    got = c.pa.run_tree(q, table, mask, prior, nodes)
    c.pa.check_pool()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
