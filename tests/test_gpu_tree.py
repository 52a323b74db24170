"""Attention for trees of drafted tokens against the definition in 64 bits (bounds: spec_util.tree_reference)."""
import numpy as np
import pytest

from spec_util import Cache, check_tree, pack, tree_masks, tree_reference

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (8, 8, 128), (16, 2, 128), (2, 1, 128), (8, 8, 64), (4, 2, 64), (32, 4, 64)]


def run(heads, prior, nodes, seed=0, words=None, q_scale=1.0, sees_all=None):
    import torch

    rng = np.random.default_rng(seed)
    prior, nodes = np.asarray(prior, dtype=np.int32), np.asarray(nodes, dtype=np.int32)
    words = words or (int(nodes.max()) + 63) // 64
    cache = Cache(*heads, prior + nodes, seed=seed).fill()
    mask, sees = tree_masks(nodes, words, rng)
    if sees_all is not None:
        sees, mask = sees_all, torch.from_numpy(np.concatenate([pack(s, words) for s in sees_all])).cuda()
    q = cache.normal(int(nodes.sum()), heads[0], heads[2], scale=q_scale)
    out, lse = cache.pa.run_tree(q, cache.table, mask, prior, nodes)
    cache.pa.check_pool()
    check_tree(out, lse, tree_reference(cache, q, prior, sees))
    return cache, q, mask, out, lse


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("prior,nodes", [([0], [1]), ([0], [5]), ([700], [8]), ([127, 128, 129], [1, 1, 1]), ([1, 500, 0, 2000], [64, 3, 17, 33])])
def test_small_batches(heads, prior, nodes):
    run(heads, prior, nodes, seed=len(prior) + heads[0])


@pytest.mark.parametrize("heads", HEADS)
def test_trees_of_more_rows_than_a_group(heads):
    run(heads, [300, 40, 1000], [256, 130, 200], seed=3)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 64)])
def test_ragged_batch(heads):
    rng = np.random.default_rng(7)
    run(heads, rng.integers(0, 3000, 40), rng.integers(1, 65, 40), seed=8, q_scale=3.0)


@pytest.mark.parametrize("heads", [(4, 1, 128), (2, 2, 64)])
def test_one_long_context_over_all_sms(heads):
    run(heads, [60000], [40], seed=9)
