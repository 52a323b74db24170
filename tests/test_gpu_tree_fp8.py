"""Tree attention over the FP8 cache against the definition in 64 bits over the values that the cache stands for
(bounds: spec_util.tree_reference)."""
import numpy as np
import pytest

from spec_util import Cache, check_tree, tree_masks, tree_reference
from test_gpu_tree import run

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (8, 8, 128), (16, 2, 128), (2, 1, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("prior,nodes", [([0], [1]), ([0], [5]), ([700], [8]), ([127, 128, 129], [1, 1, 1]), ([1, 500, 0, 2000], [64, 3, 17, 33])])
def test_small_batches(heads, prior, nodes):
    run(heads, prior, nodes, seed=len(prior) + heads[0], fp8=True)


@pytest.mark.parametrize("heads", HEADS)
def test_trees_of_more_rows_than_a_group(heads):
    run(heads, [300, 40, 1000], [256, 130, 200], seed=3, fp8=True)


def test_ragged_batches():
    rng = np.random.default_rng(7)
    run((32, 8, 128), rng.integers(0, 3000, 40), rng.integers(1, 65, 40), seed=8, q_scale=3.0, fp8=True)
    run((32, 8, 128), rng.integers(0, 300, 100), rng.integers(1, 33, 100), seed=9, fp8=True)


def test_one_long_context_over_all_sms():
    run((4, 1, 128), [60000], [40], seed=9, fp8=True)


def test_rows_that_see_nothing_and_odd_masks():
    rng = np.random.default_rng(4)
    sees = [rng.random((n, n)) < p for n, p in ((1, 0.0), (9, 0.3), (64, 0.02), (70, 0.5), (130, 0.01), (200, 0.9))]
    for s in sees[1:]:
        s[min(3, len(s) - 1)] = False
    nodes = [len(s) for s in sees]
    _, _, _, out, lse = run((8, 2, 128), [0] * len(nodes), nodes, seed=5, sees_all=sees, fp8=True)
    assert float(out[0].abs().max()) == 0 and bool((lse[0] == -np.inf).all())
    run((8, 2, 128), [0, 130, 7, 1000, 120, 400], nodes, seed=6, sees_all=sees, fp8=True)


@pytest.mark.parametrize("where", ["k", "v", "kv"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_a_node_does_not_see_has_no_part(where, value):
    """A NaN is stored as such, an infinity takes its vector's scale with it: they reach the nodes that see them and no other."""
    import torch

    rng = np.random.default_rng(12)
    prior, nodes = np.array([0, 250, 77], dtype=np.int32), np.array([20, 64, 100], dtype=np.int32)
    c = Cache(8, 2, 128, prior + nodes, seed=13, fp8=True)
    bad = ([3], [0, 40, 63], [99])
    for r in range(3):
        for i in bad[r]:
            for name in where:
                getattr(c, name)[r][prior[r] + i, :, 5:7] = value
    c.fill()
    mask, sees = tree_masks(nodes, 2, rng)
    q = c.normal(int(nodes.sum()), 8, 128)
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    t = 0
    for r in range(3):
        n = int(nodes[r])
        touched = torch.from_numpy(sees[r][:, bad[r]].any(1)).cuda()
        assert bool(touched.any()) and (r == 1 or not bool(touched.all()))
        got, got_lse = out[t:t + n], lse[t:t + n]
        assert bool(torch.isfinite(got[~touched]).all()) and bool(torch.isfinite(got_lse[~touched]).all())
        assert not bool(torch.isfinite(got[touched][:, :, 5:7]).any())
        if where == "v":
            assert bool(torch.isfinite(got_lse).all())
        t += n
    if where == "v" and value != value:
        check_tree(out, lse, tree_reference(c, q, prior, sees))


def test_queries_of_any_magnitude():
    """A row of q is brought to the range of the 8-bit operands by a power of two: rows of zeros, of the smallest and of large
    magnitudes, with elements of very different ones."""
    import torch

    prior, nodes = np.array([200], dtype=np.int32), np.array([12], dtype=np.int32)
    c = Cache(4, 2, 128, prior + nodes, seed=31, fp8=True).fill()
    mask, sees = tree_masks(nodes, 1, np.random.default_rng(1))
    q = c.normal(12, 4, 128)
    q[0] = 0
    q[1] *= 2.0 ** -60
    q[2] *= 2.0 ** -130  # subnormal in bf16
    q[3, :, ::2] *= 2.0 ** -12
    q[4, :, 1:] = 0
    q[5] = 1.75
    q[6] = 1.7578125  # just above the last value that E4M3 has below 2
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    check_tree(out, lse, tree_reference(c, q, prior, sees))
    for value in (float("nan"), float("inf")):
        bad = q.clone()
        bad[7, 1, 9] = value
        got, got_lse = c.pa.run_tree(bad, c.table, mask, prior, nodes)
        same = torch.ones(12, 4, dtype=torch.bool, device="cuda")
        same[7, 1] = False
        assert bool(torch.isnan(got[7, 1]).all()) and torch.equal(got[same], out[same]) and torch.equal(got_lse[same], lse[same])


def test_scales_far_apart():
    """Tokens whose K and V are larger and smaller than their neighbours' by orders of magnitude (V's scales within what ps_shape names)."""
    prior, nodes = np.array([300, 40], dtype=np.int32), np.array([30, 64], dtype=np.int32)
    c = Cache(8, 2, 128, prior + nodes, seed=33, fp8=True)
    for r in range(2):
        n = int(c.kv_len[r])
        import torch

        e = torch.randint(-8, 9, (n, 2, 1), generator=c.gen, device="cuda").float()
        c.v[r] = (c.v[r].float() * 2.0 ** e).bfloat16()
        c.k[r] = (c.k[r].float() * 2.0 ** (e / 8)).bfloat16()
    c.fill()
    mask, sees = tree_masks(nodes, 1, np.random.default_rng(2))
    q = c.normal(94, 8, 128)
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    check_tree(out, lse, tree_reference(c, q, prior, sees))


def test_a_step_on_the_fp8_cache_in_a_graph():
    """Append, attention, accepted path and read-back, captured and replayed, give what the calls give."""
    import torch

    prior, nodes = np.array([90, 700], dtype=np.int32), np.array([33, 60], dtype=np.int32)
    c = Cache(32, 8, 128, prior + nodes, seed=22, fp8=True).fill()
    mask, sees = tree_masks(nodes, 1, np.random.default_rng(3))
    qkv = c.normal(93, 48, 128)
    index = torch.tensor([[0, 4, 7], [2, 3, 50]], dtype=torch.int32, device="cuda")
    count = torch.tensor([3, 3], dtype=torch.int32, device="cuda")

    def step():
        q = c.pa.write_rope(qkv[:, :32], qkv[:, 32:40], qkv[:, 40:], c.table, prior, nodes, None)
        out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
        c.pa.accept(c.table, prior, nodes, index, count)
        return (out, lse) + c.pa.read(c.table, prior, nodes)

    want = step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for _ in range(2):
        for x in got:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    c.pa.check_pool()


def test_waits_that_run_out():
    import torch

    import paper_2507_17769_b200 as ps

    c, q, mask, out, lse = run((32, 8, 128), [700, 3000], [60, 33], seed=23, fp8=True)
    ps.ps_kv_set_wait_limit(c.pa.kv, 0)
    c.pa.run_tree(q, c.table, mask, [700, 3000], [60, 33])
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_TIMEOUT
    ps.ps_kv_set_wait_limit(c.pa.kv, 2_000_000_000)
    again = c.pa.run_tree(q, c.table, mask, [700, 3000], [60, 33])
    c.pa.check_pool()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("power", [0, -6, -9, -12, -13])
def test_small_values(power):
    """V's scales down to the least that ps_shape names.

    Beside the weights' rounding (2^-11 of each, and 2^-25 at the least of n weights of at most their sum), a value is code * scale / 2 in f16: the
    scale's 8 bits are exact where scale * 2^7 is normal (else off by 2^-25 of at least 2^-15: 2^-10), the product is off by 2^-12 of itself
    and 2^-25 at the least, 2^-24 of a value."""
    prior, nodes = np.array([0, 0, 300, 40], dtype=np.int32), np.array([1, 2, 30, 64], dtype=np.int32)
    c = Cache(8, 2, 128, prior + nodes, seed=34, fp8=True)
    for r in range(4):
        c.v[r] = (c.v[r].float() * 2.0 ** power).bfloat16()
    c.fill()
    mask, sees = tree_masks(nodes, 1, np.random.default_rng(2))
    q = c.normal(int(nodes.sum()), 8, 128)
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    want, want_lse, bound, lse_bound = tree_reference(c, q, prior, sees)
    largest = max(float(v.abs().max()) for v in c.v)
    rest = bound - 2.0 ** -13 + (2.0 ** -12 + (2.0 ** -10 if power < -12 else 0) + int((prior + nodes).max()) * 2.0 ** -25) * largest + 2.0 ** -24
    check_tree(out, lse, (want, want_lse, rest, lse_bound))


def test_values_out_of_range_that_a_node_does_not_see():
    """A drafted token's values beyond f16's range are finite, and have no part in the results of nodes that do not see it."""
    import torch

    prior, nodes = np.array([100], dtype=np.int32), np.array([20], dtype=np.int32)
    c = Cache(8, 2, 128, prior + nodes, seed=35, fp8=True)
    bad = [4, 11]
    for i, v in zip(bad, (3e5, -2e38)):
        c.v[0][100 + i, :, 5:7] = v
    c.fill()
    rng = np.random.default_rng(3)
    mask, sees = tree_masks(nodes, 1, rng)
    q = c.normal(20, 8, 128)
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    touched = torch.from_numpy(sees[0][:, bad].any(1)).cuda()
    assert bool(touched.any()) and not bool(touched.all())
    assert bool(torch.isfinite(out[~touched]).all())
    c.v[0][[104, 111]] = 0  # what is left is seen by the other rows
    want, want_lse, bound, lse_bound = tree_reference(c, q, prior, sees)
    rows = torch.nonzero(~touched).flatten()
    check_tree(out[rows], lse[rows], (want[rows], want_lse[rows], bound[rows], lse_bound[rows]))
