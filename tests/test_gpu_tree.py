"""Attention for trees of drafted tokens against the definition in 64 bits (bounds: spec_util.tree_reference)."""
import numpy as np
import pytest

from spec_util import Cache, check_tree, pack, tree_masks, tree_reference

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (8, 8, 128), (16, 2, 128), (2, 1, 128), (8, 8, 64), (4, 2, 64), (32, 4, 64)]


def run(heads, prior, nodes, seed=0, words=None, q_scale=1.0, sees_all=None, fp8=False):
    import torch

    rng = np.random.default_rng(seed)
    prior, nodes = np.asarray(prior, dtype=np.int32), np.asarray(nodes, dtype=np.int32)
    words = words or (int(nodes.max()) + 63) // 64
    cache = Cache(*heads, prior + nodes, seed=seed, fp8=fp8).fill()
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


def test_rows_that_see_nothing_and_odd_masks():
    """Without context: a row whose mask leaves nothing gives zeros and -inf; masks need not hold a node's own bit, nor be a tree's."""
    rng = np.random.default_rng(4)
    for heads in ((8, 2, 128), (4, 2, 64)):
        sees = [rng.random((n, n)) < p for n, p in ((1, 0.0), (9, 0.3), (64, 0.02), (70, 0.5), (130, 0.01), (200, 0.9))]
        for s in sees[1:]:
            s[min(3, len(s) - 1)] = False
        nodes = [len(s) for s in sees]
        _, _, _, out, lse = run(heads, [0] * len(nodes), nodes, seed=5, sees_all=sees)
        assert float(out[0].abs().max()) == 0 and bool((lse[0] == -np.inf).all())
        run(heads, [0, 130, 7, 1000, 120, 400], nodes, seed=6, sees_all=sees)


def test_bits_behind_the_last_node_are_not_looked_at():
    import torch

    c, q, mask, out, lse = run((8, 2, 128), [50, 300], [9, 70], seed=11)
    dirty = mask.clone()
    dirty[:9, 0] |= ~((1 << 9) - 1)
    dirty[:9, 1] = -1
    dirty[9:, 1] |= ~((1 << 6) - 1)
    again = c.pa.run_tree(q, c.table, dirty, [50, 300], [9, 70])
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 8, 64), (8, 1, 128)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["k", "v", "kv"])
def test_what_a_node_does_not_see_has_no_part(heads, value, where):
    """Infinities and NaN in K and V of nodes: they reach the nodes that see them and no other."""
    import torch

    rng = np.random.default_rng(12)
    prior, nodes = np.array([0, 250, 77], dtype=np.int32), np.array([20, 64, 100], dtype=np.int32)
    c = Cache(*heads, prior + nodes, seed=13)
    for r, bad in enumerate(([3], [0, 40, 63], [99])):  # (the root: seen by the whole tree; a leaf: by itself)
        for i in bad:
            for name in where:
                x = getattr(c, name)[r]
                x[prior[r] + i, :, 5:7] = value
    c.fill()
    mask, sees = tree_masks(nodes, 2, rng)
    q = c.normal(int(nodes.sum()), heads[0], heads[2])
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    clean = Cache(*heads, prior + nodes, seed=13)
    for r in range(3):
        for name in "kv":
            getattr(clean, name)[r].copy_(torch.nan_to_num(getattr(c, name)[r], 0, 0, 0))
    clean.fill()
    ref, ref_lse = clean.pa.run_tree(q, clean.table, mask, prior, nodes)
    t = 0
    for r, bad in enumerate(([3], [0, 40, 63], [99])):
        n = int(nodes[r])
        touched = torch.from_numpy(sees[r][:, bad].any(1)).cuda()
        rows = slice(t, t + n)
        assert bool(touched.any()) and (r == 1 or not bool(touched.all()))
        # (a row that sees none of them is as without them, up to the order of the maxima: to the bound of two runs)
        a, b = out[rows][~touched].float(), ref[rows][~touched].float()
        assert bool(torch.isfinite(a).all()) and float((a - b).abs().max() if a.numel() else 0) <= 2.0 ** -5
        if where == "v":
            seen = out[rows][touched]
            assert not bool(torch.isfinite(seen[:, :, 5:7]).any())
            other = [e for e in range(heads[2]) if e not in (5, 6)]
            assert bool(torch.isfinite(seen[:, :, other]).all())
            assert bool(torch.isfinite(lse[rows]).all())
            if value == value and r != 1:
                assert bool((seen[:, :, 5:7] == value).all())
        t += n
    if where == "v":
        check_tree(out, lse, tree_reference(c, q, prior, sees))


def test_context_behind_the_sequence_and_other_requests_are_not_read():
    """The pool starts as NaN, and a page's slots behind a sequence's end stay so; a request's rows are its own."""
    import torch

    c, q, mask, out, lse = run((8, 2, 128), [100, 3], [5, 2], seed=14)
    alone, lse_alone = c.pa.run_tree(q[5:], c.table[1:], mask[5:], [3], [2])
    assert float((alone.float() - out[5:].float()).abs().max()) <= 2.0 ** -6 and torch.allclose(lse_alone, lse[5:], atol=1e-4)


def test_given_outputs_no_lse_and_rows_behind_the_last():
    import torch

    c, q, mask, out, lse = run((8, 8, 64), [40, 9], [30, 3], seed=15)
    room, room_lse = torch.full((40, 8, 64), 3.0, device="cuda", dtype=torch.bfloat16), torch.full((40, 8), 3.0, device="cuda")
    got = c.pa.run_tree(q, c.table, mask, [40, 9], [30, 3], out=room[:33], lse=room_lse[:33])
    assert got[0].data_ptr() == room.data_ptr() and torch.equal(room[:33], out) and torch.equal(room_lse[:33], lse)
    assert bool((room[33:] == 3).all()) and bool((room_lse[33:] == 3).all())
    got = c.pa.run_tree(q, c.table, mask, [40, 9], [30, 3], want_lse=False)
    assert got[1] is None and torch.equal(got[0], out)


def test_pages_outside_the_pool_are_reported():
    import torch

    import paper_2507_17769_b200 as ps

    c, q, mask, out, lse = run((8, 2, 128), [100, 30], [5, 2], seed=16)
    table = c.table.clone()
    table[0, 2] = c.num_pages + 9
    got, _ = c.pa.run_tree(q, table, mask, [100, 30], [5, 2])
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_BOUNDS and torch.equal(got[5:], out[5:])
    assert torch.equal(c.pa.run_tree(q, c.table, mask, [100, 30], [5, 2])[0], out)
    c.pa.check_pool()


def test_more_requests_than_a_launch_takes():
    rng = np.random.default_rng(17)
    n = 2700
    run((2, 1, 64), rng.integers(0, 40, n), rng.integers(1, 4, n), seed=18)
    run((2, 1, 64), rng.integers(0, 300, 100), rng.integers(1, 9, 100), seed=19)


def test_results_are_the_same_every_time_and_with_a_dirty_workspace():
    import torch

    import paper_2507_17769_b200 as ps

    c, q, mask, out, lse = run((16, 2, 128), [5000, 900], [40, 64], seed=20)
    for fill in (0xFF, 0x7F, 0):
        torch.full((ps.binding.ps_attn_tree_workspace(c.pa.shape) + 256,), fill, dtype=torch.uint8, device="cuda")  # (freed: the call gets this memory)
        again = c.pa.run_tree(q, c.table, mask, [5000, 900], [40, 64])
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_calls_on_two_streams_at_once():
    """Calls of one pool on two streams, and two graphs replayed side by side, as a batch of many cut items uses the whole workspace."""
    import torch

    rng = np.random.default_rng(31)
    prior, nodes = rng.integers(500, 6000, 20).astype(np.int32), rng.integers(20, 64, 20).astype(np.int32)
    c = Cache(32, 8, 128, prior + nodes, seed=32).fill()
    mask, sees = tree_masks(nodes, 1, rng)
    qs = [c.normal(int(nodes.sum()), 32, 128) for _ in range(2)]
    want = [c.pa.run_tree(q, c.table, mask, prior, nodes) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(8):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(c.pa.run_tree(qs[k], c.table, mask, prior, nodes))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(x, y) for res in got[k] for x, y in zip(res, want[k]))
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = c.pa.run_tree(qs[k], c.table, mask, prior, nodes)
        graphs.append((g, res))
    for _ in range(4):
        for k in range(2):
            for x in graphs[k][1]:
                x.zero_()
        torch.cuda.synchronize()
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k][0].replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(x, y) for x, y in zip(graphs[k][1], want[k]))
    c.pa.check_pool()


def test_other_streams_and_captured_graphs():
    """A step captured whole, two graphs that take turns, and another stream than the tensors'."""
    import torch

    rng = np.random.default_rng(21)
    prior, nodes = np.array([300, 1700], dtype=np.int32), np.array([33, 60], dtype=np.int32)
    c = Cache(32, 8, 128, prior + nodes, seed=22).fill()
    mask, sees = tree_masks(nodes, 1, rng)
    qkv = c.normal(93, 48, 128)
    index = torch.tensor([[0, 4, 7], [2, 3, 50]], dtype=torch.int32, device="cuda")
    count = torch.tensor([3, 3], dtype=torch.int32, device="cuda")

    def step():
        q = c.pa.write_rope(qkv[:, :32], qkv[:, 32:40], qkv[:, 40:], c.table, prior, nodes, None)
        out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
        c.pa.accept(c.table, prior, nodes, index, count)
        k, v = c.pa.read(c.table, prior, nodes)
        return out, lse, k, v

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = step()
        graphs.append((g, res))
    for g, res in graphs + graphs[::-1]:
        for x in res:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(res, want))
    qkv.mul_(0.5)  # a graph reads its inputs as they are at its replay
    graphs[0][0].replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in graphs[0][1]]
    assert all(torch.equal(a, b) for a, b in zip(got, step())) and not torch.equal(got[0], want[0])
    c.pa.check_pool()


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 64)])
def test_waits_that_run_out(heads):
    """With a limit of zero the first wait of a CTA gives up: an error status, and the context and the pool stay usable."""
    import torch

    import paper_2507_17769_b200 as ps

    c, q, mask, out, lse = run(heads, [700, 3000], [60, 33], seed=23)
    ps.ps_kv_set_wait_limit(c.pa.kv, 0)
    c.pa.run_tree(q, c.table, mask, [700, 3000], [60, 33])
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_TIMEOUT
    ps.ps_kv_set_wait_limit(c.pa.kv, 2_000_000_000)
    again = c.pa.run_tree(q, c.table, mask, [700, 3000], [60, 33])
    c.pa.check_pool()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_one_token_is_a_decode_row():
    """Trees of one node are decode rows: run() and run_tree() agree to their bounds."""
    import torch

    prior = np.array([0, 15, 16, 300, 2000], dtype=np.int32)
    c, q, mask, out, lse = run((32, 8, 128), prior, [1] * 5, seed=24)
    c.pa.plan(prior, [1] * 5, c.table.size(1))
    ref, ref_lse = c.pa.run(q, c.table)
    c.pa.check()
    assert float((ref.float() - out.float()).abs().max()) <= 2e-2 and torch.allclose(lse, ref_lse, atol=2e-3)


def test_a_chain_is_a_chunk():
    """A chain of drafted tokens is a causal chunk."""
    import torch

    prior, nodes = np.array([500, 20], dtype=np.int32), np.array([64, 30], dtype=np.int32)
    sees = [np.tril(np.ones((n, n), dtype=bool)) for n in nodes]
    c, q, mask, out, lse = run((32, 8, 128), prior, nodes, seed=25, sees_all=sees)
    c.pa.plan(prior, nodes, c.table.size(1))
    ref, ref_lse = c.pa.run(q, c.table)
    c.pa.check()
    assert float((ref.float() - out.float()).abs().max()) <= 2e-2 and torch.allclose(lse, ref_lse, atol=2e-3)


@pytest.mark.parametrize("heads,fp8", [((32, 8, 128), False), ((32, 8, 128), True), ((8, 8, 64), False), ((4, 2, 64), False)])
@pytest.mark.parametrize("n,longest", [(1, 200), (3, 400), (9, 900), (18, 700), (18, 1500), (19, 700)])
def test_few_items_whole_or_cut(heads, fp8, n, longest):
    """Ragged batches on both sides of where items stay whole: by their count, and by their length."""
    rng = np.random.default_rng(n + longest)
    run(heads, rng.integers(0, longest, n), rng.integers(1, 65, n), seed=n, fp8=fp8)
